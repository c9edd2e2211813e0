"""The residual stream's step from block to block, and its gradients, on an MI355X against plain torch in 64 bits.

Tolerances count roundings: U = 2^-24 for one in 32 bits, half of finfo.eps for one to a tensor's type.  Every result is a sum of
products of inputs, row statistics and sums over a row; a value is off by at most (number of roundings on its longest path) U times
the same formula on absolute values with every minus a plus.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2507_13833_amd import binding
    binding.load()
    assert torch.cuda.is_available()
    return torch, binding


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def rows_of(torch, t, pad, shift):
    """The same matrix with rows `pad` elements further apart, `shift` elements into its memory, poison between the rows."""
    rows, cols = t.shape
    store = torch.full((rows * (cols + pad) + shift + 8,), math.nan, dtype=t.dtype, device=t.device)
    view = store.as_strided((rows, cols), (cols + pad, 1), shift)
    view.copy_(t)
    return view


def path(dim):
    """Roundings of a sum over a row: eight of a thread (or one in 1024 of a long row), six steps of a wave, sixteen waves."""
    return max(8, dim / 1024) + 6 + 16


def draw(torch, rows, dim, act, res, weight, post, gate, pre, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 131 + dim)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    t = types(torch)
    d = {"block": (rand(rows, dim) * torch.exp(rand(rows, 1))).to(t[act]), "residual": (rand(rows, dim) * 2).to(t[res]),
         "post": (1 + 0.3 * rand(1, dim)).to(t[weight]) if post else None, "pre": (1 + 0.3 * rand(1, dim)).to(t[weight]) if pre else None,
         "gate": {"none": None, "column": (0.5 + rand(1, dim)).to(t[weight]), "token": rand(rows, dim).to(t[act])}[gate],
         "dy": (rand(rows, dim) * 0.3).to(t[act]) if pre else None, "dh": (rand(rows, dim) * 0.3).to(t[res])}
    return d


def call_norm(env, d, rs, bs, token_gate, stat=True, out=None, res_out=None, stream=None):
    torch, B = env
    m = lambda x: None if x is None else B.make_matrix(x)  # noqa: E731
    rows, dim = d["block"].shape
    new = lambda dt: torch.full((rows, dim), -7.0, dtype=dt, device="cuda")  # noqa: E731
    res_out = new(d["residual"].dtype) if res_out is None else res_out
    out = None if d["pre"] is None else new(d["block"].dtype) if out is None else out
    st = torch.full((rows, 2), -7.0, device="cuda") if stat else None
    B.dc_residual_norm(m(d["block"]), m(d["post"]), m(d["gate"]), m(d["residual"]), m(d["pre"]),
                       B.make_norm(EPS, rs, bs, gate_rows=token_gate), m(res_out), m(out), st, stream=stream)
    return {"h": res_out, "out": out, "stat": st}


def norm_reference(torch, d, rs, bs):
    f = lambda x: None if x is None else x.double()  # noqa: E731
    b, res, post, gate, pre = (f(d[k]) for k in ("block", "residual", "post", "gate", "pre"))
    dim = b.shape[1]
    one = torch.ones((), dtype=torch.float64, device="cuda")
    gate = one if gate is None else gate
    # a root: its sum's roundings (halved by the root) and four of its own
    rel = (path(dim) / 2 + 5) * U
    r1 = (b.square().mean(1, keepdim=True) + float(torch.tensor(EPS))).rsqrt() if post is not None else None
    u = b if post is None else b * r1 * post
    branch = bs * gate * u
    h = rs * res + branch
    dh = branch.abs() * (rel + 6 * U) + (rs * res).abs() * 3 * U + h.abs() * U
    zero = torch.zeros(b.shape[0], 1, dtype=torch.float64, device="cuda")
    want, tol = {"h": h, "out": None}, {"h": dh + half_step(torch, d["residual"].dtype) * h.abs() + torch.finfo(d["residual"].dtype).tiny}
    stat, stol = [zero if r1 is None else r1], [zero if r1 is None else r1 * rel]
    if pre is not None:
        r2 = (h.square().mean(1, keepdim=True) + float(torch.tensor(EPS))).rsqrt()
        rel2 = rel + dh.square().mean(1, keepdim=True).sqrt() * r2
        want["out"] = h * r2 * pre
        tol["out"] = dh * r2 * pre.abs() + want["out"].abs() * (rel2 + 4 * U + half_step(torch, d["block"].dtype)) + torch.finfo(d["block"].dtype).tiny
        stat, stol = stat + [r2], stol + [r2 * rel2]
    else:
        stat, stol = stat + [zero], stol + [zero]
    want["stat"], tol["stat"] = torch.cat(stat, 1), torch.cat(stol, 1)
    return want, tol


def compare(torch, got, want, tol):
    for k, w in want.items():
        if w is None or got.get(k) is None:
            continue
        off = (got[k].double() - w).abs() - tol[k]
        assert float(off.max()) <= 0 if off.numel() else True, (k, float(off.max()), float(((got[k].double() - w).abs() / tol[k].clamp(min=1e-300)).max()))


def call_grad(env, d, h, stat, rs, bs, token_gate, w_grad=None, accumulate=False, into=None, stream=None):
    torch, B = env
    m = lambda x: None if x is None else B.make_matrix(x)  # noqa: E731
    rows, dim = d["block"].shape
    into = into or {}
    new = lambda dt, n=rows: torch.full((n, dim), -7.0, dtype=dt, device="cuda")  # noqa: E731
    w_grad = w_grad or torch.float32
    got = {"block": into.get("block", new(d["block"].dtype)), "residual": into.get("residual", new(h.dtype))}
    for k in ("post", "gate", "pre"):
        got[k] = None if d[k] is None else into[k] if k in into else new(d["block"].dtype) if k == "gate" and token_gate else new(w_grad, 1)
    need = B.dc_residual_norm_backward_workspace_bytes(m(d["block"]))
    ws = torch.full((max(1, need),), 0xA5, dtype=torch.uint8, device="cuda")
    got["keep"] = ws
    B.dc_residual_norm_backward(m(d["block"]), m(d["post"]), m(d["gate"]), m(h), m(d["pre"]),
                                B.make_norm(EPS, rs, bs, gate_rows=token_gate), stat, m(d["dh"]), m(d["dy"]), m(got["block"]),
                                m(got["residual"]), accumulate, m(got["post"]), m(got["gate"]), m(got["pre"]), ws, need, stream=stream)
    return got


def grad_reference(torch, d, h, stat, rs, bs, token_gate, before=None, w_grad=None):
    """Gradients from the given statistics, and the same formulas on absolute values."""
    f = lambda x: None if x is None else x.double()  # noqa: E731
    b, post, gate, pre, dy, dh0 = (f(d[k]) for k in ("block", "post", "gate", "pre", "dy", "dh"))
    rows, dim = b.shape
    r1 = stat[:, :1].double() if post is not None else 1.0
    r2 = stat[:, 1:].double() if pre is not None else 0.0
    w_grad = w_grad or torch.float32

    def formulas(size):
        a = (lambda x: x.abs()) if size else (lambda x: x)
        sign = 1.0 if size else -1.0
        g = a(gate) if gate is not None else 1.0
        p = a(post) if post is not None else 1.0
        n1 = a(b) * r1
        out = {}
        e = a(dh0)
        if pre is not None:
            n2, x = a(f(h)) * r2, a(dy) * a(pre)
            out["pre"] = (a(dy) * n2).sum(0, keepdim=True)
            e = e + r2 * (x + sign * n2 * (x * n2).mean(1, keepdim=True))
        out["residual"] = abs(rs) * e if size else rs * e
        du = (abs(bs) if size else bs) * e
        dg = du * n1 * p
        if gate is not None:
            out["gate"] = dg if token_gate else dg.sum(0, keepdim=True)
        du = du * g
        if post is not None:
            out["post"] = (du * n1).sum(0, keepdim=True)
            x = du * p
            out["block"] = r1 * (x + sign * n1 * (x * n1).mean(1, keepdim=True))
        else:
            out["block"] = du
        return out

    want, size = formulas(False), formulas(True)
    roundings = 2 * path(dim) + 30                            # one round of sums after another, and the products between them
    sums = rows / min(rows, 1024) + 4 + 64 + 16               # of a workgroup, its rows side by side, its strip, the strips
    tol = {}
    for k in want:
        one_row = k in ("post", "pre") or (k == "gate" and not token_gate)
        n = roundings + (sums if one_row else 0)
        dt = w_grad if one_row else f(h) is not None and k == "residual" and h.dtype or d["block"].dtype
        if one_row and before is not None:
            want[k] = want[k] + before[k].double()
            size[k] = size[k] + before[k].double().abs()
        tol[k] = n * U * size[k] + half_step(torch, dt) * want[k].abs() + torch.finfo(dt).tiny
    return want, tol


def check(env, rows, dim, act="bf16", res="bf16", weight="f32", post=True, gate="column", pre=True, rs=1.0, bs=1.0, pad=0, shift=0, seed=0,
          w_grad="f32"):
    torch, B = env
    d = draw(torch, rows, dim, act, res, weight, post, gate, pre, seed)
    if pad or shift:
        for k in ("block", "residual", "dy", "dh", "gate"):
            if d[k] is not None and d[k].shape[0] == rows:
                d[k] = rows_of(torch, d[k], pad, shift)
    token = gate == "token"
    got = call_norm(env, d, rs, bs, token)
    want, tol = norm_reference(torch, d, rs, bs)
    torch.cuda.synchronize()
    compare(torch, got, want, tol)
    h = rows_of(torch, got["h"], pad, shift) if pad or shift else got["h"]
    t = types(torch)
    grads = call_grad(env, d, h, got["stat"], rs, bs, token, w_grad=t[w_grad])
    want, tol = grad_reference(torch, d, h, got["stat"], rs, bs, token, w_grad=t[w_grad])
    torch.cuda.synchronize()
    compare(torch, grads, want, tol)
    return d, got, grads


DIMS = [1, 2, 7, 8, 63, 64, 65, 511, 512, 513, 1000, 2047, 2048, 2049, 2056, 4096, 4104, 5001, 8192, 8193, 20000]


@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("dim", DIMS)
def test_norm(env, rows, dim):
    check(env, rows, dim)
    check(env, rows, dim, act="f32", res="f32", gate="token", rs=0.7, bs=1.4)


@pytest.mark.parametrize("act", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("res", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("weight", ["f32", "bf16", "f16"])
def test_norm_types(env, act, res, weight):
    for dim in (120, 1337, 9000):
        check(env, 9, dim, act, res, weight, w_grad=weight)
        check(env, 9, dim, act, res, weight, gate="token", w_grad=weight)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gate", ["none", "column", "token"])
@pytest.mark.parametrize("dim", [96, 1001, 2048, 8200])
def test_norm_parts(env, dim, gate, pre, post):
    check(env, 6, dim, post=post, pre=pre, gate=gate, rs=-0.5, bs=0.25)


@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (8, 8), (3, 5), (8, 4), (24, 0)])
@pytest.mark.parametrize("act,res", [("bf16", "f32"), ("f32", "f16")])
def test_norm_strides(env, act, res, pad, shift):
    for dim in (64, 1000, 4096, 8200):
        check(env, 5, dim, act, res, gate="token", pad=pad, shift=shift)


@pytest.mark.parametrize("rows,dim,pad", [(2100, 64, (1 << 20) - 64), (600, 9000, 1 << 22)])
def test_norm_far_apart_rows(env, rows, dim, pad):
    """Rows that lie more than 4 GB apart."""
    check(env, rows, dim, gate="token", pad=pad, shift=0)


@pytest.mark.parametrize("rows,dim", [(1025, 40), (4097, 520), (3001, 2048), (1030, 4100), (300, 8192), (520, 8195)])
def test_norm_more_rows_than_workgroups(env, rows, dim):
    check(env, rows, dim)
    check(env, rows, dim, act="f32", res="f32", gate="none")


def test_norm_zero_rows_of_values(env):
    """Rows of zeros are normed to zeros by eps alone."""
    torch, B = env
    d = draw(torch, 4, 200, "f32", "f32", "f32", True, "column", True)
    d["block"][1] = 0
    d["residual"][1] = 0
    got = call_norm(env, d, 1.0, 1.0, False)
    want, tol = norm_reference(torch, d, 1.0, 1.0)
    compare(torch, got, want, tol)
    assert not got["out"][1].any() and abs(float(got["stat"][1, 0]) - EPS ** -0.5) < 1e-3


def test_norm_rows_do_not_touch_each_other(env):
    """A NaN or an infinity stays in its row (of what has rows), and the rows around it are as they are without it."""
    torch, B = env
    for dim in (100, 2048, 9000):
        d = draw(torch, 7, dim, "bf16", "f32", "f32", True, "token", True)
        clean = call_norm(env, d, 1.0, 1.0, True)
        clean_g = call_grad(env, d, clean["h"], clean["stat"], 1.0, 1.0, True)
        d["block"][3, 5], d["residual"][5, 7] = math.nan, math.inf
        got = call_norm(env, d, 1.0, 1.0, True)
        got_g = call_grad(env, d, got["h"], got["stat"], 1.0, 1.0, True)
        rest = [0, 1, 2, 4, 6]
        for a, b in ((clean["h"], got["h"]), (clean["out"], got["out"]), (clean["stat"], got["stat"]),
                     *((clean_g[k], got_g[k]) for k in ("block", "residual", "gate"))):
            assert torch.equal(a[rest], b[rest])
        assert got["out"][3].isnan().all() and not got["out"][5].isfinite().all()


@pytest.mark.parametrize("dim", [64, 2048, 2050, 9000])
def test_norm_in_place(env, dim):
    torch, B = env
    d = draw(torch, 33, dim, "bf16", "bf16", "bf16", True, "column", True)
    apart = call_norm(env, d, 0.9, 1.1, False)
    e = {k: None if v is None else v.clone() for k, v in d.items()}
    call_norm(env, e, 0.9, 1.1, False, out=e["block"], res_out=e["residual"])
    assert torch.equal(e["residual"], apart["h"]) and torch.equal(e["block"], apart["out"])
    grads = call_grad(env, d, apart["h"], apart["stat"], 0.9, 1.1, False)
    for place in ("block", "dy"):
        e = {k: None if v is None else v.clone() for k, v in d.items()}
        again = call_grad(env, e, apart["h"], apart["stat"], 0.9, 1.1, False, into={"block": e[place], "residual": e["dh"]})
        for k in ("block", "residual", "post", "gate", "pre"):
            assert torch.equal(again[k], grads[k]), (place, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [72, 1365, 8200])
def test_norm_backward_accumulates(env, dim, dtype):
    torch, B = env
    dt = types(torch)[dtype]
    for gate in ("column", "token"):
        d = draw(torch, 19, dim, "bf16", "f32", "f32", True, gate, True)
        fwd = call_norm(env, d, 1.0, 1.0, gate == "token")
        before = {k: (torch.randn(1, dim, device="cuda") * 3).to(dt) for k in (("post", "pre", "gate") if gate == "column" else ("post", "pre"))}
        got = call_grad(env, d, fwd["h"], fwd["stat"], 1.0, 1.0, gate == "token", accumulate=True, w_grad=dt, into={k: v.clone() for k, v in before.items()})
        want, tol = grad_reference(torch, d, fwd["h"], fwd["stat"], 1.0, 1.0, gate == "token", before=before, w_grad=dt)
        compare(torch, got, want, tol)


def test_norm_one_row_with_a_gate_of_its_own(env):
    """With gate_rows the gate's gradient is written, not added to, also where there is one row."""
    torch, B = env
    d = draw(torch, 1, 100, "f32", "f32", "f32", True, "token", True)
    fwd = call_norm(env, d, 1.0, 1.0, True)
    got = call_grad(env, d, fwd["h"], fwd["stat"], 1.0, 1.0, True, accumulate=True,
                    into={"post": torch.zeros(1, 100, device="cuda"), "pre": torch.zeros(1, 100, device="cuda")})
    want, tol = grad_reference(torch, d, fwd["h"], fwd["stat"], 1.0, 1.0, True)
    compare(torch, got, want, tol)


def test_norm_parts_of_the_gradient_alone(env):
    """Any gradient may be left out, and the incoming ones too; the others are the same bits."""
    torch, B = env
    d = draw(torch, 12, 700, "bf16", "f32", "f32", True, "column", True)
    fwd = call_norm(env, d, 1.0, 1.0, False)
    full = call_grad(env, d, fwd["h"], fwd["stat"], 1.0, 1.0, False)
    m = lambda x: None if x is None else B.make_matrix(x)  # noqa: E731
    need = B.dc_residual_norm_backward_workspace_bytes(m(d["block"]))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for keep in ("block", "residual", "post", "gate", "pre"):
        out = {k: torch.full_like(full[k], -7.0) if k == keep else None for k in ("block", "residual", "post", "gate", "pre")}
        B.dc_residual_norm_backward(m(d["block"]), m(d["post"]), m(d["gate"]), m(fwd["h"]), m(d["pre"]), B.make_norm(EPS), fwd["stat"],
                                    m(d["dh"]), m(d["dy"]), m(out["block"]), m(out["residual"]), False, m(out["post"]), m(out["gate"]),
                                    m(out["pre"]), ws, need)
        assert torch.equal(out[keep], full[keep]), keep
    zero = dict(d, dh=torch.zeros_like(d["dh"]))
    without = call_grad(env, dict(d, dh=None), fwd["h"], fwd["stat"], 1.0, 1.0, False)
    with_zero = call_grad(env, zero, fwd["h"], fwd["stat"], 1.0, 1.0, False)
    for k in ("block", "residual", "post", "gate", "pre"):
        assert torch.equal(without[k], with_zero[k])


def test_norm_no_rows(env):
    torch, B = env
    d = draw(torch, 0, 64, "bf16", "bf16", "f32", True, "column", True)
    fwd = call_norm(env, d, 1.0, 1.0, False)
    got = call_grad(env, d, fwd["h"], fwd["stat"], 1.0, 1.0, False)
    for k in ("post", "gate", "pre"):
        assert not got[k].any()                               # written anew: sums of nothing
    kept = torch.full((1, 64), 2.5, device="cuda")
    got = call_grad(env, d, fwd["h"], fwd["stat"], 1.0, 1.0, False, accumulate=True, into={k: kept.clone() for k in ("post", "gate", "pre")})
    for k in ("post", "gate", "pre"):
        assert torch.equal(got[k], kept)


def test_norm_backward_against_differences(env):
    """The gradients are those of the forward call: central differences of a loss along random directions, in 32 bits."""
    torch, B = env
    d = draw(torch, 5, 300, "f32", "f32", "f32", True, "column", True)
    fwd = call_norm(env, d, 0.8, 0.6, False)
    grads = call_grad(env, d, fwd["h"], fwd["stat"], 0.8, 0.6, False)

    def loss(e):
        o = call_norm(env, e, 0.8, 0.6, False)
        return float((o["h"].double() * d["dh"].double()).sum() + (o["out"].double() * d["dy"].double()).sum())

    g = torch.Generator(device="cuda").manual_seed(3)
    for name, key in (("block", "block"), ("residual", "residual"), ("post", "post"), ("gate", "gate"), ("pre", "pre")):
        along = torch.randn(d[name].shape, generator=g, device="cuda")
        step = 2.0 ** -6
        up, down = (dict(d, **{name: (d[name] + s * step * along)}) for s in (1, -1))
        diff = (loss(up) - loss(down)) / (2 * step)
        want = float((grads[key].double() * along.double()).sum())
        scale = float((grads[key].double().abs() * along.double().abs()).sum())
        # a third derivative's share step^2 / 6 of sizes around the gradient's own, and the roundings of two losses over the step
        assert abs(diff - want) <= scale * step ** 2 * 4 + 64 * U * 1500 / step * 0.05, (name, diff, want)


def test_norm_repeats_bit_for_bit_on_another_stream_and_in_a_graph(env):
    torch, B = env
    d = draw(torch, 2100, 1024, "bf16", "f32", "f32", True, "column", True)
    m = lambda x: None if x is None else B.make_matrix(x)  # noqa: E731
    first = call_norm(env, d, 1.0, 1.0, False)
    first_g = call_grad(env, d, first["h"], first["stat"], 1.0, 1.0, False)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = call_norm(env, d, 1.0, 1.0, False)
        other_g = call_grad(env, d, other["h"], other["stat"], 1.0, 1.0, False)
    s.synchronize()
    for k in ("h", "out", "stat"):
        assert torch.equal(first[k], other[k])
    for k in ("block", "residual", "post", "gate", "pre"):
        assert torch.equal(first_g[k], other_g[k])
    h, out, stat = torch.empty_like(first["h"]), torch.empty_like(first["out"]), torch.empty_like(first["stat"])
    g = {k: torch.empty_like(first_g[k]) for k in ("block", "residual", "post", "gate", "pre")}
    need = B.dc_residual_norm_backward_workspace_bytes(m(d["block"]))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    prm = B.make_norm(EPS)

    def both():
        B.dc_residual_norm(m(d["block"]), m(d["post"]), m(d["gate"]), m(d["residual"]), m(d["pre"]), prm, m(h), m(out), stat)
        B.dc_residual_norm_backward(m(d["block"]), m(d["post"]), m(d["gate"]), m(h), m(d["pre"]), prm, stat, m(d["dh"]), m(d["dy"]),
                                    m(g["block"]), m(g["residual"]), False, m(g["post"]), m(g["gate"]), m(g["pre"]), ws, need)

    with torch.cuda.stream(s):
        both()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both()
    for turn in range(4):
        fresh = draw(torch, 2100, 1024, "bf16", "f32", "f32", True, "column", True, seed=turn)
        for k, v in fresh.items():
            if v is not None:
                d[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        eager = call_norm(env, d, 1.0, 1.0, False)
        eager_g = call_grad(env, d, eager["h"], eager["stat"], 1.0, 1.0, False)
        torch.cuda.synchronize()
        assert torch.equal(h, eager["h"]) and torch.equal(out, eager["out"]) and torch.equal(stat, eager["stat"])
        for k in g:
            assert torch.equal(g[k], eager_g[k]), (turn, k)
