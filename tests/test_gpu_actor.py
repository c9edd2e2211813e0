"""The actor's update on an MI355X against plain torch in 64 bits, through the binding.

Tolerances count roundings: U = 2^-24 for one in 32 bits, half of finfo.eps for one to a tensor's type.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2507_13833_amd import binding
    binding.load()                                            # raises if libdc.so is missing: no fallback
    assert torch.cuda.is_available()
    return torch, binding


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def rows_of(torch, t, pad, shift, poison=math.nan):
    """The same matrix with rows `pad` elements further apart and the first one `shift` elements into its memory, what lies
    between the rows poisoned."""
    rows, cols = t.shape
    store = torch.full((rows * (cols + pad) + shift + 8,), poison, dtype=t.dtype, device=t.device)
    view = store.as_strided((rows, cols), (cols + pad, 1), shift)
    view.copy_(t)
    return view


# ---- log-probabilities ----

def logprob_call(env, x, temperature, token, mask, n_top, stat=True, entropy=True, stream=None):
    torch, B = env
    n, dev = x.shape[0], x.device
    new = lambda *s, dtype=torch.float32: torch.full(s, -7, dtype=dtype, device=dev)  # noqa: E731
    out = {"logprob": new(n) if token is not None else None, "stat": new(n, 2) if stat else None,
           "entropy": new(n) if entropy else None, "top_token": new(n, n_top, dtype=torch.int32) if n_top else None,
           "top_logprob": new(n, n_top) if n_top else None}
    mx = B.make_matrix(x)
    need = B.dc_token_logprob_workspace_bytes(mx, n_top)
    ws = torch.full((max(need, 1),), 0xA5, dtype=torch.uint8, device=dev)
    out["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    out["keep"] = ws
    B.dc_token_logprob(mx, temperature, token, mask, n_top, out["logprob"], out["stat"], out["entropy"], out["top_token"],
                       out["top_logprob"], ws, need, out["status"], stream=stream)
    return out


def logprob_reference(torch, x, temperature, token, mask, n_top):
    """Values in 64 bits, and by how much each may be off: z = (x - M) / T carries 3 roundings, an exponential's argument 2
    more and 2 for the exponential itself, so S is off by (5 E|z| + 3) U and, each partial sum running over at most
    vocabulary / 256 + 32 terms, by as many U again."""
    x = x.double()
    n, vocab = x.shape
    live = torch.ones(n, dtype=torch.bool, device=x.device) if mask is None else mask != 0
    top = x.max(1).values
    z = (x - top[:, None]) / temperature
    e = z.exp()
    s = e.sum(1)
    p, log_sum = e / s[:, None], s.log()
    zf = torch.where(e > 0, z, 0.0)
    ez, ez2 = (p * zf.abs()).sum(1), (p * zf * zf).sum(1)
    adds = vocab / 256 + 32
    tol_sum = U * (5 * ez + 3 + adds + 2 * log_sum.abs() + 2)
    bad = ~(s >= 1)
    want = {"stat": torch.stack([top, log_sum], 1), "entropy": log_sum + ez}
    tol = {"stat": torch.stack([torch.zeros_like(top), tol_sum], 1),
           "entropy": tol_sum + U * ((2 * adds + 8) * ez + 8 * ez2 + 2 * (log_sum + ez) + 1)}
    if token is not None:
        t = token.long().clamp(0, vocab - 1)
        zt = z.gather(1, t[:, None])[:, 0]
        want["logprob"], tol["logprob"] = zt - log_sum, tol_sum + U * (3 * zt.abs() + (zt - log_sum).abs())
        tol["logprob"] = torch.where(zt.isinf(), 0.0, tol["logprob"])
    if n_top:
        value, column = (x + 0.0).sort(dim=1, descending=True, stable=True)
        zt = (value[:, :n_top] - top[:, None]) / temperature
        want["top_token"] = column[:, :n_top].int()
        want["top_logprob"] = zt - log_sum[:, None]
        tol["top_logprob"] = torch.where(zt.isinf(), 0.0, tol_sum[:, None] + U * (3 * zt.abs() + want["top_logprob"].abs()))
    for k in ("logprob", "top_logprob"):                      # what 32 bits cannot hold is -infinity in them
        if k in want:
            want[k] = torch.where(want[k] < -torch.finfo(torch.float32).max, -math.inf, want[k])
    for k, w in want.items():
        if k == "top_token":
            w[bad] = -1
            w[~live] = -1
        else:
            w[bad] = math.nan
            w[~live] = 0.0
            tol[k][~live] = 0.0
    return want, tol


def check_logprob(env, x, temperature=1.0, token=None, mask=None, n_top=0, status=0, **kw):
    torch, B = env
    got = logprob_call(env, x, temperature, token, mask, n_top, **kw)
    want, tol = logprob_reference(torch, x, temperature, token, mask, n_top)
    torch.cuda.synchronize()
    assert int(got["status"]) == status
    for k, w in want.items():
        g = got[k]
        if g is None:
            continue
        if k == "top_token":
            assert torch.equal(g, w), (k, g[(g != w).any(1)][:2], w[(g != w).any(1)][:2])
            continue
        g = g.double()
        assert torch.equal(g.isnan(), w.isnan()), k
        inf = w.isinf()
        assert torch.equal(g[inf], w[inf]), k
        off = ((g - w).abs() - tol[k])[w.isfinite()]
        assert not off.numel() or float(off.max()) <= 0, (k, float(off.max()))
    return got


def draw_logits(torch, rows, vocab, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 31 + vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    token = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    x[torch.arange(rows), token.long()] += 5
    return x.to(dtype), token, (torch.rand(rows, generator=g, device="cuda") < 0.7).to(torch.uint8)


SHAPES = [(1, 1), (2, 2), (1, 7), (5, 63), (3, 64), (4, 65), (7, 257), (33, 1000), (3, 2047), (2, 4096), (5, 8193), (2, 32003),
          (300, 2050), (1, 152064), (3, 152064), (70, 20011), (1, 300001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprob(env, rows, vocab, dtype):
    torch, B = env
    x, token, mask = draw_logits(torch, rows, vocab, types(torch)[dtype])
    check_logprob(env, x, 1.0, token, None, 0)
    check_logprob(env, x, 0.7, token, mask, min(5, vocab))
    check_logprob(env, x, 1.0, token, None, min(64, vocab), stat=False, entropy=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (3, 5), (8, 0), (8, 4), (13, 7)])
def test_logprob_strides(env, pad, shift, dtype):
    torch, B = env
    for rows, vocab in ((9, 1001), (2, 40000), (600, 520)):
        x, token, mask = draw_logits(torch, rows, vocab, types(torch)[dtype])
        check_logprob(env, rows_of(torch, x, pad, shift), 1.3, token, mask, 20)


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("vocab", [500, 33000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprob_special_rows(env, dtype, vocab, rows):
    """Banned tokens, ties, zeros of both signs, the type's lowest value, rows without a distribution; each kind of row
    among ordinary ones."""
    torch, B = env
    dt = types(torch)[dtype]
    low = torch.finfo(dt).min
    kinds = ["one_finite", "all_banned", "nan", "inf", "nan_and_inf", "equal", "zeros", "lowest", "lowest_and_one", "large", "steps",
             "few_finite", "last_finite", "first_finite"]
    for at, kind in enumerate(kinds):
        x, token, _ = draw_logits(torch, rows, vocab, dt, seed=at)
        r, v = 1, torch.arange(vocab, device="cuda")
        if kind == "one_finite":
            x[r] = -math.inf
            x[r, vocab // 3] = -2.5
            token[r] = vocab // 3
            token[2] = vocab - 1
            x[2, vocab - 1] = -math.inf                       # a given token that is banned: -infinity
        elif kind == "all_banned":
            x[r] = -math.inf
        elif kind == "nan":
            x[r, vocab - 1] = math.nan
        elif kind == "inf":
            x[r, vocab // 2] = math.inf
        elif kind == "nan_and_inf":
            x[r, 0], x[r, 1] = math.nan, math.inf
        elif kind == "equal":
            x[r] = 1.5
        elif kind == "zeros":
            x[r] = torch.where(v % 3 == 1, 0.0, -0.0).to(dt)
        elif kind == "lowest":
            x[r] = low
        elif kind == "lowest_and_one":
            x[r] = low
            x[r, vocab - 2] = 1.0
        elif kind == "large":
            x[r] = (x[r].float() * 1000).clamp(-60000, 60000).to(dt)
        elif kind == "steps":
            x[r] = (v % 7).to(dt)                             # every value many times
        elif kind == "few_finite":
            x[r] = -math.inf
            x[r, vocab // 2], x[r, 3], x[r, vocab - 1] = 1.0, 2.0, 1.0
            token[r] = 3
        elif kind == "last_finite":
            x[r] = -math.inf
            x[r, vocab - 1] = 0.25
            token[r] = vocab - 1
        elif kind == "first_finite":
            x[r] = -math.inf
            x[r, 0] = 0.25
            token[r] = 0
        check_logprob(env, x, 1.0, token, None, 20)
        check_logprob(env, rows_of(torch, x, 1, 1), 0.5, token, None, 7)


def test_logprob_masked_rows_are_not_read(env):
    torch, B = env
    for rows, vocab in ((4, 152064), (500, 777)):
        x, token, mask = draw_logits(torch, rows, vocab, torch.bfloat16)
        mask[0], mask[rows - 1] = 0, 0
        x[mask == 0] = math.nan
        token[mask == 0] = vocab + 5                          # not an error there
        check_logprob(env, x, 1.0, token, mask, 5)
        check_logprob(env, x, 1.0, token, torch.zeros_like(mask), 5)


def test_logprob_token_outside(env):
    torch, B = env
    for bad in (-1, 777, 1 << 30, -(1 << 31)):
        x, token, _ = draw_logits(torch, 5, 777, torch.float32)
        good = logprob_call(env, x, 1.0, token, None, 3)
        token[2] = bad
        got = logprob_call(env, x, 1.0, token, None, 3)
        assert int(got["status"]) == B.DC_ERR_TOKEN_RANGE
        assert got["logprob"][2].isnan() and torch.equal(got["entropy"], good["entropy"])
        keep = torch.tensor([0, 1, 3, 4], device="cuda")
        assert torch.equal(got["logprob"][keep], good["logprob"][keep])


def test_logprob_no_rows_and_parts(env):
    torch, B = env
    x, token, _ = draw_logits(torch, 4, 3000, torch.bfloat16)
    full = logprob_call(env, x, 1.0, token, None, 9)
    only_top = logprob_call(env, x, 1.0, None, None, 9, stat=False, entropy=False)
    assert torch.equal(full["top_token"], only_top["top_token"]) and torch.equal(full["top_logprob"], only_top["top_logprob"])
    bare = logprob_call(env, x, 1.0, token, None, 0, stat=False, entropy=False)
    torch.testing.assert_close(bare["logprob"], full["logprob"], rtol=1e-5, atol=1e-5)
    none = logprob_call(env, x[:0], 1.0, token[:0], None, 3)
    torch.cuda.synchronize()
    assert int(none["status"]) == 0


def test_logprob_repeats_bit_for_bit(env):
    torch, B = env
    for rows, vocab in ((1, 152064), (130, 32000)):
        x, token, _ = draw_logits(torch, rows, vocab, torch.bfloat16)
        a, b = (logprob_call(env, x, 1.0, token, None, 20) for _ in range(2))
        for k in ("logprob", "stat", "entropy", "top_token", "top_logprob"):
            assert torch.equal(a[k], b[k]), k


def test_packed_layout_by_shifted_pointers(env):
    """Row t of the logits predicts token t + 1: token ids, masks and outputs from their second element on."""
    torch, B = env
    T, vocab = 41, 300
    x, ids, mask = draw_logits(torch, T, vocab, torch.bfloat16)
    ids = torch.randint(0, vocab, (T,), device="cuda", dtype=torch.int32)
    out, status = torch.zeros(T, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_token_logprob(B.make_matrix(x[:-1]), 1.0, ids[1:], mask[1:], 0, out[1:], None, None, None, None, None, 0, status)
    want = torch.log_softmax(x.double(), 1)[:-1].gather(1, ids[1:].long()[:, None])[:, 0] * mask[1:]
    assert int(status) == 0
    torch.testing.assert_close(out[1:].double(), want, rtol=0, atol=1e-5)


# ---- their gradient ----

def grad_inputs(torch, x, temperature, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = x.shape[0]
    z = x.double()
    m = z.max(1, keepdim=True).values
    z = (z - m) / temperature
    e = z.exp()
    s = e.sum(1)
    stat = torch.stack([m[:, 0], s.log()], 1).float()
    entropy = (s.log() - (e * torch.where(e > 0, z, 0.0)).sum(1) / s).float()
    return stat, entropy, torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda") * 0.1


def check_grad(env, x, out, temperature, token, mask, stat, entropy, gl, ge, status=0, reference=None):
    torch, B = env
    keep = x.double() if reference is None else reference     # (the logits before an update in place)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_token_logprob_backward(B.make_matrix(x), temperature, token, mask, stat, entropy if ge is not None else None, gl, ge,
                                B.make_matrix(out), st)
    torch.cuda.synchronize()
    assert int(st) == status
    n, vocab = keep.shape
    lp = (keep - stat[:, :1].double()) / temperature - stat[:, 1:].double()
    p = lp.exp()
    a = gl.double()[:, None]
    b = torch.zeros_like(a) if ge is None else ge.double()[:, None]
    h = entropy.double()[:, None]
    hot = torch.zeros_like(p)
    if token is not None:
        t = token.long()
        ok = (t >= 0) & (t < vocab)
        hot[torch.arange(n, device="cuda")[ok], t[ok]] = 1.0
    lpf = torch.where(p > 0, lp, 0.0)
    want = (a * (hot - p) - torch.where(p > 0, b * p * (lpf + h), 0.0)) / temperature
    dead = (a[:, 0] == 0) & (b[:, 0] == 0)
    if mask is not None:
        dead |= mask == 0
    want[dead] = 0.0
    # log p: 3 roundings of z, one of the difference; p: 5 |z| + |log p| + 4; the sum of terms: 6 of their magnitudes
    z = lpf.abs() + stat[:, 1:].double().abs()
    tol = U * (p * (a.abs() + b.abs() * (lpf.abs() + h)) * (7 * z + 10) + p * b.abs() * (4 * z + 2) + 6 * (a.abs() * hot)) / temperature
    # rounded once: half a step, or half the smallest step of the type near zero
    half = half_step(torch, out.dtype)
    tol = tol * (1 + half) + half * want.abs() + torch.finfo(out.dtype).smallest_normal * torch.finfo(out.dtype).eps / 2
    tol[dead] = 0.0
    off = (out.double() - want).abs() - tol
    assert not bool(out.isnan().any())
    assert float(off.max()) <= 0, float(off.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprob_backward(env, rows, vocab, dtype):
    torch, B = env
    x, token, mask = draw_logits(torch, rows, vocab, types(torch)[dtype])
    for temperature, m, with_entropy in ((1.0, None, True), (0.7, mask, False)):
        stat, entropy, gl, ge = grad_inputs(torch, x, temperature)
        check_grad(env, x, torch.full_like(x, math.nan), temperature, token, m, stat, entropy, gl, ge if with_entropy else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift,gpad,gshift", [(1, 0, 1, 0), (0, 1, 0, 1), (3, 5, 8, 0), (8, 0, 3, 5), (8, 8, 16, 8), (5, 3, 5, 3)])
def test_logprob_backward_strides(env, pad, shift, gpad, gshift, dtype):
    torch, B = env
    for rows, vocab in ((9, 1001), (3, 40000), (5, 3)):
        x, token, mask = draw_logits(torch, rows, vocab, types(torch)[dtype])
        stat, entropy, gl, ge = grad_inputs(torch, x, 1.0)
        out = rows_of(torch, torch.zeros_like(x), gpad, gshift, poison=77.0)
        store = out.as_strided((rows * (vocab + gpad) + gshift + 8,), (1,), 0)
        check_grad(env, rows_of(torch, x, pad, shift), out, 1.0, token, mask, stat, entropy, gl, ge)
        assert int((store == 77.0).sum()) >= store.numel() - rows * vocab       # nothing between the rows was written
        assert bool((store[:gshift] == 77.0).all()) and bool((store[-8:] == 77.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_logprob_backward_in_place(env, pad, shift, dtype):
    torch, B = env
    for rows, vocab in ((9, 1001), (3, 40000)):
        x, token, mask = draw_logits(torch, rows, vocab, types(torch)[dtype])
        stat, entropy, gl, ge = grad_inputs(torch, x, 1.0)
        ref = x.double()
        x = rows_of(torch, x, pad, shift)
        check_grad(env, x, x, 1.0, token, mask, stat, entropy, gl, ge, reference=ref)


def test_logprob_backward_rows_without_gradient(env):
    """Masked rows and rows whose gradients are both zero: +0, NaN logits or statistics notwithstanding; banned tokens; the
    type's lowest value; a token outside."""
    torch, B = env
    x, token, mask = draw_logits(torch, 12, 5000, torch.bfloat16)
    x[:, 100:200] = -math.inf
    x[:, 200:300] = torch.finfo(torch.bfloat16).min
    token[:] = 7
    stat, entropy, gl, ge = grad_inputs(torch, x, 1.0)
    mask[:] = 1
    mask[3], gl[4], ge[4] = 0, 0.0, 0.0
    gl[5] = 0.0
    for r in (3, 4):
        x[r], stat[r], entropy[r] = math.nan, math.nan, math.nan
    out = torch.full_like(x, math.nan)
    good = torch.tensor([i for i in range(12) if i not in (3, 4)], device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_token_logprob_backward(B.make_matrix(x), 1.0, token, mask, stat, entropy, gl, ge, B.make_matrix(out), st)
    assert int(st) == 0 and not bool(out[3].any()) and not bool(out[4].any())
    check_grad(env, x[good], torch.full_like(x[good], math.nan), 1.0, token[good], None, stat[good], entropy[good], gl[good], ge[good])
    assert not bool(out[good][:, 100:300].any())
    token[2] = 5000
    check_grad(env, x[good], torch.full_like(x[good], math.nan), 1.0, token[good], None, stat[good], entropy[good], gl[good], ge[good],
               status=B.DC_ERR_TOKEN_RANGE)
    check_grad(env, x[good], torch.full_like(x[good], math.nan), 1.0, None, None, stat[good], entropy[good], gl[good], ge[good])


def test_logprob_backward_against_differences(env):
    """The forward call's own outputs, moved by a step in one logit: (f(x + h) - f(x - h)) / 2h.  With h = 2^-6 the third
    derivative adds at most h^2 / 6 (|p'''| <= 1, times the weights' 1.5 and, for the entropy, at most 4) = 2.5e-4 and the
    outputs' roundings (8 units of 2^-24 of at most 8) / h = 2.5e-4."""
    torch, B = env
    vocab, t = 40, 1.25
    x, token, _ = draw_logits(torch, 1, vocab, torch.float32)
    a, b = 0.9, -0.6
    h = 2.0 ** -6
    moved = x.repeat(2 * vocab, 1)
    v = torch.arange(vocab, device="cuda")
    moved[v, v] += h
    moved[vocab + v, v] -= h
    f = logprob_call(env, moved, t, token.repeat(2 * vocab), None, 0)
    value = a * f["logprob"].double() + b * f["entropy"].double()
    want = (value[:vocab] - value[vocab:]) / (2 * h)
    base = logprob_call(env, x, t, token, None, 0)
    out = torch.empty_like(x)
    B.dc_token_logprob_backward(B.make_matrix(x), t, token, None, base["stat"], base["entropy"], torch.tensor([a], device="cuda"),
                                torch.tensor([b], device="cuda"), B.make_matrix(out), base["status"])
    assert float((out[0].double() - want).abs().max()) <= 5e-4


# ---- embedding ----

@pytest.mark.parametrize("w_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("o_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (1, 50, 2048), (5, 9, 7), (64, 1000, 64), (33, 100, 1000), (1000, 77, 130), (3, 5, 9001)])
def test_embedding(env, tokens, vocab, dim, w_type, o_type):
    torch, B = env
    g = torch.Generator(device="cuda").manual_seed(tokens + vocab)
    w = torch.randn(vocab, dim, generator=g, device="cuda").to(types(torch)[w_type])
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda").to(torch.int32)
    ids[tokens // 2] = -1 if tokens > 2 else ids[0]
    dt = types(torch)[o_type]
    want = w.double()[ids.long().clamp(min=0)] * float(torch.tensor(dim ** 0.5))
    want[ids < 0] = 0.0
    tol = want.abs() * (half_step(torch, dt) * (1 + U) + 2 * U) + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps / 2
    for wp, ws, op, os_ in ((0, 0, 0, 0), (1, 1, 0, 0), (0, 0, 3, 1), (8, 0, 16, 8), (3, 5, 3, 5)):
        src = rows_of(torch, w, wp, ws)
        out = rows_of(torch, torch.zeros(tokens, dim, dtype=dt, device="cuda"), op, os_, poison=55.0)
        store = out.as_strided((tokens * (dim + op) + os_ + 8,), (1,), 0)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.dc_embedding(B.make_matrix(src), ids, dim ** 0.5, B.make_matrix(out), st)
        torch.cuda.synchronize()
        assert int(st) == 0
        assert bool(((out.double() - want).abs() <= tol).all())
        assert bool((store[:os_] == 55.0).all()) and bool((store[-8:] == 55.0).all())
        if op:
            gaps = store[os_:os_ + tokens * (dim + op)].view(tokens, dim + op)[:, dim:]
            assert bool((gaps == 55.0).all())


def test_embedding_outside_and_empty(env):
    torch, B = env
    w = torch.ones(10, 64, device="cuda")
    for bad in (10, -2, 1 << 30):
        ids = torch.tensor([3, bad, 9, -1], dtype=torch.int32, device="cuda")
        out, st = torch.full((4, 64), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        B.dc_embedding(B.make_matrix(w), ids, 2.0, B.make_matrix(out), st)
        assert int(st) == B.DC_ERR_TOKEN_RANGE
        assert out[:, 0].tolist() == [2.0, 0.0, 2.0, 0.0]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_embedding(B.make_matrix(w), ids[:0], 2.0, B.make_matrix(w[:0]), st)
    empty = torch.empty(0, 64, device="cuda")
    out = torch.full((2, 64), 9.0, device="cuda")
    B.dc_embedding(B.make_matrix(empty), torch.tensor([-1, -1], dtype=torch.int32, device="cuda"), 2.0, B.make_matrix(out), st)
    assert int(st) == 0 and not bool(out.any())


# ---- its gradient ----

def embedding_grad_call(env, g, ids, scale, accumulate, dw, status=0):
    torch, B = env
    mg, mw = B.make_matrix(g), B.make_matrix(dw)
    need = B.dc_embedding_backward_workspace_bytes(mg, mw)
    ws = torch.full((max(need, 1),), 0xA5, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_embedding_backward(mg, ids, scale, accumulate, mw, ws, need, st)
    torch.cuda.synchronize()
    assert int(st) == status


def check_embedding_grad(env, g, ids, scale, accumulate, dw, status=0):
    torch, B = env
    before = dw.double()
    vocab, dim = dw.shape
    s = float(torch.tensor(scale))                            # the factor as the kernel has it, in 32 bits
    ok = (ids >= 0) & (ids < vocab)
    gd, t = g.double()[ok], ids.long()[ok]
    total = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, t, gd)
    size = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, t, gd.abs())
    count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, t, torch.ones_like(t, dtype=torch.float64))
    want = total * s + (before if accumulate else 0.0)
    half = half_step(torch, dw.dtype)
    tol = U * s * size * (count[:, None] + 2) * 1.01 + (half + 2 * U) * want.abs() * 1.01 + torch.finfo(dw.dtype).smallest_normal * torch.finfo(dw.dtype).eps / 2
    embedding_grad_call(env, g, ids, scale, accumulate, dw, status)
    got = dw.double()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    absent = count == 0
    assert torch.equal(got[absent], before[absent] if accumulate else torch.zeros_like(got[absent]))


GRADS = [(1, 1, 1), (1, 50, 2048), (0, 20, 33), (5, 9, 7), (64, 1000, 64), (333, 100, 1000), (3000, 77, 130), (3, 5, 9001), (5000, 152064, 8),
         (9000, 3, 70), (20000, 1, 65), (70000, 500, 9), (131072, 30000, 4)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("g_type,w_type", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,vocab,dim", GRADS)
def test_embedding_backward(env, tokens, vocab, dim, g_type, w_type, accumulate):
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(tokens + vocab)
    g = (torch.randn(tokens, dim, generator=gen, device="cuda") * 0.1).to(types(torch)[g_type])
    ids = (torch.rand(tokens, generator=gen, device="cuda").double() ** 3 * vocab).int()
    ids[tokens // 3:tokens // 3 + 2] = -1                     # places without a token
    dw = torch.randn(vocab, dim, generator=gen, device="cuda").to(types(torch)[w_type])
    check_embedding_grad(env, g, ids, 1.5, accumulate, dw)


@pytest.mark.parametrize("pattern", ["same", "ascending", "descending", "two", "blocks", "none"])
def test_embedding_backward_orders(env, pattern):
    torch, B = env
    tokens, vocab, dim = 12345, 4000, 40
    at = torch.arange(tokens, device="cuda")
    ids = {"same": at * 0 + 1234, "ascending": at * vocab // tokens, "descending": vocab - 1 - at * vocab // tokens,
           "two": (at % 2) * (vocab - 1), "blocks": (at // 64) % vocab, "none": at * 0 - 1}[pattern].int()
    g = torch.randn(tokens, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    for accumulate in (False, True):
        check_embedding_grad(env, g, ids, 1.0, accumulate, torch.ones(vocab, dim, device="cuda"))


@pytest.mark.parametrize("gpad,gshift,wpad,wshift", [(1, 0, 0, 0), (0, 1, 1, 1), (8, 8, 4, 4), (3, 5, 2, 3)])
def test_embedding_backward_strides(env, gpad, gshift, wpad, wshift):
    torch, B = env
    for tokens, vocab, dim in ((500, 60, 200), (40, 300, 1025)):
        gen = torch.Generator(device="cuda").manual_seed(5)
        g = torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
        ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda").int()
        for accumulate in (False, True):
            dw = rows_of(torch, torch.ones(vocab, dim, device="cuda"), wpad, wshift, poison=33.0)
            store = dw.as_strided((vocab * (dim + wpad) + wshift + 8,), (1,), 0)
            check_embedding_grad(env, rows_of(torch, g, gpad, gshift), ids, 0.5, accumulate, dw)
            assert bool((store[:wshift] == 33.0).all()) and bool((store[-8:] == 33.0).all())
            if wpad:
                assert bool((store[wshift:wshift + vocab * (dim + wpad)].view(vocab, dim + wpad)[:, dim:] == 33.0).all())


def test_embedding_backward_outside(env):
    torch, B = env
    g = torch.randn(700, 24, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    for bad in (50, -2, 1 << 30, -(1 << 31)):
        ids = torch.randint(0, 50, (700,), device="cuda", dtype=torch.int32)
        ids[13] = bad
        check_embedding_grad(env, g, ids, 1.0, False, torch.ones(50, 24, device="cuda"), status=B.DC_ERR_TOKEN_RANGE)


def test_embedding_backward_repeats_bit_for_bit(env):
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(9)
    g = torch.randn(30000, 72, generator=gen, device="cuda").bfloat16()
    ids = (torch.rand(30000, generator=gen, device="cuda") ** 4 * 5000).int()
    a, b = torch.empty(5000, 72, device="cuda"), torch.empty(5000, 72, device="cuda")
    embedding_grad_call(env, g, ids, 1.0, False, a)
    embedding_grad_call(env, g, ids, 1.0, False, b)
    assert torch.equal(a, b)


def test_embedding_backward_against_differences(env):
    """dL for L = <forward(W), R>: linear in W, so a difference is exact but for roundings (at most 80 tokens of one id,
    values below 8, sums below 640: 640 * 80 * 2^-24 / 2h with h = 1 is 1.6e-3)."""
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(4)
    vocab, dim, tokens = 6, 5, 80
    w = torch.randn(vocab, dim, generator=gen, device="cuda")
    r = torch.randn(tokens, dim, generator=gen, device="cuda")
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda").int()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def loss(w):
        out = torch.empty(tokens, dim, device="cuda")
        B.dc_embedding(B.make_matrix(w), ids, 1.75, B.make_matrix(out), st)
        return (out.double() * r.double()).sum()
    dw = torch.empty_like(w)
    embedding_grad_call(env, r, ids, 1.75, False, dw)
    for v, c in ((0, 0), (3, 4), (5, 2)):
        up, down = w.clone(), w.clone()
        up[v, c] += 1.0
        down[v, c] -= 1.0
        assert abs(float(loss(up) - loss(down)) / 2 - float(dw[v, c])) <= 1.6e-3


# ---- AdamW ----

def adamw_tensors(torch, sizes, param, grad, master, state, seed=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = types(torch)
    items = []

    def own(x, dtype):                                        # `shift` elements into its memory
        store = torch.zeros(x.numel() + shift + 8, dtype=dtype, device="cuda")
        store[shift:shift + x.numel()] = x.to(dtype)
        return store[shift:shift + x.numel()]
    for i, n in enumerate(sizes):
        w = torch.randn(n, generator=gen, device="cuda")
        it = dict(param=own(w, t[param]), master=own(w, torch.float32) if master else None,
                  grad=own(torch.randn(n, generator=gen, device="cuda") * 10.0 ** (i % 3 - 1), t[grad]), weight_decay=0.1 * (i % 2))
        m, v = torch.randn(n, generator=gen, device="cuda") * 0.1, torch.randn(n, generator=gen, device="cuda") ** 2
        if state == 32:
            it |= dict(exp_avg=own(m, torch.float32), exp_avg_sq=own(v, torch.float32))
        else:
            blocks = -(-n // 256)
            it |= dict(exp_avg=own(m.clamp(-0.4, 0.4) * 1000, torch.float8_e4m3fn), exp_avg_sq=own(v.sqrt().clamp(max=4) * 100, torch.float8_e4m3fn),
                       exp_avg_scale=torch.rand(blocks, generator=gen, device="cuda") * 0.01,
                       exp_avg_sq_scale=torch.rand(blocks, generator=gen, device="cuda") * 0.01)
        items.append(it)
    return items


def snapshot(it):
    return {k: (v.clone() if hasattr(v, "clone") else v) for k, v in it.items()}


def adamw_call(env, items, prm, grad_scale=None, status=0):
    torch, B = env
    ts = B.AdamwTensors(items)
    need = B.dc_adamw_table_bytes(ts)
    table = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_adamw_table(ts, table, need)
    B.dc_adamw(ts, prm, grad_scale, table, need, st)
    torch.cuda.synchronize()
    assert int(st) == status
    return ts, table, need, st


def spread(torch, scale, n):
    return scale.double().repeat_interleave(256)[:n]


def check_adamw(torch, before, after, prm, grad_scale):
    n = before["param"].numel()
    if n == 0:
        return
    small = before["exp_avg"].dtype == torch.float8_e4m3fn
    g = before["grad"].double() * grad_scale
    m, v = before["exp_avg"].double(), before["exp_avg_sq"].double()
    if small:
        m, v = m * spread(torch, before["exp_avg_scale"], n), (v * spread(torch, before["exp_avg_sq_scale"], n)) ** 2
    m_size = (prm.beta1 * m).abs() + ((1 - prm.beta1) * g).abs()
    g2 = torch.where(g.abs() < 2.0 ** -75, 0.0, g * g)        # a square that 32 bits cannot hold is zero in them
    m, v = prm.beta1 * m + (1 - prm.beta1) * g, prm.beta2 * v + (1 - prm.beta2) * g2
    root = v.sqrt()
    # m: the factor's rounding, its product's and the state's decoding, the sum's: 5; v one more for the square: 7; a root halves
    tol_m, tol_v = 5 * U * m_size, 7 * U * v
    bc1, bc2 = 1 - prm.beta1 ** prm.step, 1 - prm.beta2 ** prm.step
    denom = root / math.sqrt(bc2) + prm.eps
    w = (before["param"] if before["master"] is None else before["master"]).double()
    kept, move = w * (1 - prm.lr * before["weight_decay"]), prm.lr / bc1 * m / denom
    want = kept - move
    # the move: m's own error, the denominator's (4.5 + 3), the quotient, the factor twice
    tol_w = 2 * U * kept.abs() + (prm.lr / bc1) * tol_m / denom + 12 * U * move.abs() + U * want.abs()
    if before["master"] is not None:
        assert bool(((after["master"].double() - want).abs() <= tol_w).all())
        assert torch.equal(after["param"], after["master"].to(after["param"].dtype))
    else:
        half = half_step(torch, after["param"].dtype)
        least = torch.finfo(after["param"].dtype).smallest_normal * torch.finfo(after["param"].dtype).eps / 2
        assert bool(((after["param"].double() - want).abs() <= tol_w * (1 + half) + half * want.abs() + least).all())
    if not small:
        assert bool(((after["exp_avg"].double() - m).abs() <= tol_m).all())
        assert bool(((after["exp_avg_sq"].double() - v).abs() <= tol_v).all())
        return
    for name, x, tol in (("exp_avg", m, tol_m), ("exp_avg_sq", root, 4.5 * U * root)):
        got_scale = after[name + "_scale"].double()
        pad = torch.zeros(len(got_scale) * 256, dtype=torch.float64, device="cuda")
        pad[:n] = x.abs()
        top = pad.view(-1, 256).amax(1) / 448
        assert bool(((got_scale - top).abs() <= 8 * U * top).all())
        s = spread(torch, after[name + "_scale"], n)
        off = (after[name].double() * s - x).abs() - tol - 4 * U * x.abs()
        step = torch.maximum(x.abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 16 * U)       # half a step of e4m3, normal and subnormal
        if name == "exp_avg_sq":
            step = torch.where(x < s * 2.0 ** -9, s * 2.0 ** -9, step)                 # kept from becoming zero
            assert bool((after[name].double()[(x > 0) & (s > 0)] > 0).all())
        assert bool((off <= step).all()), (name, float((off - step).max()))
        assert not bool(after[name].float().isnan().any())


SIZES = [1, 5, 255, 256, 257, 0, 1000, 2048, 2049, 4096, 40003, 3]


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("param,grad,master", [("f32", "f32", False), ("bf16", "bf16", True), ("bf16", "bf16", False), ("f16", "f32", True),
                                               ("f16", "f16", False), ("bf16", "f32", True), ("f32", "bf16", False), ("f32", "f32", True)])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_adamw(env, param, grad, master, state, shift):
    torch, B = env
    items = adamw_tensors(torch, SIZES, param, grad, master, state, shift=shift)
    gs = torch.tensor([0.5], device="cuda")
    for step, scale in ((1, None), (7, gs)):
        before = [snapshot(it) for it in items]
        prm = B.make_adamw(1e-2, 0.9, 0.99, 1e-8, step)
        adamw_call(env, items, prm, scale)
        for b, a in zip(before, items):
            check_adamw(torch, b, a, prm, 1.0 if scale is None else 0.5)
            assert torch.equal(a["grad"], b["grad"])


def test_adamw_tensors_of_different_kinds_together(env):
    torch, B = env
    items = (adamw_tensors(torch, [700, 3000], "bf16", "bf16", True, 8) + adamw_tensors(torch, [33, 5000], "f32", "f32", False, 32)
             + adamw_tensors(torch, [1] * 100, "bf16", "f32", True, 32))
    before = [snapshot(it) for it in items]
    prm = B.make_adamw(3e-3, step=3)
    adamw_call(env, items, prm)
    for b, a in zip(before, items):
        check_adamw(torch, b, a, prm, 1.0)


def test_adamw_from_nothing_and_zero_gradients(env):
    """States that are all zero, gradients that are zero or tiny in whole blocks: no NaN, nothing moves without a gradient."""
    torch, B = env
    n = 2000
    for state in (8, 32):
        it = adamw_tensors(torch, [n], "f32", "f32", False, state)[0]
        for k in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"):
            if it.get(k) is not None:
                it[k].zero_()
        it["grad"][:600] = 0.0
        it["grad"][600:1100] = 1e-30
        before = snapshot(it)
        prm = B.make_adamw(1e-2, step=1)
        adamw_call(env, [it], prm)
        check_adamw(torch, before, it, prm, 1.0)
        assert torch.equal(it["param"][:512], before["param"][:512])
        for k in ("exp_avg", "exp_avg_sq"):
            assert not bool(it[k].float()[:512].any())


def test_adamw_follows_torch(env):
    """Thirty steps in 32 bits beside torch.optim.AdamW in 64: each step's roundings, at most 20 U of a weight of about 1,
    add up."""
    torch, B = env
    it = adamw_tensors(torch, [5000], "f32", "f32", False, 32)[0]
    it["exp_avg"].zero_(), it["exp_avg_sq"].zero_()
    it["weight_decay"] = 0.1
    p = torch.nn.Parameter(it["param"].double().clone())
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    ts = B.AdamwTensors([it])
    need = B.dc_adamw_table_bytes(ts)
    table, st = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_adamw_table(ts, table, need)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for step in range(1, 31):
        it["grad"].copy_(torch.randn(5000, generator=gen, device="cuda"))
        p.grad = it["grad"].double()
        opt.step()
        B.dc_adamw(ts, B.make_adamw(1e-2, 0.9, 0.95, 1e-8, step), None, table, need, st)
    assert int(st) == 0
    assert float((it["param"].double() - p.detach()).abs().max()) <= 30 * 20 * U * 4


def test_adamw_refuses_another_table(env):
    torch, B = env
    items = adamw_tensors(torch, [3000, 5000], "f32", "f32", False, 32)
    ts, table, need, st = adamw_call(env, items, B.make_adamw(1e-3))
    other = B.AdamwTensors(items[:1])
    before = snapshot(items[0])
    B.dc_adamw(other, B.make_adamw(1e-3), None, table, need, st)
    torch.cuda.synchronize()
    assert int(st) == B.DC_ERR_BAD_LAYOUT
    assert torch.equal(before["param"], items[0]["param"]) and torch.equal(before["exp_avg"], items[0]["exp_avg"])
    empty = B.AdamwTensors([])
    adamw_call(env, [], B.make_adamw(1e-3))
    assert B.dc_adamw_table_bytes(empty) > 0


def test_adamw_repeats_bit_for_bit(env):
    torch, B = env
    a, b = (adamw_tensors(torch, SIZES, "bf16", "bf16", True, 8, seed=3) for _ in range(2))
    for items in (a, b):
        adamw_call(env, items, B.make_adamw(1e-3, step=2))
    for x, y in zip(a, b):
        for k in ("param", "master", "exp_avg_scale", "exp_avg_sq_scale"):
            assert torch.equal(x[k], y[k])
        for k in ("exp_avg", "exp_avg_sq"):
            assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8))


# ---- streams and graphs ----

def test_another_stream_and_a_graph(env):
    """All calls on a stream of their own, then captured and replayed over changed inputs, eager work between the replays."""
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(6)
    T, vocab, dim = 300, 2000, 96
    w = torch.randn(vocab, dim, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, vocab, (T,), generator=gen, device="cuda").int()
    logits = torch.randn(T, vocab, generator=gen, device="cuda").bfloat16()
    gl = torch.randn(T, generator=gen, device="cuda")
    out, dw = torch.empty(T, dim, device="cuda", dtype=torch.bfloat16), torch.empty(vocab, dim, device="cuda")
    lp, stat, h = torch.empty(T, device="cuda"), torch.empty(T, 2, device="cuda"), torch.empty(T, device="cuda")
    tt, tl = torch.empty(T, 5, device="cuda", dtype=torch.int32), torch.empty(T, 5, device="cuda")
    one_lp, one_tt, one_tl = torch.empty(1, device="cuda"), torch.empty(1, 5, device="cuda", dtype=torch.int32), torch.empty(1, 5, device="cuda")
    wide = torch.randn(1, 100000, generator=gen, device="cuda")
    dlogits = torch.empty_like(logits)
    items = adamw_tensors(torch, [5000, 33], "bf16", "bf16", True, 8)
    ts = B.AdamwTensors(items)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    sizes = {"lp": B.dc_token_logprob_workspace_bytes(B.make_matrix(logits), 5), "one": B.dc_token_logprob_workspace_bytes(B.make_matrix(wide), 5),
             "eg": B.dc_embedding_backward_workspace_bytes(B.make_matrix(out), B.make_matrix(dw)), "aw": B.dc_adamw_table_bytes(ts)}
    ws = {k: torch.full((max(n, 1),), 0x5A, dtype=torch.uint8, device="cuda") for k, n in sizes.items()}
    B.dc_adamw_table(ts, ws["aw"], sizes["aw"])

    def step():
        B.dc_embedding(B.make_matrix(w), ids, 2.0, B.make_matrix(out), st)
        B.dc_token_logprob(B.make_matrix(logits), 1.0, ids, None, 5, lp, stat, h, tt, tl, ws["lp"], sizes["lp"], st)
        B.dc_token_logprob(B.make_matrix(wide), 1.0, ids[:1], None, 5, one_lp, None, None, one_tt, one_tl, ws["one"], sizes["one"], st)
        B.dc_token_logprob_backward(B.make_matrix(logits), 1.0, ids, None, stat, h, gl, gl, B.make_matrix(dlogits), st)
        B.dc_embedding_backward(B.make_matrix(out), ids, 2.0, False, B.make_matrix(dw), ws["eg"], sizes["eg"], st)
        B.dc_adamw(ts, B.make_adamw(1e-2, step=4), None, ws["aw"], sizes["aw"], st)

    state0 = [snapshot(it) for it in items]

    def reset():
        for it, b in zip(items, state0):
            for k, v in b.items():
                if hasattr(v, "copy_"):
                    it[k].copy_(v)

    def results():
        torch.cuda.synchronize()
        assert int(st) == 0
        r = [x.clone() for x in (out, lp, stat, h, tt, tl, one_lp, one_tt, one_tl, dlogits, dw)]
        return r + [it[k].clone().view(torch.uint8) for it in items for k in ("param", "master", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")]

    inputs = [(logits.clone(), ids.clone(), wide.clone()), (logits.flip(1).contiguous(), ids.flip(0).contiguous(), wide * -1)]

    def use(k):
        logits.copy_(inputs[k][0]), ids.copy_(inputs[k][1]), wide.copy_(inputs[k][2])
        reset()
        torch.cuda.synchronize()

    want = []
    for k in range(2):
        use(k)
        step()
        want.append(results())
    side = torch.cuda.Stream()
    use(0)
    with torch.cuda.stream(side):
        step()
    for a, b in zip(results(), want[0]):
        assert torch.equal(a, b)
    use(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for k in (1, 0, 0, 1):
        use(k)
        for x in (out, lp, dw, dlogits, tt):
            x.fill_(7)
        graph.replay()
        for a, b in zip(results(), want[k]):
            assert torch.equal(a, b)
        step()                                                # eager work between the replays
        torch.cuda.synchronize()


# ---- places that 32 bits do not reach, more rows than a launch has workgroups ----

def test_rows_far_apart(env):
    """Rows 2^31 elements apart: every place is computed in 64 bits."""
    torch, B = env
    far, vocab = 1 << 31, 3001
    store = torch.empty(3 * far, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((3, vocab), (far, 1), 0)
    v, token, _ = draw_logits(torch, 3, vocab, torch.bfloat16)
    x.copy_(v)
    check_logprob(env, x, 1.0, token, None, 5)
    stat, entropy, gl, ge = grad_inputs(torch, x, 1.0)
    ref = x.double()
    check_grad(env, x, x, 1.0, token, None, stat, entropy, gl, ge, reference=ref)
    x.copy_(v)
    dense = v.contiguous()
    ids = torch.tensor([2, 0, 1, 2], dtype=torch.int32, device="cuda")
    out, st = torch.empty(4, vocab, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_embedding(B.make_matrix(x), ids, 1.0, B.make_matrix(out), st)
    assert torch.equal(out, dense[ids.long()])
    B.dc_embedding(B.make_matrix(dense), ids[:3], 1.0, B.make_matrix(x), st)
    assert torch.equal(x, dense[ids[:3].long()])
    g = torch.randn(4, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    check_embedding_grad(env, g, ids, 1.0, False, x)
    x.copy_(v)
    check_embedding_grad(env, x, ids[:3], 1.0, True, torch.ones(3, vocab, device="cuda"))
    assert int(st) == 0


def test_more_rows_than_workgroups(env):
    torch, B = env
    rows, vocab = (1 << 20) + 77, 3
    x, token, mask = draw_logits(torch, rows, vocab, torch.bfloat16)
    check_logprob(env, x, 1.0, token, mask, 2)
    stat, entropy, gl, ge = grad_inputs(torch, x, 1.0)
    check_grad(env, x, torch.full_like(x, math.nan), 1.0, token, mask, stat, entropy, gl, ge)


@pytest.mark.parametrize("vocab", [1, 4, 9000, 1 << 24])
def test_embedding_backward_many_tokens(env, vocab):
    """More tokens than one level of merges takes, ids of one to three digits."""
    torch, B = env
    tokens, dim = 300007, 2
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    g = torch.randn(tokens, dim, generator=gen, device="cuda")
    ids = (torch.rand(tokens, generator=gen, device="cuda").double() ** 2 * vocab).int().clamp_(max=vocab - 1)
    check_embedding_grad(env, g, ids, 1.0, False, torch.ones(vocab, dim, device="cuda"))


@pytest.mark.parametrize("tokens", [15, 16, 17, 18, 33, 289, 290])
def test_embedding_backward_rows_below_the_lowest_token(env, tokens):
    """Rows of the table that lie before all tokens, and rows between two, sought among so few that the searches of one wave
    end at different steps."""
    torch, B = env
    g = torch.randn(tokens, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(tokens))
    for base in (0, 1, 2, 3, 50):
        ids = (base + 2 * torch.arange(tokens, device="cuda")).int()
        check_embedding_grad(env, g, ids, 1.0, False, torch.ones(60 + 2 * tokens, 8, device="cuda"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(2, 700), (2, 152064), (300, 33000)])
@pytest.mark.parametrize("at", [1.1e7, 3e8, 2.5e9, -2.5e9, -1e10, 7e15, -3e22, 1e30, -1e35])
def test_logprob_of_far_logits(env, at, rows, vocab, dtype):
    """A row around a large value, and one of such values and a single ordinary logit."""
    torch, B = env
    dt = types(torch)[dtype]
    x, token, _ = draw_logits(torch, rows, vocab, dt)
    near = torch.tensor(at, device="cuda").to(dt)
    x[0] = near
    x[0, ::3] = torch.nextafter(near, torch.zeros_like(near))
    x[0, vocab // 2:] = -abs(at) * 1.5
    x[1] = -abs(at)
    x[1, vocab - 3] = 2.0
    check_logprob(env, x, 1.0, token, None, 9)
    check_logprob(env, x, 1e-3, token, None, 0)


def test_logprob_of_far_logits_in_one_long_row(env):
    """Many masked logits before an ordinary one in the same thread: their sum is taken over before it is left behind."""
    torch, B = env
    rows, vocab = 257, 1 << 20
    x = torch.full((rows, vocab), -1e35, dtype=torch.bfloat16, device="cuda")
    x[:, -5:] = torch.tensor([1.0, 2.0, 0.5, -1.0, 0.25], device="cuda").bfloat16()
    token = torch.full((rows,), vocab - 4, dtype=torch.int32, device="cuda")
    check_logprob(env, x, 1.0, token, None, 3)


@pytest.mark.parametrize("w_type", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1), (8, 8)])
@pytest.mark.parametrize("tokens,vocab,dim", [(0, 100001, 520), (1, 100001, 1000), (700, 152064, 1024), (30000, 152064, 1023), (100003, 152064, 515),
                                              (140000, 60000, 520)])
def test_embedding_backward_rows_without_a_token(env, tokens, vocab, dim, pad, shift, w_type):
    """Tables of which most rows have no token: +0 in every one, nothing between them touched, exact sums (whole numbers) in
    the others."""
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim)
    g = torch.randint(-1, 2, (tokens, dim), generator=gen, device="cuda").bfloat16()
    ids = (torch.rand(tokens, generator=gen, device="cuda").double() ** 2 * vocab).int().clamp_(max=vocab - 1)
    if tokens > 100:
        ids[::97], ids[3] = -1, 0
        ids[ids % 1000 == 77] = vocab - 1                     # many of one id, the table's last
    dt = types(torch)[w_type]
    store = torch.full((vocab * (dim + pad) + shift + 8,), 77.0, dtype=dt, device="cuda")
    dw = store.as_strided((vocab, dim), (dim + pad, 1), shift)
    dw.fill_(math.nan)
    embedding_grad_call(env, g, ids, 1.0, False, dw)
    ok = ids >= 0
    want = torch.zeros(vocab, dim, device="cuda").index_add_(0, ids[ok].long(), g[ok].float())
    assert torch.equal(dw, want.to(dt))
    assert bool((store[:shift] == 77.0).all()) and bool((store[-8:] == 77.0).all())
    if pad:
        assert bool((store[shift:shift + vocab * (dim + pad)].view(vocab, dim + pad)[:, dim:] == 77.0).all())


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tokens", [1, 2, 8, 9, 63, 64, 65, 129, 511, 1000, 1023, 1024, 1025])
def test_embedding_backward_few_tokens(env, tokens, accumulate):
    """On both sides of the sizes that one launch takes: all of one id, an id many times among others, ids once each."""
    torch, B = env
    vocab, dim = 1500, 600
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    at = torch.arange(tokens, device="cuda")
    for ids in (at * 0 + 7, torch.where(at % 3 == 0, 1499, at), at, torch.where(at % 5 == 0, -1, at // 9)):
        g = torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
        check_embedding_grad(env, g, ids.int(), 1.5, accumulate, torch.ones(vocab, dim, device="cuda"))
        check_embedding_grad(env, rows_of(torch, g, 1, 1), ids.int(), 1.5, accumulate, torch.ones(vocab, dim, device="cuda").bfloat16())


@pytest.mark.parametrize("tokens", [15, 16, 17, 33])
def test_embedding_backward_widest_rows(env, tokens):
    """Rows of DC_MAX_DIM columns: few tokens, and those that are too many workgroups for one launch."""
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    for dim in (B.DC_MAX_DIM, B.DC_MAX_DIM - 3):
        g = torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
        for ids in (torch.arange(tokens, device="cuda") * 0 + 3, torch.arange(tokens, device="cuda") % 7 - 1):
            for accumulate in (False, True):
                check_embedding_grad(env, g, ids.int(), 1.0, accumulate, torch.ones(40, dim, device="cuda"))


@pytest.mark.parametrize("n,shift", [(2048, 0), (1000, 0), (1000, 3)])
@pytest.mark.parametrize("grad,master", [("f32", False), ("bf16", True)])
@pytest.mark.parametrize("most", [1e20, 1e30, 3e38])
def test_adamw_finite_gradients_whose_squares_are_not(env, most, grad, master, n, shift):
    """In 8 bits the second moment is kept as its root: a finite gradient whose square is beyond 32 bits leaves finite states
    and weights, and what 64 bits make of it, in that step and in those behind it."""
    torch, B = env
    it = adamw_tensors(torch, [n], "bf16" if master else "f32", grad, master, 8, seed=4, shift=shift)[0]
    gen = torch.Generator(device="cuda").manual_seed(5)
    for step in range(1, 5):
        it["grad"].copy_(torch.randn(n, generator=gen, device="cuda"))
        if step < 3:
            it["grad"][[5, 300, n - 1]] = torch.tensor([most, -most, most / 3], device="cuda").to(it["grad"].dtype)
        before = snapshot(it)
        prm = B.make_adamw(1e-2, 0.9, 0.95, 1e-8, step)
        adamw_call(env, [it], prm)
        for k in ("param", "master", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"):
            assert it[k] is None or bool(it[k].float().isfinite().all()), (step, k)
        check_adamw(torch, before, it, prm, 1.0)


@pytest.mark.parametrize("beta2,steps", [(0.95, 400), (0.97, 600), (0.98, 600), (0.99, 1000), (0.999, 6000)])
def test_adamw_8_bit_second_moment_follows(env, beta2, steps):
    """Many steps with 8-bit states beside the second moment in 64 bits: at a sixth of the steps the gradients of every other
    element fall to a tenth, and the kept roots have to fall with them.  A root moves by about (1 - beta2) / 2 of itself in a
    step, the block's scale by as much; rounded by chance to codes at most 1/8 apart each move adds at most its own size times
    1/8 to the variance, and a step takes 1 - beta2 of what there is off: a relative variance of at most 1/16.  A median is
    off by no more than the mean's bias of that size twice, 5 of 100 by no more than two deviations."""
    torch, B = env
    n, gen = 64 * 256, torch.Generator(device="cuda").manual_seed(9)
    it = dict(param=torch.zeros(n, device="cuda"), master=None, grad=torch.empty(n, device="cuda"),
              exp_avg=torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), exp_avg_scale=torch.zeros(n // 256, device="cuda"),
              exp_avg_sq=torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), exp_avg_sq_scale=torch.zeros(n // 256, device="cuda"))
    ts = B.AdamwTensors([it])
    need = B.dc_adamw_table_bytes(ts)
    table, st = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_adamw_table(ts, table, need)
    v = torch.zeros(n, dtype=torch.float64, device="cuda")
    for step in range(1, steps + 1):
        it["grad"].normal_(generator=gen)
        if step > steps // 6:
            it["grad"][1::2] *= 0.1
        v.mul_(beta2).add_(it["grad"].double() ** 2, alpha=1 - beta2)
        B.dc_adamw(ts, B.make_adamw(1e-3, 0.9, beta2, 1e-8, step), None, table, need, st)
    ratio = it["exp_avg_sq"].double() * spread(torch, it["exp_avg_sq_scale"], n) / v.sqrt()
    assert int(st) == 0
    for part in (ratio[1::2], ratio[0::2]):
        low, mid, high = part.quantile(torch.tensor([0.05, 0.5, 0.95], dtype=torch.float64, device="cuda")).tolist()
        assert abs(mid - 1) <= 2 / 16 and low >= 0.5 and high <= 1.5 + 2 / 16, (beta2, low, mid, high)


@pytest.mark.parametrize("shift", [0, 3])
def test_adamw_8_bit_roots_by_chance(env, shift):
    """Behind the first steps of a large beta2 every root becomes the code below or above it, without a bias, the same again
    for the same inputs and another way in another step."""
    torch, B = env
    n = 200 * 256 + 77
    before = adamw_tensors(torch, [n], "f32", "f32", False, 8, seed=6, shift=shift)[0]
    held = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()         # all that e4m3 has from 0 up
    got = []
    for step in (24000, 24000, 24001):
        it = adamw_tensors(torch, [n], "f32", "f32", False, 8, seed=6, shift=shift)[0]
        adamw_call(env, [it], B.make_adamw(1e-3, 0.9, 0.999, 1e-8, step))
        got.append(it["exp_avg_sq"].clone())
        old = before["exp_avg_sq"].double() * spread(torch, before["exp_avg_sq_scale"], n)
        root = (0.999 * old ** 2 + 0.001 * before["grad"].double() ** 2).sqrt()
        c = root / spread(torch, it["exp_avg_sq_scale"], n)   # off by the scale's, the root's and the products' roundings
        code, near = it["exp_avg_sq"].double(), 16 * U * c
        above = torch.searchsorted(held, c + near).clamp(max=126)
        below = (torch.searchsorted(held, c - near, right=True) - 1).clamp(min=1)
        assert bool(((code >= held[below]) & (code <= held[above])).all())
        inside = (c > 2.0 ** -9) & (c < 447)
        gap = torch.where(c < 2.0 ** -6, 2.0 ** -9, torch.exp2(torch.floor(torch.log2(c)) - 3))
        off = ((code - c) / gap)[inside]
        # each is off by a number of mean 0 and a variance of at most 1/4: six deviations of the mean
        assert abs(float(off.mean())) <= 6 * 0.5 / math.sqrt(off.numel()) and float(off.abs().max()) < 1 + 1e-4
    assert torch.equal(got[0].view(torch.uint8), got[1].view(torch.uint8))
    assert float((got[0].view(torch.uint8) != got[2].view(torch.uint8)).double().mean()) > 0.1


@pytest.mark.parametrize("change", ["shorter", "swapped", "gradient", "decay", "state"])
def test_adamw_refuses_a_table_of_as_many_pieces(env, change):
    """Tables with the right numbers of tensors and of pieces, but of other tensors.  Every buffer has room for all of them."""
    torch, B = env
    room = adamw_tensors(torch, [4096, 4096], "f32", "f32", False, 32)
    other = torch.zeros(4096, device="cuda")

    def tensors(sizes, **more):
        return [{k: v[:n] if hasattr(v, "numel") else v for k, v in it.items()} | (more if i == 0 else {})
                for i, (it, n) in enumerate(zip(room, sizes))]
    made = tensors([2000, 4000])
    now = {"shorter": tensors([1, 4000]), "swapped": tensors([2000, 4000])[::-1], "gradient": tensors([2000, 4000], grad=other[:2000]),
           "decay": tensors([2000, 4000], weight_decay=0.5), "state": tensors([2000, 4000], exp_avg=other[:2000])}[change]
    ts, table, need, st = adamw_call(env, made, B.make_adamw(1e-3))
    again = B.AdamwTensors(now)
    assert B.dc_adamw_table_bytes(again) == need
    before = [snapshot(it) for it in room]
    B.dc_adamw(again, B.make_adamw(1e-3, step=2), None, table, need, st)
    torch.cuda.synchronize()
    assert int(st) == B.DC_ERR_BAD_LAYOUT
    for b, it in zip(before, room):
        for k in ("param", "grad", "exp_avg", "exp_avg_sq"):
            assert torch.equal(b[k], it[k])
    st.zero_()
    B.dc_adamw_table(again, table, need)                      # made again it serves
    B.dc_adamw(again, B.make_adamw(1e-3, step=2), None, table, need, st)
    torch.cuda.synchronize()
    assert int(st) == 0 and not torch.equal(before[1]["param"], room[1]["param"])


@pytest.mark.parametrize("g_type,w_type", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens,vocab,dim", [(140000, 60000, 520), (66000, 3000, 1024)])
def test_embedding_backward_adds_in_long_chunks(env, tokens, vocab, dim, g_type, w_type):
    """Chunks of 32 entries, whole lines, two slabs of columns, segments of every length, added to whole numbers: exact sums,
    rows without a token as they were."""
    torch, B = env
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim)
    g = torch.randint(-1, 2, (tokens, dim), generator=gen, device="cuda").to(types(torch)[g_type])
    ids = (torch.rand(tokens, generator=gen, device="cuda").double() ** 3 * vocab).int().clamp_(max=vocab - 1)
    ids[::97] = -1
    ids[ids % 500 == 77] = vocab - 1
    ids[ids % 7 == 3] -= 1
    dw = torch.randint(-8, 9, (vocab, dim), generator=gen, device="cuda").to(types(torch)[w_type])
    ok = ids >= 0
    named = torch.zeros(vocab, dtype=torch.bool, device="cuda").index_fill_(0, ids[ok].long(), True)
    dw[~named] = 0.3
    want = dw.float().index_add_(0, ids[ok].long(), g[ok].float()).to(dw.dtype)
    embedding_grad_call(env, g, ids, 1.0, True, dw)
    assert not bool(named.all()) and torch.equal(dw, want)
