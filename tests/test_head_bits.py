"""The head's products have the bits that their contract names: 24 of each factor of 32 bits up to 64 rows, 22 above and in the gradients,
where G has 22 for a weights' gradient in 32 bits too.  Compared in root mean square (`head_bits.py`), which a factor that has lost
its second part exceeds: shown here on the CPU with factors that are cut on purpose."""
import math

import pytest

import head_bits as hb
from head_bits import U

SMALL = [(65, 511, 2048), (200, 1000, 515), (130, 3001, 1024)]


def draw(torch, rows, vocab, dim, dtype, device, seed=0):
    g = torch.Generator().manual_seed(seed + rows * 31 + vocab * 7 + dim)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    w = rand(vocab, dim) * (2 / math.sqrt(dim))
    token = torch.randint(0, vocab, (rows,), generator=g)
    h = rand(rows, dim) + 1.5 * w[token]
    a, b = rand(rows) * 0.3, rand(rows) * 0.05
    return h.to(device, dtype), w.to(device, dtype), token.to(device).int(), a.to(device), b.to(device)


def bits_off(dtype_is_f32, bits):
    """How far a product of two factors is off of itself."""
    return 3 * 2.0 ** -bits if dtype_is_f32 else 0.0


# ---- on the CPU: what the bounds hold and what they do not ----

def cut(torch, x, top, planes, wrong=1.0):
    """x as that many f16, 2^(15 - exponent of top) times as much, the second times 2048 (or `wrong` times what it is)."""
    up = 2.0 ** (15 - torch.frexp(top).exponent).double()
    first = (x * up).half().double()
    rest = ((x * up - first) * 2048).half().double() / 2048 * wrong if planes == 2 else 0.0
    return first / up, rest / up if planes == 2 else torch.zeros_like(first)


def parts_product(x, y):
    """All products of parts but the two small ones'."""
    t = lambda m: m.t().contiguous()  # noqa: E731
    return x[0] @ t(y[0]) + x[1] @ t(y[0]) + x[0] @ t(y[1])


def cut_products(torch, h, w, temperature, token, a, b, planes, wrong=1.0):
    """The forward results and the gradients with factors of so many f16: of hidden, the weights and G."""
    hd, wd = h.double(), w.double()
    row_top = lambda m: m.abs().amax(1, keepdim=True)  # noqa: E731
    hp, wp = cut(torch, hd, row_top(hd), planes[0], wrong), cut(torch, wd, wd.abs().max(), planes[1], wrong)
    x = parts_product(hp, wp)
    exact = hd @ wd.t()
    top = exact.max(1).values
    stat = torch.stack([top, ((exact - top[:, None]) / temperature).exp().sum(1).log()], 1)
    p = torch.log_softmax(exact / temperature, 1)
    entropy = -(p.exp() * p).sum(1)
    zero = (x, torch.zeros_like(x))
    out, _ = hb.forward(torch, h, w, temperature, token, zero)
    g, _, largest = hb.logits_gradient(torch, zero, temperature, token, stat, entropy, a, b)
    gp = cut(torch, g, largest, planes[2], wrong)
    # (hidden rows for the weights' gradient: one power of two, as G's rows have their own already)
    weigh = 2.0 ** torch.frexp(largest).exponent.double()
    scaled = hd * weigh
    xp = cut(torch, scaled, scaled.abs().max(), planes[0], wrong)
    gs = [m / weigh for m in gp]
    t = lambda ms: [m.t() for m in ms]  # noqa: E731
    return {**out, "hidden": parts_product(gp, t(wp)), "weight": parts_product(t(gs), t(xp))}, stat, entropy


def bounds_of(torch, h, w, temperature, token, stat, entropy, a, b, x_bits, g_bits):
    """Exact results and bounds.  x_bits: of the logits' factors (None: exact ones), g_bits: of G in the hidden and in the weights' gradient."""
    f32 = h.dtype == torch.float32
    hd, wd = h.double(), w.double()
    x_bound = hb.product_bound(torch, hd, wd, 3 * 2.0 ** -x_bits if x_bits else 0.0, {24: 6, 22: 3, None: 1}[x_bits])
    want, bound = hb.forward(torch, h, w, temperature, token, x_bound)
    g, dg, _ = hb.logits_gradient(torch, x_bound, temperature, token, stat, entropy, a, b)
    for name, left, off, right, bits in (("hidden", g, dg, wd.t(), g_bits[0]), ("weight", g.t(), dg.t(), hd.t(), g_bits[1])):
        want[name], bound[name] = hb.product_bound(torch, left, right.contiguous(), off + (3 if f32 else 1) * 2.0 ** -bits, 3 if f32 else 2)
    return want, bound


@pytest.mark.parametrize("rows,vocab,dim", SMALL)
def test_bounds_hold_two_parts_and_no_fewer(rows, vocab, dim):
    import torch
    h, w, token, a, b = draw(torch, rows, vocab, dim, torch.float32, "cpu")

    def off(planes, wrong=1.0):
        got, stat, entropy = cut_products(torch, h, w, 0.8, token, a, b, planes, wrong)
        want, bound = bounds_of(torch, h, w, 0.8, token, stat, entropy, a, b, 22, (22, 22))
        return {k: hb.off_by(got[k], want[k], bound[k]) for k in want}

    assert max(off((2, 2, 2)).values()) < 0.5, off((2, 2, 2))
    for planes, names in (((1, 2, 2), ("top", "logprob", "weight")), ((2, 1, 2), ("top", "logprob", "hidden")), ((2, 2, 1), ("hidden", "weight"))):
        found = off(planes)
        assert all(found[k] > 2 for k in names), (planes, found)
    found = off((2, 2, 2), wrong=0.5)                         # a second part that counts for half as much
    assert all(found[k] > 2 for k in ("top", "logprob", "hidden", "weight")), found


FEW = [(64, 3001, 128), (33, 5000, 96), (20, 20011, 256), (64, 999, 33)]


@pytest.mark.parametrize("rows,vocab,dim", FEW)
def test_bounds_of_few_rows_hold_three_parts_and_no_fewer(rows, vocab, dim):
    """Three of bf16, cut off and not rounded, and the six largest products of theirs."""
    import torch
    h, w, token, _, _ = draw(torch, rows, vocab, dim, torch.float32, "cpu")

    def parts(x, n):
        out, rest = [], x.clone()
        for _ in range(n):
            out.append((rest.view(torch.int32) & -65536).view(torch.float32))
            rest = rest - out[-1]
        return [p.double() for p in out]

    for n in (3, 2):
        hp, wp = parts(h, n), parts(w, n)
        x = sum(hp[i] @ wp[j].t() for i in range(n) for j in range(n) if i + j < 3)
        x_bound = hb.product_bound(torch, h.double(), w.double(), 3 * 2.0 ** -24, 6)
        want, bound = hb.forward(torch, h, w, 0.8, token, x_bound)
        got, _ = hb.forward(torch, h, w, 0.8, token, (x, x_bound[1]))
        tt = x.topk(64).indices
        off = {**{k: hb.off_by(got[k], want[k], bound[k]) for k in want},
               "alternatives": hb.off_by(*hb.alternatives(torch, x_bound, 0.8, tt, (x / 0.8).gather(1, tt)))}
        assert max(off.values()) < 0.5 if n == 3 else min(off["top"], off["alternatives"]) > 2, (n, off)


# ---- on the GPU ----

@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2507_13833_amd import binding
    binding.load()
    assert torch.cuda.is_available()
    return torch, binding


def call(env, h, w, temperature, token, n_top=0):
    torch, B = env
    n, m = h.shape[0], B.make_matrix
    lp, st, en = (torch.empty(s, device="cuda") for s in ((n,), (n, 2), (n,)))
    tt, tl = (torch.empty(n, n_top, dtype=d, device="cuda") if n_top else None for d in (torch.int32, torch.float32))
    need = B.dc_head_logprob_workspace_bytes(m(h), m(w), n_top)
    ws, status = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_head_logprob(m(h), m(w), temperature, token, None, n_top, lp, st, en, tt, tl, ws, need, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    return {"logprob": lp, "stat": st, "entropy": en, "top_token": tt, "top_logprob": tl}


def call_grad(env, h, w, temperature, token, stat, entropy, a, b, dtype):
    torch, B = env
    m = B.make_matrix
    gh, gw = torch.empty_like(h), torch.empty(w.shape, dtype=dtype, device="cuda")
    need = B.dc_head_logprob_backward_workspace_bytes(m(h), m(w), m(gw))
    ws, status = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_head_logprob_backward(m(h), m(w), temperature, token, None, stat, entropy, a, b, m(gh), False, m(gw), ws, need, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    return {"hidden": gh, "weight": gw}


def close(torch, got, want, bound, names):
    found = {k: hb.off_by(got[k], want[k], bound[k]) for k in names}
    assert all(math.isfinite(v) and v <= 1 for v in found.values()), found
    return found


# several pieces of the weights (130 x 20011 x 8192: three of the forward product, two of the gradients'), several shares of the sums
# over the vocabulary, odd sizes
@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,dim", SMALL + [(300, 8191, 515), (700, 700, 96), (130, 20011, 8192), (1100, 4000, 2048)])
def test_factors_of_32_bits(env, rows, vocab, dim):
    torch, B = env
    h, w, token, a, b = draw(torch, rows, vocab, dim, torch.float32, "cuda")
    f = call(env, h, w, 0.8, token)
    got = {"top": f["stat"][:, 0], "logprob": f["logprob"], "entropy": f["entropy"],
           **call_grad(env, h, w, 0.8, token, f["stat"], f["entropy"], a, b, torch.float32)}
    want, bound = bounds_of(torch, h, w, 0.8, token, f["stat"], f["entropy"], a, b, 22, (22, 22))
    print(close(torch, got, want, bound, want))
    f = call(env, h, w, 0.8, token, 64)
    x_bound = hb.product_bound(torch, h.double(), w.double(), 3 * 2.0 ** -22, 3)
    assert hb.off_by(*hb.alternatives(torch, x_bound, 0.8, f["top_token"], f["top_logprob"])) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,dim", FEW)
def test_factors_of_32_bits_few_rows(env, rows, vocab, dim):
    """A part that is lost here is 2^-16 of a factor: seen where rows are short."""
    torch, B = env
    h, w, token, a, b = draw(torch, rows, vocab, dim, torch.float32, "cuda")
    f = call(env, h, w, 0.8, token, 64)
    x_bound = hb.product_bound(torch, h.double(), w.double(), 3 * 2.0 ** -24, 6)
    assert hb.off_by(*hb.alternatives(torch, x_bound, 0.8, f["top_token"], f["top_logprob"])) <= 1
    want, bound = hb.forward(torch, h, w, 0.8, token, x_bound)
    got = {"top": f["stat"][:, 0], "logprob": f["logprob"], "entropy": f["entropy"]}
    print(close(torch, got, want, bound, want))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,dim", SMALL + [(700, 700, 96), (1100, 20011, 256)])
def test_weights_gradient_in_32_bits(env, rows, vocab, dim, dtype):
    """G in two parts, hidden states as they are."""
    torch, B = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    h, w, token, a, b = draw(torch, rows, vocab, dim, dt, "cuda")
    f = call(env, h, w, 0.8, token)
    got = call_grad(env, h, w, 0.8, token, f["stat"], f["entropy"], a, b, torch.float32)
    want, bound = bounds_of(torch, h, w, 0.8, token, f["stat"], f["entropy"], a, b, None, (11, 22))
    print(close(torch, got, want, bound, ("weight",)))
