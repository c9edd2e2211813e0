"""Log-probabilities from hidden states and the head's weights, and the gradients of both, on an MI355X against plain torch in 64 bits.

Tolerances count roundings: U = 2^-24 for one in 32 bits, half of finfo.eps for one to a tensor's type.  A logit is a sum of `dim`
products (16-bit factors: exact ones; 32-bit factors: six times as many, off by 4 U of each product): it is off by at most
2 U (additions) sum |h w|, where an addition on the matrix cores is given two roundings' worth.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


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


def rows_of(torch, t, pad, shift, poison=math.nan):
    """The same matrix with rows `pad` elements further apart, `shift` elements into its memory, poison between the rows."""
    rows, cols = t.shape
    store = torch.full((rows * (cols + pad) + shift + 8,), poison, dtype=t.dtype, device=t.device)
    view = store.as_strided((rows, cols), (cols + pad, 1), shift)
    view.copy_(t)
    return view


def draw(torch, rows, vocab, dim, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 31 + vocab * 7 + dim)
    w = torch.randn(vocab, dim, generator=g, device="cuda") * (2 / math.sqrt(dim))
    token = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    h = torch.randn(rows, dim, generator=g, device="cuda") + 1.5 * w[token]
    mask = (torch.rand(rows, generator=g, device="cuda") < 0.7).to(torch.uint8)
    dt = types(torch)[dtype]
    return h.to(dt), w.to(dt), token.to(torch.int32), mask


def call(env, h, w, temperature, token, mask, n_top, stat=True, entropy=True, stream=None, ws=None):
    torch, B = env
    n = h.shape[0]
    new = lambda *s, dtype=torch.float32: torch.full(s, -7, dtype=dtype, device="cuda")  # noqa: E731
    out = {"logprob": new(n) if token is not None else None, "stat": new(n, 2) if stat else None, "entropy": new(n) if entropy else None,
           "top_token": new(n, n_top, dtype=torch.int32) if n_top else None, "top_logprob": new(n, n_top) if n_top else None}
    mh, mw = B.make_matrix(h), B.make_matrix(w)
    need = B.dc_head_logprob_workspace_bytes(mh, mw, n_top)
    if ws is None:
        ws = torch.full((max(need, 1),), 0xA5, dtype=torch.uint8, device="cuda")
    out["status"], out["keep"] = torch.zeros(1, dtype=torch.int32, device="cuda"), ws
    B.dc_head_logprob(mh, mw, temperature, token, mask, n_top, out["logprob"], out["stat"], out["entropy"], out["top_token"],
                      out["top_logprob"], ws, ws.numel(), out["status"], stream=stream)
    return out


def logits_of(torch, h, w):
    """Logits in 64 bits and how far 32-bit sums may be off them."""
    hd, wd = h.double(), w.double()
    x = hd @ wd.t().contiguous()
    size = hd.abs() @ wd.abs().t().contiguous()
    adds = h.shape[1] * (6 if h.dtype == torch.float32 else 1) + 8
    return x, (2 * adds + 4) * U * size


def reference(torch, h, w, temperature, token, mask, n_top):
    """Values and how far they may be off: a logit's error dx moves the sum's logarithm by at most its largest, and the roundings
    behind the logits are those of a sum over the vocabulary: z = (x - M) / T carries 3 roundings, 2^z 3 more, and a partial sum
    runs over at most 32 terms of a tile, as many tiles as there are and 16 joins."""
    x, dx = logits_of(torch, h, w)
    n, vocab = x.shape
    live = torch.ones(n, dtype=torch.bool, device="cuda") if mask is None else mask != 0
    top = x.max(1).values
    far = dx.max(1).values / temperature
    z = (x - top[:, None]) / temperature
    e = z.exp()
    s = e.sum(1)
    p, log_sum = e / s[:, None], s.log()
    ez, ez2 = (p * z.abs()).sum(1), (p * z * z).sum(1)
    adds = vocab / 8 + 64 if vocab < 4096 else vocab / 256 + 512
    tol_sum = 2 * far + U * (6 * ez + 6 + adds + 2 * log_sum.abs())
    want = {"stat": torch.stack([top, log_sum], 1), "entropy": log_sum + ez}
    tol = {"stat": torch.stack([far * temperature + U * top.abs(), tol_sum], 1),
           "entropy": tol_sum + 2 * far * (ez + 1) + U * ((2 * adds + 10) * ez + 8 * ez2 + 2 * (log_sum + ez) + 1)}
    if token is not None:
        t = token.long().clamp(0, vocab - 1)
        zt = z.gather(1, t[:, None])[:, 0]
        want["logprob"], tol["logprob"] = zt - log_sum, 2 * far + tol_sum + U * (3 * zt.abs() + (zt - log_sum).abs())
    if n_top:
        value, column = x.sort(dim=1, descending=True, stable=True)
        zt = (value[:, :n_top] - top[:, None]) / temperature
        want["top_token"] = column[:, :n_top].int()
        want["top_logprob"] = zt - log_sum[:, None]
        tol["top_logprob"] = (2 * far + tol_sum)[:, None] + U * (3 * zt.abs() + want["top_logprob"].abs())
    for k, v in want.items():
        v[~live] = -1 if k == "top_token" else 0.0
        if k != "top_token":
            tol[k][~live] = 0.0
    return want, tol, x, dx


def check(env, h, w, temperature=1.0, token=None, mask=None, n_top=0, status=0, **kw):
    torch, B = env
    got = call(env, h, w, temperature, token, mask, n_top, **kw)
    want, tol, x, dx = reference(torch, h, w, temperature, token, mask, n_top)
    torch.cuda.synchronize()
    assert int(got["status"]) == status
    for k, v in want.items():
        g = got[k]
        if g is None:
            continue
        if k == "top_token":
            # tokens whose logits lie nearer to each other than they may be off may change places
            live = torch.ones(x.shape[0], dtype=torch.bool, device="cuda") if mask is None else mask != 0
            assert torch.equal(g[~live], v[~live])
            a, b = (x[live].gather(1, t[live].long()) for t in (g, v))
            assert not ((a - b).abs() > 2 * dx[live].max(1, keepdim=True).values).any()
            assert (g[live].sort(1).values.diff(dim=1) > 0).all()
            continue
        off = (g.double() - v).abs() - tol[k]
        assert not off.numel() or float(off.max()) <= 0, (k, float(off.max()))
    return got


SHAPES = [(1, 1, 1), (1, 7, 3), (2, 2, 64), (3, 255, 31), (5, 257, 64), (16, 300, 96), (17, 1000, 515), (33, 700, 128), (64, 5000, 32), (65, 511, 2048),
          (127, 256, 64), (128, 512, 64), (129, 513, 65), (300, 2050, 128), (700, 700, 40), (1, 152064, 64), (70, 20011, 96), (1100, 1300, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,dim", SHAPES)
def test_head(env, rows, vocab, dim, dtype):
    torch, B = env
    h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
    check(env, h, w, 1.0, token, None, 0)
    check(env, h, w, 0.7, token, mask, 0)
    check(env, h, w, 0.7, token, mask, min(5, vocab))
    check(env, h, w, 1.0, token, None, min(64, vocab), stat=False, entropy=False)
    check(env, h, w, 1.3, token, mask, 0, stat=False, entropy=False)
    check(env, h, w, 1.3, None, mask, 0, entropy=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 48, 64])
@pytest.mark.parametrize("vocab,dim", [(5, 256), (4099, 768), (33003, 128), (20011, 2048), (1037, 320)])
def test_head_few_rows(env, rows, vocab, dim, dtype):
    h, w, token, mask = draw(env[0], rows, vocab, dim, dtype)
    check(env, h, w, 0.9, token, mask, 0)
    check(env, h, w, 1.0, token, None, 3)


# ---- rows that lie more than 4 GB apart ----

@pytest.mark.parametrize("rows,pad,vocab,wpad", [(9, 0, 2500, (1 << 20) - 64), (300, 0, 2500, (1 << 20) - 64), (1500, (1 << 21) - 64, 520, 0),
                                                 (300, (1 << 23) - 64, 600, (1 << 22) + 64)])
def test_head_far_apart_rows(env, rows, pad, vocab, wpad):
    h, w, token, mask = draw(env[0], rows, vocab, 64, "bf16")
    h, w = rows_of(env[0], h, pad, 0), rows_of(env[0], w, wpad, 0)
    for m in (None, mask):
        check(env, h, w, 0.9, token, m, 0)
        check_grad(env, h, w, 0.9, token, m, pads=(wpad, 0) if rows == 9 else None)
    check(env, h, w, 0.9, token, mask, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift,wpad,wshift", [(1, 0, 0, 0), (0, 1, 8, 8), (8, 8, 3, 5), (8, 0, 16, 0), (0, 0, 1, 1), (32, 16, 32, 8)])
def test_head_strides(env, pad, shift, wpad, wshift, dtype):
    torch, B = env
    for rows, vocab, dim in ((9, 1001, 64), (300, 520, 96), (40, 300, 33)):
        h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
        check(env, rows_of(torch, h, pad, shift), rows_of(torch, w, wpad, wshift), 1.3, token, mask, 0)
        check(env, rows_of(torch, h, pad, shift), rows_of(torch, w, wpad, wshift), 1.3, token, mask, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_head_masked_rows_are_not_looked_at(env, rows, dtype):
    """Masked rows hold NaN and infinities and tokens outside; all rows masked; one row left."""
    torch, B = env
    h, w, token, mask = draw(torch, rows, 600, 64, dtype)
    for kind in ("some", "all", "one"):
        k = mask.clone()
        if kind != "some":
            k.zero_()
        if kind == "one":
            k[rows // 2] = 3
        hp, tp = h.clone(), token.clone()
        hp[k == 0] = math.nan
        hp[k == 0, 1] = math.inf
        tp[k == 0] = 1 << 30
        for n_top in (0, 3):
            got = call(env, hp, w, 1.0, tp, k, n_top)
            want = call(env, h, w, 1.0, token, k, n_top)
            torch.cuda.synchronize()
            assert int(got["status"]) == 0
            for name in ("logprob", "stat", "entropy", "top_token", "top_logprob"):
                if got[name] is not None:
                    assert torch.equal(got[name], want[name]), (kind, n_top, name)
        check(env, h, w, 1.0, token, k, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_head_rows_without_a_distribution(env, dtype):
    """A NaN in a row of hidden makes NaN and -1 of that row alone."""
    torch, B = env
    for rows in (5, 200):
        h, w, token, mask = draw(torch, rows, 900, 64, dtype)
        clean = {n: call(env, h, w, 1.0, token, None, n) for n in (0, 4)}
        h[2, 9] = math.nan
        h[4, 3] = math.inf
        for n in (0, 4):
            got = call(env, h, w, 1.0, token, None, n)
            rest = torch.ones(rows, dtype=torch.bool, device="cuda")
            rest[2] = rest[4] = False
            for name in ("logprob", "stat", "entropy", "top_token", "top_logprob"):
                if got[name] is None:
                    continue
                assert torch.equal(got[name][rest], clean[n][name][rest])
                bad = got[name][~rest]
                assert (bad == -1).all() if name == "top_token" else bad.isnan().all(), name


def test_head_token_outside(env):
    torch, B = env
    h, w, token, mask = draw(torch, 40, 300, 64, "bf16")
    for bad in (-1, 300, 1 << 30, -(1 << 31)):
        for n_top in (0, 2):
            t = token.clone()
            t[7] = bad
            got = call(env, h, w, 1.0, t, None, n_top)
            want = call(env, h, w, 1.0, token, None, n_top)
            torch.cuda.synchronize()
            assert int(got["status"]) == B.DC_ERR_TOKEN_RANGE
            rest = torch.arange(40, device="cuda") != 7
            assert got["logprob"][7].isnan() and torch.equal(got["logprob"][rest], want["logprob"][rest])
            assert torch.equal(got["stat"], want["stat"]) and torch.equal(got["entropy"], want["entropy"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_equal_logits(env, dtype):
    """Weights that are all the same: a uniform distribution, alternatives in order of their tokens."""
    torch, B = env
    h, w, token, mask = draw(torch, 20, 700, 64, dtype)
    w[:] = w[:1]
    got = call(env, h, w, 1.0, token, None, 6)
    assert torch.equal(got["top_token"], torch.arange(6, device="cuda", dtype=torch.int32).expand(20, 6))
    check(env, h, w, 1.0, token, None, 0)
    h[:] = 0
    check(env, h, w, 1.0, token, None, 0)


@pytest.mark.parametrize("at", [1e4, -1e4, 3e7, -3e9])
def test_head_far_logits(env, at):
    """Logits far from zero but near to each other: one column of hidden and weight carries the distance exactly."""
    torch, B = env
    for dtype, rows in (("f32", 9), ("f32", 200), ("bf16", 200)):
        h, w, token, mask = draw(torch, rows, 1000, 64, dtype)
        h[:, 0] = 2.0 ** round(math.log2(abs(at)))
        w[:, 0] = math.copysign(1.0, at)
        check(env, h, w, 1.0, token, None, 0)


def test_head_pieces_of_the_weights(env):
    """Weights that are laid out in pieces: long rows in 32 bits, and 16-bit ones that no step takes whole."""
    torch, B = env
    for rows, vocab, dim, dtype in ((3, 50000, 2048, "f32"), (140, 50000, 2048, "f32"), (5, 140001, 1027, "bf16")):
        h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
        check(env, h, w, 1.0, token, mask, 0)
        check(env, h, w, 1.0, token, None, 3)


def test_head_agrees_with_the_logits_path(env):
    """As dc_token_logprob has it on the same logits, made by a product in 32 bits."""
    torch, B = env
    h, w, token, mask = draw(torch, 50, 3001, 128, "f32")
    got = call(env, h, w, 0.9, token, mask, 8)
    x = (h.double() @ w.double().t().contiguous()).float()
    n = 50
    lp, st, en = (torch.empty(s, device="cuda") for s in ((n,), (n, 2), (n,)))
    tt, tl = torch.empty(n, 8, dtype=torch.int32, device="cuda"), torch.empty(n, 8, device="cuda")
    mx = B.make_matrix(x)
    need = B.dc_token_logprob_workspace_bytes(mx, 8)
    ws, status = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_token_logprob(mx, 0.9, token, mask, 8, lp, st, en, tt, tl, ws, need, status)
    for a, b in ((got["logprob"], lp), (got["stat"], st), (got["entropy"], en), (got["top_logprob"], tl)):
        assert float((a - b).abs().max()) < 1e-3
    assert torch.equal(got["top_token"], tt)


def test_head_no_rows_and_smaller_calls(env):
    """No rows; a workspace for the largest call serves fewer rows and fewer alternatives."""
    torch, B = env
    h, w, token, mask = draw(torch, 0, 300, 64, "bf16")
    call(env, h, w, 1.0, token, None, 0)
    for dtype in ("bf16", "f32"):
        h, w, token, mask = draw(torch, 700, 3000, 72, dtype)
        mw = B.make_matrix(w)
        last = 0
        for n in (1, 2, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257, 384, 500, 640, 641, 700):
            need = B.dc_head_logprob_workspace_bytes(B.make_matrix(h[:n]), mw, 9)
            assert need >= last and need >= B.dc_head_logprob_workspace_bytes(B.make_matrix(h[:n]), mw, 0)
            last = need
        ws = torch.full((last,), 0xA5, dtype=torch.uint8, device="cuda")
        for n in (1, 17, 64, 129, 640):
            check(env, h[:n], w, 1.0, token[:n], mask[:n], 0, ws=ws)
            check(env, h[:n], w, 1.0, token[:n], mask[:n], 4, ws=ws)


# ---- the gradients ----

def call_grad(env, h, w, temperature, token, mask, stat, entropy, a, b, grad_w="same", hidden=True, before=None, stream=None, ws=None, pads=None):
    torch, B = env
    dt = h.dtype if grad_w == "same" else torch.float32
    gh = torch.full_like(h.contiguous(), -7.0) if hidden else None
    gw = None if grad_w is None else torch.full(w.shape, -7.0, dtype=dt, device="cuda") if before is None else before.clone()
    if pads:
        gh = rows_of(torch, gh, *pads) if gh is not None else None
        gw = rows_of(torch, gw, *pads) if gw is not None else None
    m = lambda x: None if x is None else B.make_matrix(x)  # noqa: E731
    need = B.dc_head_logprob_backward_workspace_bytes(m(h), m(w), m(gw))
    if ws is None:
        ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dc_head_logprob_backward(m(h), m(w), temperature, token, mask, stat, entropy, a, b, m(gh), before is not None, m(gw), ws, ws.numel(),
                               status, stream=stream)
    return {"hidden": gh, "weight": gw, "status": status, "keep": ws}


def grad_reference(torch, h, w, temperature, token, mask, stat, entropy, a, b, before=None, f32_weight=False):
    """Values and tolerances.  p is off by the logit's error and the roundings of log2 p = (x - M) k - log2 S (|z| and log S are
    rounded, 2^ is good to 2), G by those of its two factors; G is rounded to 2^-11 of itself (16-bit types: f16's half step,
    eps / 2 = 2^-11; two of them, where the weights' gradient is in 32 bits, 2^-22; 32-bit types: two for each factor, and the product of
    the small parts is left off, 3 times 2^-22 < 2^-20, which the 2 (6 n + 8) U of their sums hold with room for 2^-23 more) or 2^-38 of
    its bound; sums of n terms are off by 2 n U.  The last rounding is of
    what was computed, not of the exact value v: off by e before it, |round(v + e) - v| <= e + half_step (|v| + e)."""
    x, dx = logits_of(torch, h, w)
    n, vocab = x.shape
    hd, wd = h.double(), w.double()
    st = stat.double()
    logp = (x - st[:, :1]) / temperature - st[:, 1:]
    p = logp.exp()
    ad = a.double()[:, None] / temperature
    bd = (b.double()[:, None] if b is not None else torch.zeros_like(ad)) / temperature if b is not None else torch.zeros_like(ad)
    H = entropy.double()[:, None] if entropy is not None else torch.zeros_like(ad)
    dead = torch.zeros(n, dtype=torch.bool, device="cuda") if mask is None else mask == 0
    weigh = ad + bd * (logp + H)
    g = -p * weigh
    own = torch.zeros_like(g)
    if token is not None:
        ok = (token >= 0) & (token < vocab)
        own[torch.arange(n, device="cuda")[ok], token[ok].long()] = 1.0
    g = g + own * ad
    size = p * (ad.abs() + bd.abs() * (logp.abs() + H.abs())) + own * ad.abs()
    dlog = dx / temperature + U * (6 * ((x - st[:, :1]) / temperature).abs() + 4 * st[:, 1:].abs() + 4)
    dg = size * (dlog + 10 * U) + p * bd.abs() * dlog
    g[dead], dg[dead], size[dead] = 0.0, 0.0, 0.0
    bound = (ad.abs() + bd.abs() * (H.abs() + 1))
    bound[dead] = 0.0
    f32 = h.dtype == torch.float32
    one = (2.0 ** -23 if f32 else 2.0 ** -11) * g.abs() + (0 if f32 else 2.0 ** -37) * bound
    two = (2.0 ** -23 if f32 else 2.0 ** -22) * g.abs() + (0 if f32 else 2.0 ** -37) * bound
    factor = 6 if f32 else 1
    gh = g @ wd
    th = (dg + one) @ wd.abs() + (2 * (factor * vocab + 64) + 8) * U * (g.abs() @ wd.abs()) 
    if not f32:
        th = th + 2.0 ** -37 * g.abs().sum(1, keepdim=True) * wd.abs().max()
    th = th + half_step(torch, h.dtype) * (gh.abs() + th) + torch.finfo(h.dtype).tiny
    gt = g.t().contiguous()
    hz = torch.where(dead[:, None], 0.0, hd)
    gw = gt @ hz
    dt = torch.float32 if f32_weight else h.dtype
    tw = (dg + (two if f32_weight else one)).t().contiguous() @ hz.abs() + (2 * (2 * factor * n + 8) + 8) * U * (gt.abs() @ hz.abs())
    if not f32:
        tw = tw + 2.0 ** -36 * n * (bound[:, 0] * hz.abs().max(1).values).max()
    if before is not None:
        gw = gw + before.double()
        tw = tw + U * gw.abs()
    tw = tw + half_step(torch, dt) * (gw.abs() + tw) + torch.finfo(dt).tiny
    return {"hidden": gh, "weight": gw}, {"hidden": th, "weight": tw}


def gradients(torch, rows, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows)
    return torch.randn(rows, generator=g, device="cuda") * 0.3, torch.randn(rows, generator=g, device="cuda") * 0.05


def check_grad(env, h, w, temperature, token, mask, entropy=True, grad_w="same", before=None, status=0, a=None, b=None, **kw):
    torch, B = env
    fwd = call(env, torch.where(mask[:, None] == 0, torch.zeros_like(h), h) if mask is not None else h, w, temperature,
               None if token is None else token.clamp(0, w.shape[0] - 1), mask, 0)
    if a is None:
        a, b = gradients(torch, h.shape[0])
    if not entropy:
        b = None
    got = call_grad(env, h, w, temperature, token, mask, fwd["stat"], fwd["entropy"], a, b, grad_w=grad_w, before=before, **kw)
    want, tol = grad_reference(torch, torch.nan_to_num(h, 0, 0, 0), w, temperature, token, mask, fwd["stat"], fwd["entropy"], a, b, before, grad_w == "f32" or h.dtype == torch.float32)
    torch.cuda.synchronize()
    assert int(got["status"]) == status
    for k, v in want.items():
        if got[k] is None:
            continue
        off = (got[k].double() - v).abs() - tol[k]
        assert not off.numel() or float(off.max()) <= 0, (k, float(off.max()), float(((got[k].double() - v).abs() / tol[k]).max()))
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,dim", SHAPES)
def test_head_backward(env, rows, vocab, dim, dtype):
    torch, B = env
    h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
    check_grad(env, h, w, 1.0, token, None)
    check_grad(env, h, w, 0.7, token, mask, grad_w="f32")
    before = torch.randn(vocab, dim, device="cuda")
    check_grad(env, h, w, 1.3, token, mask, entropy=False, grad_w="f32", before=before)
    check_grad(env, h, w, 1.0, None, None, before=before.to(h.dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift,wpad,wshift", [(1, 0, 0, 0), (0, 1, 8, 8), (8, 8, 3, 5), (8, 0, 16, 0), (32, 16, 32, 8)])
def test_head_backward_strides(env, pad, shift, wpad, wshift, dtype):
    torch, B = env
    for rows, vocab, dim in ((9, 1001, 64), (300, 520, 96), (40, 300, 33)):
        h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
        got = check_grad(env, rows_of(torch, h, pad, shift), rows_of(torch, w, wpad, wshift), 1.3, token, mask, pads=(pad, shift))
        for k in ("hidden", "weight"):                        # nothing between the rows is written
            t = got[k]
            if pad:
                gap = t.as_strided((t.shape[0] - 1, pad), (t.stride(0), 1), t.storage_offset() + t.shape[1])
                assert gap.isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_head_backward_rows_that_add_nothing(env, rows, dtype):
    """Masked rows and rows whose a and b are zero, full of NaN, with tokens outside."""
    torch, B = env
    h, w, token, mask = draw(torch, rows, 600, 64, dtype)
    a, b = gradients(torch, rows)
    for kind in ("some", "all", "one", "zero"):
        k, a2, b2 = mask.clone(), a.clone(), b.clone()
        if kind in ("all", "one"):
            k.zero_()
        if kind == "one":
            k[rows // 2] = 3
        if kind == "zero":
            k.fill_(1)
            a2[::2] = 0
            b2[::2] = -0.0
        idle = (k == 0) | ((a2 == 0) & (b2 == 0))
        hp, tp = h.clone(), token.clone()
        hp[idle] = math.nan
        tp[idle] = -5
        keep = (~idle).to(torch.uint8)
        got = check_grad(env, hp, w, 1.0, tp, keep, a=a2, b=b2)
        assert not got["hidden"][idle].any() and not got["hidden"].isnan().any()
        fwd = call(env, torch.nan_to_num(hp, 0, 0, 0), w, 1.0, tp.clamp(0, 599), None, 0)
        again = call_grad(env, hp, w, 1.0, tp, k if kind != "zero" else None, fwd["stat"], fwd["entropy"], a2, b2)
        torch.cuda.synchronize()
        assert int(again["status"]) == 0
        assert torch.equal(again["hidden"], got["hidden"]) and torch.equal(again["weight"], got["weight"])


def test_head_backward_token_outside_and_rows_without_a_distribution(env):
    torch, B = env
    h, w, token, mask = draw(torch, 40, 300, 64, "bf16")
    t = token.clone()
    t[7] = 300
    check_grad(env, h, w, 1.0, t, None, status=B.DC_ERR_TOKEN_RANGE)
    a, b = gradients(torch, 40)
    fwd = call(env, h, w, 1.0, token, None, 0)
    clean = call_grad(env, h, w, 1.0, token, None, fwd["stat"], fwd["entropy"], a, b)
    fwd["stat"][5] = math.nan
    got = call_grad(env, h, w, 1.0, token, None, fwd["stat"], fwd["entropy"], a, b)
    rest = torch.arange(40, device="cuda") != 5
    assert got["hidden"][5].isnan().all() and torch.equal(got["hidden"][rest], clean["hidden"][rest]) and got["weight"].isnan().all()


@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("scale", [2.0 ** -19, 2.0 ** 13])
def test_head_f16_at_the_ends_of_its_range(env, rows, scale):
    """Weights among the type's subnormal numbers, and next to its largest."""
    h, w, token, mask = draw(env[0], rows, 700, 96, "f16")
    w = (w * scale).clamp(-6e4, 6e4)
    h = h if scale < 1 else h / scale
    check(env, h, w, 1.0, token, mask, 0)
    check_grad(env, h, w, 1.0, token, mask)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_head_backward_rows_of_very_different_size(env, dtype):
    """Gradients from 2^-90 to 2^6 in one batch, and hidden rows of different sizes: each row's own gradient is as exact as if it were
    alone."""
    torch, B = env
    h, w, token, mask = draw(torch, 60, 500, 64, dtype)
    a, b = gradients(torch, 60)
    scale = 2.0 ** torch.linspace(-90 if dtype == "bf16" else -12, 6, 60, device="cuda").round()
    h = (h.float() * 2.0 ** torch.linspace(2, -4, 60, device="cuda").round()[:, None]).to(h.dtype)
    check_grad(env, h, w, 1.0, token, None, a=a * scale, b=b * scale)
    check_grad(env, h, w, 1.0, token, None, a=a * scale, b=b * scale, grad_w="f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,temperature,scale", [(-60, 1.0, 20), (-105, 0.7, 20), (-115, 1.0, 30), (-118, 1.0, 40), (-118, 2.0 ** 24, 60), (-145, 1.0, 60),
                                                    (118, 2.0 ** -20, -40)])
def test_head_backward_gradients_at_the_ends_of_the_range(env, dtype, size, temperature, scale):
    """Gradients of the logits that are subnormal in 32 bits, or beyond their range, with weights (then hidden rows) that take a result
    back into it: as exact as any other."""
    torch, B = env
    h, w, token, mask = draw(torch, 60, 500, 64, dtype)
    a, b = gradients(torch, 60)
    # (a subnormal a has few bits of its own, and is given as it is)
    a, b = (torch.ldexp(x.double(), torch.tensor(float(size), device="cuda").double()).float() for x in (a, b))
    # (the other gradient goes further out of the range by as much: below 2^-149, or to 2^158 and more)
    for k in (scale, -scale):
        hk, wk = (torch.ldexp(x.float(), torch.tensor(float(e), device="cuda")).to(x.dtype) for x, e in ((h, -k), (w, k)))
        hk = torch.ldexp(hk.float(), torch.tensor(math.log2(temperature), device="cuda").round()).to(h.dtype)
        check_grad(env, hk, wk, temperature, token, mask, a=a, b=b, **(dict(grad_w=None) if k == scale else dict(hidden=False)))
        if k != scale:
            check_grad(env, hk, wk, temperature, token, None, a=a, b=b, hidden=False, grad_w="f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [100, 114, 120, 124, -100, -114, -120])
def test_head_backward_weights_at_the_ends_of_the_range(env, dtype, scale):
    """Weights next to the largest and the smallest numbers, hidden states that take the logits back: gradients that 32 bits hold are
    finite and as exact as any other."""
    torch, B = env
    for rows, vocab, dim in ((9, 700, 64), (300, 1000, 96)):
        h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
        h, w = (torch.ldexp(x.float(), torch.tensor(float(e), device="cuda")).to(x.dtype) for x, e in ((h, -scale), (w, scale)))
        check_grad(env, h, w, 1.0, token, mask)
        check_grad(env, h, w, 0.7, token, None, grad_w="f32")


def test_head_backward_parts_alone(env):
    """Either gradient without the other is the same bits."""
    torch, B = env
    for dtype in ("bf16", "f32"):
        h, w, token, mask = draw(torch, 200, 900, 64, dtype)
        a, b = gradients(torch, 200)
        fwd = call(env, h, w, 1.0, token, mask, 0)
        both = call_grad(env, h, w, 1.0, token, mask, fwd["stat"], fwd["entropy"], a, b)
        only_h = call_grad(env, h, w, 1.0, token, mask, fwd["stat"], fwd["entropy"], a, b, grad_w=None)
        only_w = call_grad(env, h, w, 1.0, token, mask, fwd["stat"], fwd["entropy"], a, b, hidden=False)
        assert torch.equal(both["hidden"], only_h["hidden"]) and torch.equal(both["weight"], only_w["weight"])


@pytest.mark.parametrize("rows,vocab,dim,dtype", [(3, 600000, 8, "bf16"), (66000, 5000, 16, "bf16"), (5, 140001, 1027, "bf16"), (40, 70000, 520, "f32")])
def test_head_backward_pieces_of_the_vocabulary(env, rows, vocab, dim, dtype):
    torch, B = env
    h, w, token, mask = draw(torch, rows, vocab, dim, dtype)
    check_grad(env, h, w, 1.0, token, mask)


def test_head_backward_no_rows_and_smaller_calls(env):
    torch, B = env
    h, w, token, mask = draw(torch, 0, 300, 64, "bf16")
    none = torch.empty(0, device="cuda")
    got = call_grad(env, h, w, 1.0, token, None, torch.empty(0, 2, device="cuda"), none, none, none)
    assert not got["weight"].any()
    before = torch.randn(300, 64, device="cuda").to(torch.bfloat16)
    got = call_grad(env, h, w, 1.0, token, None, torch.empty(0, 2, device="cuda"), none, none, none, before=before)
    assert torch.equal(got["weight"], before)
    for dtype in ("bf16", "f32"):
        h, w, token, mask = draw(torch, 700, 3000, 72, dtype)
        last = 0
        for n in (1, 2, 16, 17, 64, 65, 127, 128, 129, 200, 256, 257, 384, 500, 640, 641, 700):
            need = B.dc_head_logprob_backward_workspace_bytes(B.make_matrix(h[:n]), B.make_matrix(w), B.make_matrix(w))
            assert need >= last
            last = need
        ws = torch.full((last,), 0xFF, dtype=torch.uint8, device="cuda")
        for n in (1, 17, 64, 129, 640):
            check_grad(env, h[:n], w, 1.0, token[:n], mask[:n], ws=ws)


def test_head_backward_against_differences(env):
    """The gradients are those of the forward call: differences of its outputs along random directions, in 32 bits."""
    torch, B = env
    h, w, token, mask = draw(torch, 12, 200, 32, "f32")
    a, b = gradients(torch, 12)
    fwd = call(env, h, w, 0.8, token, mask, 0)
    got = call_grad(env, h, w, 0.8, token, mask, fwd["stat"], fwd["entropy"], a, b)

    def loss(h2, w2):
        o = call(env, h2, w2, 0.8, token, mask, 0)
        return float((o["logprob"].double() * a.double()).sum() + (o["entropy"].double() * b.double()).sum())

    g = torch.Generator(device="cuda").manual_seed(5)
    step = 2.0 ** -7
    for name in ("hidden", "weight"):
        along = torch.randn((h if name == "hidden" else w).shape, generator=g, device="cuda") * (1.0 if name == "hidden" else 0.25)
        pair = [loss(h + s * step * along, w) if name == "hidden" else loss(h, w + s * step * along) for s in (1, -1)]
        diff = (pair[0] - pair[1]) / (2 * step)
        want = float((got[name].double() * along.double()).sum())
        # logits move by at most |along| |w| step: the third derivative's share, and the roundings of twelve values of about 8
        move = step * (float((along.double() @ w.double().t()).abs().max()) if name == "hidden" else float((h.double() @ along.double().t()).abs().max())) / 0.8
        size = float(a.abs().sum() + 8 * b.abs().sum())
        assert abs(diff - want) <= size * move ** 2 / step * move + 12 * 16 * U * 8 / step, (name, diff, want, move)


def test_head_repeats_bit_for_bit_on_another_stream_and_in_a_graph(env):
    torch, B = env
    for dtype, rows in (("bf16", 300), ("f32", 40)):
        h, w, token, mask = draw(torch, rows, 2000, 96, dtype)
        a, b = gradients(torch, rows)
        m = B.make_matrix

        def eager(stream=None):
            f = call(env, h, w, 0.9, token, mask, 0, stream=stream)
            t = call(env, h, w, 0.9, token, mask, 3, stream=stream)
            g = call_grad(env, h, w, 0.9, token, mask, f["stat"], f["entropy"], a, b, grad_w="f32", stream=stream)
            return [f["logprob"], f["stat"], f["entropy"], t["top_token"], t["top_logprob"], g["hidden"], g["weight"]], (f, t, g)

        first, _ = eager()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            other, keep = eager()
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, other))
        outs = [torch.empty_like(x) for x in first]
        need = max(B.dc_head_logprob_workspace_bytes(m(h), m(w), 3), B.dc_head_logprob_backward_workspace_bytes(m(h), m(w), m(outs[6])))
        ws, status = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        lp3, st3, en3 = (torch.empty_like(x) for x in first[:3])

        def all_calls():
            B.dc_head_logprob(m(h), m(w), 0.9, token, mask, 3, lp3, st3, en3, outs[3], outs[4], ws, need, status)
            B.dc_head_logprob(m(h), m(w), 0.9, token, mask, 0, outs[0], outs[1], outs[2], None, None, ws, need, status)
            B.dc_head_logprob_backward(m(h), m(w), 0.9, token, mask, outs[1], outs[2], a, b, m(outs[5]), False, m(outs[6]), ws, need, status)

        with torch.cuda.stream(s):
            all_calls()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            all_calls()
        for turn in range(4):
            h2, w2, t2, m2 = draw(torch, rows, 2000, 96, dtype, seed=turn + 1)
            for x, y in ((h, h2), (w, w2), (token, t2), (mask, m2)):
                x.copy_(y)
            for x in outs:
                x.fill_(-7)
            graph.replay()
            torch.cuda.synchronize()
            want, keep = eager()
            torch.cuda.synchronize()
            assert int(status) == 0
            assert all(torch.equal(x, y) for x, y in zip(outs, want)), turn


def test_residual_norm_head_and_back_together(env):
    """A step of a small model: the stream normed for the head, log-probabilities, and the gradients all the way back, against torch's
    own differentiation in 64 bits."""
    torch, B = env
    rows, dim, vocab, eps = 150, 256, 1111, 1e-6
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    block, stream = rand(rows, dim), rand(rows, dim) * 2
    post, pre = 1 + 0.1 * rand(1, dim), 1 + 0.1 * rand(1, dim)
    w = rand(vocab, dim) * (1.5 / math.sqrt(dim))
    token = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    mask = (torch.rand(rows, generator=g, device="cuda") < 0.8).to(torch.uint8)
    a, b = gradients(torch, rows)
    m = B.make_matrix
    h, out, st = torch.empty_like(stream), torch.empty_like(block), torch.empty(rows, 2, device="cuda")
    prm = B.make_norm(eps, 1.0, 0.5)
    B.dc_residual_norm(m(block), m(post), None, m(stream), m(pre), prm, m(h), m(out), st)
    f = call(env, out, w, 1.0, token, mask, 0)
    gr = call_grad(env, out, w, 1.0, token, mask, f["stat"], f["entropy"], a, b)
    need = B.dc_residual_norm_backward_workspace_bytes(m(block))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    db, ds, dpost, dpre = torch.empty_like(block), torch.empty_like(stream), torch.empty_like(post), torch.empty_like(pre)
    B.dc_residual_norm_backward(m(block), m(post), None, m(h), m(pre), prm, st, None, m(gr["hidden"]), m(db), m(ds), False, m(dpost), None,
                                m(dpre), ws, need)
    leaves = [x.double().requires_grad_() for x in (block, stream, post, pre, w)]
    bb, ss, po, pr, ww = leaves
    hh = ss + 0.5 * bb * (bb.square().mean(1, keepdim=True) + eps).rsqrt() * po
    y = hh * (hh.square().mean(1, keepdim=True) + eps).rsqrt() * pr
    lp = torch.log_softmax(y @ ww.t(), 1)
    live = mask.double()
    loss = (lp[torch.arange(rows), token.long()] * a.double() * live).sum() - ((lp.exp() * lp).sum(1) * b.double() * live).sum()
    want = torch.autograd.grad(loss, leaves)
    torch.cuda.synchronize()
    for got, ref in zip((db, ds, dpost, dpre, gr["weight"]), want):
        # 32 bits throughout: a few thousand roundings of sums whose terms cancel to no less than a hundredth of their size
        assert float((got.double() - ref).norm() / ref.norm()) < 3000 * 100 * U * 0.01
