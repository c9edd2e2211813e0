"""How far the head's products may be off where each factor has so many bits, in root mean square over many results.

The tolerances of single values add up every rounding at its worst, so on long rows they would hold with a factor that is cut to half
its bits.  Roundings do not conspire: of n errors that are independent of each other, the sum's standard deviation is the root of the
sum of squares.  Here a factor of `bits` bits is off by at most 2^-bits of itself and a product of two, with the product of their
smallest parts that is left off, by 3 times that; the products' errors join as squares.  Additions in 32 bits (of the 32 products of
parts that an instruction of the matrix cores sums, four, each given two roundings' worth: 2 U of the sum until then, which is at
most the root of x^2 + sum of squares in root mean square) join as squares too.  Everything works on any device.
"""
import math

U = 2.0 ** -24


def joined(*parts):
    return sum(p * p for p in parts) ** 0.5


def rms(x):
    return float(x.double().square().mean().sqrt())


def product_bound(torch, left, right, off, parts):
    """left (n x k) times right (m x k): the product in 64 bits, and how far it may be off in root mean square where each product of two
    factors is off by `off` of itself (a number, or one for each element of left)."""
    x = left @ right.t().contiguous()
    squares = right.square().t().contiguous()
    size = (left.square() @ squares).sqrt()
    lost = ((left * off).square() @ squares).sqrt()
    return x, joined(lost, 2 * U * math.sqrt(parts * left.shape[1] / 8) * joined(x, size))


def forward(torch, h, w, temperature, token, x_bound):
    """What the logits' own bound makes of a row's results: exact values and bounds."""
    x, dx = x_bound
    n, vocab = x.shape
    top, at = x.max(1)
    z = (x - top[:, None]) / temperature
    log_sum = z.exp().sum(1).log()
    logp = z - log_sum[:, None]
    p = logp.exp()
    entropy = -(p * logp).sum(1)
    # behind the logits: z, its power and a sum over the vocabulary
    soft = U * (6 * (p * z.abs()).sum(1) + 6 + 2 * log_sum.abs() + math.sqrt(vocab))
    dz, rows = dx / temperature, torch.arange(n, device=x.device)
    t = token.long()
    zt, lt = z[rows, t], logp[rows, t]
    want = {"top": top, "logprob": lt, "entropy": entropy}
    bound = {"top": dx[rows, at], "logprob": joined(dz[rows, t], (p * dz).square().sum(1).sqrt(), soft + U * (3 * zt.abs() + lt.abs())),
             "entropy": joined((p * (logp + entropy[:, None]) * dz).square().sum(1).sqrt(), soft * (2 + (p * z.abs()).sum(1)))}
    return want, bound


def alternatives(torch, x_bound, temperature, top_token, top_logprob):
    """Differences of alternatives' log-probabilities from the first one's are those of logits: got, exact, bound."""
    x, dx = x_bound
    v, d = (y.gather(1, top_token.long()) / temperature for y in (x, dx))
    lp = top_logprob.double()
    z = v - v[:, :1]
    return lp - lp[:, :1], z, joined(d, d[:, :1], U * (3 * z.abs() + lp.abs() + lp[:, :1].abs()))


def logits_gradient(torch, x_bound, temperature, token, stat, entropy, a, b):
    """G of all rows from the given statistics: its value, how far off it may be of itself, and the largest possible of each row."""
    x, dx = x_bound
    st, ad, bd, hd = stat.double(), a.double()[:, None] / temperature, b.double()[:, None] / temperature, entropy.double()[:, None]
    z = (x - st[:, :1]) / temperature
    logp = z - st[:, 1:]
    g = -logp.exp() * (ad + bd * (logp + hd))
    dlog = dx / temperature + U * (6 * z.abs() + 4 * st[:, 1:].abs() + 4)
    dg = g.abs() * (dlog + 10 * U) + logp.exp() * bd.abs() * (dlog + 2 * U * (logp.abs() + hd.abs()))
    own = torch.zeros_like(g)
    own[torch.arange(len(g), device=x.device), token.long()] = 1.0
    g = g + own * ad
    return g, (dg + own * ad.abs() * 4 * U) / g.abs().clamp(min=1e-300), ad.abs() + bd.abs() * (hd.abs() + 1)


def off_by(got, want, bound):
    """The root mean square of what it is off, in units of the bound's."""
    return rms(got.double() - want) / rms(bound)
