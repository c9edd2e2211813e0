"""What the speed of the head's log-probabilities and of the residual norm is measured on.

Between the embedding of the packed tokens and their log-probabilities the actor's update has a decoder's residual stream and
its head.  Measured here: the residual stream's step from one block to the next (the block's result normed, gated and added,
the sum normed for the next block) with its gradient, and log-probabilities, entropy and top alternatives straight from hidden
states and the head's weights, without a matrix of logits, with the gradients of both.  The cases go from one decoded token to
a micro-batch of the long-tailed workload.  Vocabularies are those of ``workloads.py`` (32 000 and 152 064) and odd ones
beside them, token counts its micro-batch budgets and parts of them, widths those of the actor's update.

``own`` false: plain torch operations in 32 bits, rounded once at the end.  ``own`` true: the framework's kernels through
the binding.  Inputs come from the seed; a state holds what a program keeps between two calls (weights, outputs, workspaces).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _head(name, rows, vocab, dim, type_, **more):
    c = {"kind": "head", "rows": rows, "vocab": vocab, "dim": dim, "type": type_, "temperature": 1.0, "entropy": True,
         "top": 0, "loss_share": 1.0}
    return {**({"name": name} if name else {}), **c, **more}


def _head_grad(name, rows, vocab, dim, type_, **more):
    c = {"kind": "head_grad", "rows": rows, "vocab": vocab, "dim": dim, "type": type_, "temperature": 1.0, "entropy": True,
         "loss_share": 1.0, "grad": type_, "accumulate": False}
    return {**({"name": name} if name else {}), **c, **more}


def _norm(name, kind, rows, dim, act, residual, **more):
    # gate: "none", "column" (one factor for each column) or "token" (one for each element)
    c = {"kind": kind, "rows": rows, "dim": dim, "act": act, "residual": residual, "weight": act, "post": True, "pre": True,
         "gate": "column", "residual_scale": 1.0, "block_scale": 1.0}
    if kind == "norm_grad":
        c.update(grad="f32", accumulate=False)
    return {**({"name": name} if name else {}), **c, **more}


def listed():
    return [
        # one decoded token with five alternatives
        _head("head-decode-1", 1, 152064, 2048, "bf16", top=5),
        # a decode step of 64 sequences sampled at a temperature
        _head("head-decode-64", 64, 152064, 2048, "bf16", temperature=0.7, top=5),
        # a short ragged sequence of a small model in 32 bits, odd rows and columns
        _head("head-odd-32", 333, 32003, 515, "f32", temperature=0.8, loss_share=0.6),
        # a micro-batch of workload 1 scored by the actor: prompts (a quarter of the tokens) are masked
        _head("head-score-8192", 8192, 32000, 1024, "bf16", loss_share=0.75),
        # part of a micro-batch of the large vocabulary, scored with entropy
        _head("head-score-large", 8192, 152064, 2048, "bf16"),
        # the gradients of a ragged sequence, 16-bit floats with odd columns
        _head_grad("head-grad-odd", 517, 32003, 515, "f16", temperature=0.8, loss_share=0.6),
        # a micro-batch of workload 1, the weights' gradient added in 32 bits to what earlier micro-batches left
        _head_grad("head-grad-8192", 8192, 32000, 1024, "bf16", loss_share=0.75, grad="f32", accumulate=True),
        # the gradients at the large vocabulary
        _head_grad("head-grad-large", 8192, 152064, 2048, "bf16"),
        # one decoded token between two blocks
        _norm("norm-decode-1", "norm", 1, 2048, "bf16", "bf16"),
        # a whole micro-batch of the long-tailed workload, the residual stream in 32 bits
        _norm("norm-131072", "norm", 131072, 2048, "bf16", "f32"),
        # a ragged sequence of a small model, a gate for every element
        _norm("norm-grad-odd", "norm_grad", 777, 1365, "f32", "f32", gate="token", residual_scale=0.9, block_scale=0.5),
        # a whole micro-batch of the long-tailed workload
        _norm("norm-grad-131072", "norm_grad", 131072, 2048, "bf16", "bf16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["head", "head", "head_grad", "head_grad", "norm", "norm_grad"])
    type_ = rng.choice(["bf16", "bf16", "f32", "f16"])
    if kind in ("head", "head_grad"):
        vocab = rng.choice([32000, 152064, _spread(rng, 1000, 152064)])
        dim = rng.choice([512, 1024, 2048, _spread(rng, 64, 4096)])
        most = 8192 * 152064 * 2048 / (8 if type_ == "f32" else 1)           # (a product in 32 bits takes that much longer)
        rows = _spread(rng, 1, max(2, min(65536, int(most / vocab / dim), int(8192 * 152064 / vocab))))
        more = {"temperature": rng.choice([1.0, 1.0, 0.6, 1.3]), "entropy": rng.random() < 0.7,
                "loss_share": rng.choice([1.0, rng.uniform(0.3, 0.95)])}
        if kind == "head":
            if rows <= 512:
                more["top"] = rng.choice([0, 1, 5])
            return _head(None, rows, vocab, dim, type_, **more)
        return _head_grad(None, rows, vocab, dim, type_, grad=rng.choice([type_, "f32"]), accumulate=rng.random() < 0.5, **more)
    dim = rng.choice([512, 1024, 2048, 4096, _spread(rng, 64, 8192)])
    rows = _spread(rng, 1, int(131072 * 2048 / max(dim, 2048) / (2 if type_ == "f32" else 1)))
    more = {"weight": rng.choice([type_, "f32"]), "gate": rng.choice(["none", "column", "token"]),
            "residual_scale": rng.choice([1.0, rng.uniform(0.5, 1.5)]), "block_scale": rng.choice([1.0, rng.uniform(0.1, 1.0)])}
    more["post"] = rng.random() < 0.7
    more["pre"] = rng.random() < 0.9
    if kind == "norm_grad":
        more.update(grad=rng.choice(["f32", type_]), accumulate=rng.random() < 0.3)
    return _norm(None, kind, rows, dim, type_, rng.choice(["f32", type_]), **more)


# ---- inputs ----

EPS = 1e-6


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _head_inputs(case, g):
    rows, vocab, dim, t = case["rows"], case["vocab"], case["dim"], TYPES[case["type"]]
    weight = (_randn(g, vocab, dim) * (2.0 / math.sqrt(dim))).to(t)
    token = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    # logits spread by about 2; most given tokens are likely ones
    hidden = _randn(g, rows, dim) + 2.25 * _rand(g, rows, 1) * weight[token].float()
    s = {"hidden": hidden.to(t), "weight": weight, "token": token.to(torch.int32)}
    s["mask"] = None if case["loss_share"] >= 1.0 else (_rand(g, rows) < case["loss_share"]).to(torch.uint8)
    return s


def _norm_inputs(case, g):
    rows, dim, act = case["rows"], case["dim"], TYPES[case["act"]]
    s = {"block": (_randn(g, rows, dim) * torch.exp(0.5 * _randn(g, rows, 1))).to(act)}
    near_one = lambda *shape: (1.0 + 0.2 * _randn(g, *shape))  # noqa: E731
    s["post"] = near_one(1, dim).to(TYPES[case["weight"]]) if case["post"] else None
    s["pre"] = near_one(1, dim).to(TYPES[case["weight"]]) if case["pre"] else None
    s["gate"] = None if case["gate"] == "none" else near_one(1, dim).to(TYPES[case["weight"]]) if case["gate"] == "column" \
        else _rand(g, rows, dim).to(act)
    return s


def prepare(case, seed):
    g = _gen(seed)
    kind, rows, dim = case["kind"], case["rows"], case["dim"]
    s = {"case": case}
    if kind in ("head", "head_grad"):
        s.update(_head_inputs(case, g))
        if kind == "head":
            top = case["top"]
            s["logprob"] = torch.empty(rows, device=DEV)
            s["stat"] = torch.empty(rows, 2, device=DEV)
            s["entropy"] = torch.empty(rows, device=DEV) if case["entropy"] else None
            s["top_token"] = torch.empty(rows, top, dtype=torch.int32, device=DEV) if top else None
            s["top_logprob"] = torch.empty(rows, top, device=DEV) if top else None
        else:
            z = torch.mm(s["hidden"].float(), s["weight"].float().t())
            m = z.amax(1, keepdim=True)
            z.sub_(m).div_(case["temperature"])
            e = z.exp()
            total = e.sum(1)
            s["stat"] = torch.stack([m[:, 0], total.log()], 1)
            s["entropy"] = total.log() - e.mul_(z).sum(1) / total
            del z, e
            s["grad_logprob"] = _randn(g, rows) * 0.1
            s["grad_entropy"] = _randn(g, rows) * 0.01 if case["entropy"] else None
            s["grad_hidden"] = torch.empty_like(s["hidden"])
            s["grad_weight"] = (_randn(g, case["vocab"], dim) * 0.1).to(TYPES[case["grad"]])
    else:
        s.update(_norm_inputs(case, g))
        r, act = TYPES[case["residual"]], TYPES[case["act"]]
        # a residual stream several blocks deep
        stream = (_randn(g, rows, dim) * 3.0).to(r)
        if kind == "norm":
            s["stream"], s["stream_out"] = stream, torch.empty_like(stream)
            s["out"] = torch.empty(rows, dim, dtype=act, device=DEV) if case["pre"] else None
            s["stat"] = torch.empty(rows, 2, device=DEV)
        else:
            s["stream_out"] = stream
            root = lambda x: (x.float().square().mean(1) + EPS).rsqrt()  # noqa: E731
            s["stat"] = torch.stack([root(s["block"]), root(stream)], 1)
            s["grad_stream_out"] = (_randn(g, rows, dim) * 0.1).to(r)
            s["grad_out"] = (_randn(g, rows, dim) * 0.1).to(act) if case["pre"] else None
            s["grad_block"] = torch.empty_like(s["block"])
            s["grad_stream"] = torch.empty_like(stream)
            for name in ("post", "pre", "gate"):
                if s[name] is None:
                    s["grad_" + name] = None
                elif name == "gate" and case["gate"] == "token":
                    s["grad_gate"] = torch.empty_like(s["gate"])
                else:
                    s["grad_" + name] = _randn(g, 1, dim).to(TYPES[case["grad"]])
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the framework makes once: the status word and workspaces."""
    from paper_2507_13833_amd import binding as B
    case, m = s["case"], B.make_matrix
    s["B"], s["status"] = B, torch.zeros(1, dtype=torch.int32, device=DEV)
    n = 0
    if case["kind"] == "head":
        n = B.dc_head_logprob_workspace_bytes(m(s["hidden"]), m(s["weight"]), case["top"])
    elif case["kind"] == "head_grad":
        n = B.dc_head_logprob_backward_workspace_bytes(m(s["hidden"]), m(s["weight"]), m(s["grad_weight"]))
    elif case["kind"] == "norm_grad":
        n = B.dc_residual_norm_backward_workspace_bytes(m(s["block"]))
    s["ws_bytes"] = n
    s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def run(state):
    return _RUN[state["case"]["kind"]][1 if own else 0](state)


def _outputs(s, *names):
    return {k: s[k] for k in names}


_HEAD = ("logprob", "stat", "entropy", "top_token", "top_logprob")
_HEAD_GRAD = ("grad_hidden", "grad_weight")
_NORM = ("stream_out", "out", "stat")
_NORM_GRAD = ("grad_block", "grad_stream", "grad_gate", "grad_post", "grad_pre")


# ---- the framework's operators ----

def _matrix(s, name):
    return None if s[name] is None else s["B"].make_matrix(s[name])


def _norm_params(s):
    case = s["case"]
    return s["B"].make_norm(EPS, case["residual_scale"], case["block_scale"], gate_rows=case["gate"] == "token")


def _own_head(s):
    case = s["case"]
    s["B"].dc_head_logprob(_matrix(s, "hidden"), _matrix(s, "weight"), case["temperature"], s["token"], s["mask"], case["top"],
                           s["logprob"], s["stat"], s["entropy"], s["top_token"], s["top_logprob"], s["ws"], s["ws_bytes"],
                           s["status"])
    return _outputs(s, *_HEAD)


def _own_head_grad(s):
    case = s["case"]
    s["B"].dc_head_logprob_backward(_matrix(s, "hidden"), _matrix(s, "weight"), case["temperature"], s["token"], s["mask"],
                                    s["stat"], s["entropy"], s["grad_logprob"], s["grad_entropy"], _matrix(s, "grad_hidden"),
                                    case["accumulate"], _matrix(s, "grad_weight"), s["ws"], s["ws_bytes"], s["status"])
    return _outputs(s, *_HEAD_GRAD)


def _own_norm(s):
    s["B"].dc_residual_norm(_matrix(s, "block"), _matrix(s, "post"), _matrix(s, "gate"), _matrix(s, "stream"),
                            _matrix(s, "pre"), _norm_params(s),
                            _matrix(s, "stream_out"), _matrix(s, "out"), s["stat"])
    return _outputs(s, *_NORM)


def _own_norm_grad(s):
    case = s["case"]
    s["B"].dc_residual_norm_backward(
        _matrix(s, "block"), _matrix(s, "post"), _matrix(s, "gate"), _matrix(s, "stream_out"), _matrix(s, "pre"),
        _norm_params(s), s["stat"], _matrix(s, "grad_stream_out"),
        _matrix(s, "grad_out"), _matrix(s, "grad_block"), _matrix(s, "grad_stream"), case["accumulate"],
        _matrix(s, "grad_post"), _matrix(s, "grad_gate"), _matrix(s, "grad_pre"), s["ws"], s["ws_bytes"])
    return _outputs(s, *_NORM_GRAD)


# ---- the plain form ----

def _top(x, n):
    """The n largest of every row and their columns, ties to the lowest column."""
    value, column = torch.sort(x, dim=1, descending=True, stable=True)
    return value[:, :n], column[:, :n]


def _plain_head(s):
    case = s["case"]
    x = torch.mm(s["hidden"].float(), s["weight"].float().t())
    keep = torch.ones(case["rows"], dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    m = x.amax(1, keepdim=True)
    z = (x - m) / case["temperature"]
    e = z.exp()
    total = e.sum(1)
    log_sum = total.log()
    out = {"top_token": None, "top_logprob": None, "entropy": None}
    out["logprob"] = (z.gather(1, s["token"].long()[:, None])[:, 0] - log_sum).where(keep, 0.0)
    out["stat"] = torch.stack([m[:, 0], log_sum], 1).where(keep[:, None], 0.0)
    if case["entropy"]:
        out["entropy"] = (log_sum - (e * z).sum(1) / total).where(keep, 0.0)
    if case["top"]:
        value, column = _top(x, case["top"])
        out["top_token"] = column.where(keep[:, None], -1).to(torch.int32)
        out["top_logprob"] = ((value - m) / case["temperature"] - log_sum[:, None]).where(keep[:, None], 0.0)
    return out


def _plain_head_grad(s):
    case = s["case"]
    hidden, weight = s["hidden"].float(), s["weight"].float()
    logp = (torch.mm(hidden, weight.t()) - s["stat"][:, :1]) / case["temperature"] - s["stat"][:, 1:]
    p = logp.exp()
    a = s["grad_logprob"][:, None]
    d = -a * p
    if s["grad_entropy"] is not None:
        d -= s["grad_entropy"][:, None] * p * (logp + s["entropy"][:, None])
    d.scatter_add_(1, s["token"].long()[:, None], a)
    d /= case["temperature"]
    if s["mask"] is not None:
        d = d.where(s["mask"][:, None] != 0, 0.0)
    s["grad_hidden"].copy_(torch.mm(d, weight))
    dw = torch.mm(d.t(), hidden)
    s["grad_weight"].copy_(dw + s["grad_weight"].float() if case["accumulate"] else dw)
    return _outputs(s, *_HEAD_GRAD)


def _root(x):
    return (x.square().mean(1, keepdim=True) + EPS).rsqrt()


def _plain_norm(s):
    case = s["case"]
    b = s["block"].float()
    r1, r2 = torch.zeros(case["rows"], 1, device=DEV), torch.zeros(case["rows"], 1, device=DEV)
    if case["post"]:
        r1 = _root(b)
        b = b * r1 * s["post"].float()
    if s["gate"] is not None:
        b = b * s["gate"].float()
    h = s["stream"].float() * case["residual_scale"] + b * case["block_scale"]
    s["stream_out"].copy_(h)
    if case["pre"]:
        r2 = _root(h)
        s["out"].copy_(h * r2 * s["pre"].float())
    s["stat"].copy_(torch.cat([r1, r2], 1))
    return _outputs(s, *_NORM)


def _plain_norm_grad(s):
    case = s["case"]
    dh = s["grad_stream_out"].float()
    sums = {}
    if case["pre"]:
        dy, r2 = s["grad_out"].float(), s["stat"][:, 1:]
        n = s["stream_out"].float() * r2
        sums["grad_pre"] = (dy * n).sum(0, keepdim=True)
        dn = dy * s["pre"].float()
        dh = dh + r2 * (dn - n * (dn * n).mean(1, keepdim=True))
    s["grad_stream"].copy_(dh * case["residual_scale"])
    du = dh * case["block_scale"]
    b, r1 = s["block"].float(), s["stat"][:, :1]
    n = b * r1 if case["post"] else b
    u = n * s["post"].float() if case["post"] else b
    if s["gate"] is not None:
        sums["grad_gate"] = du * u
        if case["gate"] == "column":
            sums["grad_gate"] = sums["grad_gate"].sum(0, keepdim=True)
        du = du * s["gate"].float()
    if case["post"]:
        sums["grad_post"] = (du * n).sum(0, keepdim=True)
        dn = du * s["post"].float()
        du = r1 * (dn - n * (dn * n).mean(1, keepdim=True))
    s["grad_block"].copy_(du)
    for name, v in sums.items():
        add = case["accumulate"] and not (name == "grad_gate" and case["gate"] == "token")
        s[name].copy_(v + s[name].float() if add else v)
    return _outputs(s, *_NORM_GRAD)


_RUN = {"head": (_plain_head, _own_head), "head_grad": (_plain_head_grad, _own_head_grad),
        "norm": (_plain_norm, _own_norm), "norm_grad": (_plain_norm_grad, _own_norm_grad)}


# ---- what a pass cannot do without ----

def work(case):
    kind, n, d = case["kind"], case["rows"], case["dim"]
    if kind in ("head", "head_grad"):
        live, v, size = n * case["loss_share"], case["vocab"], SIZE[case["type"]]
        if kind == "head":
            out = 4 + 8 + 4 * case["entropy"] + 8 * case["top"]
            return {"bytes": (live + v) * d * size + n * (out + 4), "flops": live * v * (2 * d + 5 + 2 * case["entropy"])}
        dw = SIZE[case["grad"]] * (2 if case["accumulate"] else 1)
        return {"bytes": (live + n + v) * d * size + v * d * dw + n * 24, "flops": live * v * (6 * d + 6 + 3 * case["entropy"])}
    a, r = SIZE[case["act"]], SIZE[case["residual"]]
    gate = a if case["gate"] == "token" else 0
    if kind == "norm":
        return {"bytes": n * d * (a + gate + 2 * r + a * case["pre"]) + 8 * n, "flops": 12 * n * d}
    return {"bytes": n * d * (2 * a + 2 * gate + 3 * r + a * case["pre"]) + 8 * n, "flops": 30 * n * d}


# ---- the definition in 64 bits ----

def _exact_head(case, s):
    f64 = torch.float64
    hidden, weight = s["hidden"].to(f64), s["weight"].to(f64)
    token, at = s["token"].long(), torch.arange(case["rows"], device=DEV)
    dead = torch.zeros(case["rows"], dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] == 0
    x = hidden @ weight.t().contiguous()
    if case["kind"] == "head_grad":
        # p from the given statistics: dx = (a (one-hot - p) - b p (log p + H)) / T
        logp = x.sub_(s["stat"][:, 0].to(f64)[:, None]).div_(case["temperature"]).sub_(s["stat"][:, 1].to(f64)[:, None])
        a = s["grad_logprob"].to(f64)
        weigh = a[:, None]
        if case["entropy"]:
            weigh = (logp + s["entropy"].to(f64)[:, None]).mul_(s["grad_entropy"].to(f64)[:, None]).add_(weigh)
        dx = logp.exp_().mul_(weigh).neg_()
        dx[at, token] += a
        dx /= case["temperature"]
        dx[dead] = 0.0
        dw = dx.t().contiguous() @ hidden
        if case["accumulate"]:
            dw += s["grad_weight"].to(f64)
        return {"grad_hidden": dx @ weight, "grad_weight": dw}
    logp = torch.log_softmax(x / case["temperature"], 1)
    high = x.max(1).values
    out = {"logprob": logp[at, token].masked_fill(dead, 0.0), "entropy": None, "top_token": None, "top_logprob": None}
    out["stat"] = torch.stack([high, torch.logsumexp((x - high[:, None]) / case["temperature"], 1)], 1)
    out["stat"][dead] = 0.0
    if case["top"]:
        best, where = torch.topk(x, case["top"], dim=1)
        out["top_token"] = where.masked_fill(dead[:, None], -1).to(torch.int32)
        out["top_logprob"] = logp.gather(1, where).masked_fill(dead[:, None], 0.0)
    if case["entropy"]:
        out["entropy"] = torch.xlogy(p := logp.exp(), p).sum(1).neg().masked_fill(dead, 0.0)
    return out


def _exact_norm(case, s):
    """The gradient by torch's own differentiation of the forward pass, with the given statistics as the norms' factors where
    these enter as such and as functions of their rows where they are differentiated."""
    f64 = torch.float64
    b = s["block"].to(f64)
    post, pre, gate = (None if s[k] is None else s[k].to(f64) for k in ("post", "pre", "gate"))
    if case["kind"] == "norm":
        r1 = 1 / torch.sqrt((b * b).sum(1) / case["dim"] + EPS)
        u = b if post is None else post * (b * r1[:, None])
        h = case["residual_scale"] * s["stream"].to(f64) + case["block_scale"] * (u if gate is None else gate * u)
        r2 = 1 / torch.sqrt((h * h).sum(1) / case["dim"] + EPS)
        zero = torch.zeros_like(r1)
        return {"stream_out": h, "out": None if pre is None else pre * (h * r2[:, None]),
                "stat": torch.stack([zero if post is None else r1, zero if pre is None else r2], 1)}
    out = {k: None for k in _NORM_GRAD}
    before = {k: s[k].to(f64) for k in ("grad_post", "grad_pre", "grad_gate") if s[k] is not None and s[k].shape[0] == 1 and case["accumulate"]
              and not (k == "grad_gate" and case["gate"] == "token")}

    def through_norm(x, r, w, dy):
        """Gradients of w * x * r(x) for r = (mean x^2 + eps)^(-1/2), whose derivative along x is -r^3 x / dim."""
        dyw = dy * w
        along = (dyw * x).sum(1, keepdim=True)
        return dyw * r - x * (r ** 3) * along / case["dim"], (dy * x * r).sum(0, keepdim=True)

    dh = s["grad_stream_out"].to(f64)
    if pre is not None:
        more, out["grad_pre"] = through_norm(s["stream_out"].to(f64), s["stat"][:, 1:].to(f64), pre, s["grad_out"].to(f64))
        dh = dh + more
    out["grad_stream"] = case["residual_scale"] * dh
    db, r1 = case["block_scale"] * dh, s["stat"][:, :1].to(f64)
    if gate is not None:
        dg = db * (b if post is None else post * b * r1)
        out["grad_gate"] = dg if case["gate"] == "token" else dg.sum(0, keepdim=True)
        db = db * gate
    if post is not None:
        db, out["grad_post"] = through_norm(b, r1, post, db)
    out["grad_block"] = db
    for k, v in before.items():
        out[k] = out[k] + v
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _exact_head(case, s) if case["kind"] in ("head", "head_grad") else _exact_norm(case, s)
