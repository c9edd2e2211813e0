"""What the speed of the actor's update operators is measured on.

The packed training layout that the reshard makes is read by the actor's update: the embedding of its token ids, the
log-probabilities (with entropy and top alternatives) of those ids under the head's logits, the gradients of both, and
the AdamW step over all weights.  The cases go from one row of a decode step to a micro-batch of the long-tailed workload.
Vocabularies are those of ``workloads.py`` (32 000 and 152 064) and odd ones beside them; token counts are its
micro-batch budgets and parts of them.

``own`` false: plain torch operations in 32 bits, rounded once at the end.  ``own`` true: the framework's kernels through
the binding.  Inputs come from the seed; a state holds what a program keeps between two calls (weights, optimizer
states, outputs, workspaces, the optimizer's table).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                                     # elements that share a scale of an 8-bit optimizer state


def _logprob(name, rows, vocab, type_, **more):
    c = {"kind": "logprob", "rows": rows, "vocab": vocab, "type": type_, "temperature": 1.0, "entropy": True, "top": 0,
         "loss_share": 1.0, "banned": 0.0}
    return {**({"name": name} if name else {}), **c, **more}


def _logprob_grad(name, rows, vocab, type_, **more):
    c = {"kind": "logprob_grad", "rows": rows, "vocab": vocab, "type": type_, "temperature": 1.0, "entropy": True,
         "loss_share": 1.0}
    return {**({"name": name} if name else {}), **c, **more}


def _embedding(name, kind, tokens, vocab, dim, weight, act, **more):
    c = {"kind": kind, "tokens": tokens, "vocab": vocab, "dim": dim, "weight": weight, "act": act, "skew": 4.0}
    if kind == "embedding_grad":
        c["accumulate"] = False
    return {**({"name": name} if name else {}), **c, **more}


def _adamw(name, layers, dim, inner, vocab, state, **more):
    c = {"kind": "adamw", "layers": layers, "dim": dim, "inner": inner, "vocab": vocab, "state": state, "param": "bf16",
         "grad": "bf16", "master": True}
    return {**({"name": name} if name else {}), **c, **more}


def listed():
    return [
        # one decoded token: its log-probability, entropy and five alternatives, some tokens banned by the sampler
        _logprob("logprob-decode-1", 1, 152064, "bf16", top=5, banned=0.01),
        # a decode step of 64 sequences, logits in 32 bits, sampled at a temperature, twenty alternatives
        _logprob("logprob-decode-64", 64, 152064, "f32", top=20, temperature=0.7),
        # a micro-batch of workload 1 scored by the actor: prompts (a quarter of the tokens) are masked
        _logprob("logprob-score-8192", 8192, 32000, "bf16", loss_share=0.75),
        # part of a micro-batch of the large vocabulary, scored with entropy
        _logprob("logprob-score-large", 8192, 152064, "bf16"),
        # a short ragged sequence on a vocabulary with odd rows, 32-bit logits
        _logprob_grad("logprob-grad-odd", 333, 32003, "f32", temperature=0.8, loss_share=0.6),
        # the gradient of the large vocabulary's logits, prompts masked
        _logprob_grad("logprob-grad-large", 8192, 152064, "bf16", loss_share=0.75),
        # the next token of 64 sequences
        _embedding("embedding-decode-64", "embedding", 64, 152064, 2048, "bf16", "bf16"),
        # a whole micro-batch of the long-tailed workload
        _embedding("embedding-131072", "embedding", 131072, 152064, 2048, "bf16", "bf16"),
        # a micro-batch of workload 1, gradient added to what earlier micro-batches left
        _embedding("embedding-grad-8192", "embedding_grad", 8192, 32000, 1024, "f32", "bf16", accumulate=True),
        # a whole micro-batch of the long-tailed workload
        _embedding("embedding-grad-131072", "embedding_grad", 131072, 152064, 2048, "f32", "bf16"),
        # the step of a small model, everything in 32 bits: many tensors, the norms among them tiny
        _adamw("adamw-small-32", 12, 512, 1365, 32000, 32, param="f32", grad="f32", master=False),
        # the step of a larger one with 8-bit states and 32-bit master weights
        _adamw("adamw-large-8", 6, 2048, 5461, 152064, 8),
    ]


def _spread(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "logprob_grad", "embedding", "embedding_grad", "adamw"])
    type_ = rng.choice(["bf16", "bf16", "f32", "f16"])
    vocab = rng.choice([32000, 152064, _spread(rng, 1000, 152064)])
    if kind in ("logprob", "logprob_grad"):
        rows = _spread(rng, 1, max(2, int(8192 * 152064 * 2 / vocab / SIZE[type_] / 2)))
        rows = min(rows, 65536)
        more = {"temperature": rng.choice([1.0, 1.0, 0.6, 1.3]), "entropy": rng.random() < 0.7,
                "loss_share": rng.choice([1.0, rng.uniform(0.3, 0.95)])}
        if kind == "logprob":
            more["banned"] = rng.choice([0.0, 0.0, 0.02])
            if rows <= 1024:
                more["top"] = rng.choice([0, 1, 5, 20])
            return _logprob(None, rows, vocab, type_, **more)
        return _logprob_grad(None, rows, vocab, type_, **more)
    if kind == "embedding":
        dim = rng.choice([512, 1024, 2048, 4096, _spread(rng, 100, 4096)])
        tokens = _spread(rng, 1, max(2, int(131072 * 2048 * 2 / dim / 4)))
        return _embedding(None, kind, min(tokens, 131072), vocab, dim, rng.choice(["f32", "bf16"]), type_,
                          skew=rng.choice([1.0, 4.0]))
    if kind == "embedding_grad":
        dim = rng.choice([512, 1024, 2048, _spread(rng, 100, 2048)])
        tokens = _spread(rng, 1, 131072)
        return _embedding(None, kind, tokens, vocab, dim, rng.choice(["f32", "bf16"]), type_,
                          accumulate=rng.random() < 0.5, skew=rng.choice([1.0, 4.0]))
    dim = rng.choice([256, 512, 1024, _spread(rng, 64, 1024)])
    grad = rng.choice(["f32", "bf16"])
    param = rng.choice(["f32", "bf16"])
    return _adamw(None, rng.randint(1, 12), dim, _spread(rng, 2 * dim, 4 * dim), 32000, rng.choice([8, 32]), grad=grad,
                  param=param, master=param != "f32" and rng.random() < 0.7)


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 11)
    return g


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _logits(case, g):
    rows, vocab = case["rows"], case["vocab"]
    x = _randn(g, rows, vocab).mul_(2.0)
    token = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    at = torch.arange(rows, device=DEV)
    x[at, token] += 9.0 * _rand(g, rows)                     # most tokens are likely ones
    if case.get("banned"):
        ban = torch.randperm(vocab, generator=g, device=DEV)[: int(case["banned"] * vocab)]
        x[:, ban] = -math.inf
        x[at, token] = 4.0                                   # a sampled token is not a banned one
    return x.to(TYPES[case["type"]]), token.to(torch.int32)


def _mask(case, g):
    return None if case["loss_share"] >= 1.0 else (_rand(g, case["rows"]) < case["loss_share"]).to(torch.uint8)


def _tokens(case, g):
    """Ids as text has them: the lowest often, most of the vocabulary hardly ever."""
    u = _rand(g, case["tokens"]).double() ** case["skew"]
    return (u * case["vocab"]).long().clamp_(max=case["vocab"] - 1).to(torch.int32)


def _shapes(case):
    """(elements, whether weight decay applies) of every tensor of a decoder, those with decay first."""
    d, f = case["dim"], case["inner"]
    big = [case["vocab"] * d] + [n for _ in range(case["layers"]) for n in (d * d, d * d, d * d, d * d, d * f, d * f, d * f)]
    small = [d for _ in range(case["layers"]) for _ in range(2)] + [d]
    return [(n, True) for n in big] + [(n, False) for n in small]


def _places(case):
    """Where each tensor lies in the flat buffers (every one starts on a block's border), the first element without decay
    and the buffers' length."""
    at, end, no_decay = [], 0, None
    for n, decay in _shapes(case):
        if not decay and no_decay is None:
            no_decay = end
        at.append((end, n, decay))
        end += -(-n // BLOCK) * BLOCK
    return at, no_decay, end


LR, BETAS, EPS, DECAY, STEP = 3e-4, (0.9, 0.95), 1e-8, 0.1, 20

FP8 = torch.float8_e4m3fn                       # what an 8-bit state holds, times its block's scale
FP8_MOST, FP8_LEAST = 448.0, 2.0 ** -9


def _adamw_inputs(case, g):
    places, no_decay, n = _places(case)
    used = torch.zeros(n // BLOCK, BLOCK, dtype=torch.bool, device=DEV)
    flat = used.view(-1)
    for at, count, _ in places:
        flat[at:at + count] = True
    # blocks differ in size, and so do the values in them
    size = torch.exp(2.0 * _randn(g, n // BLOCK, 1))
    grad = (_randn(g, n // BLOCK, BLOCK) * size * 1e-3).mul_(used).view(-1)
    s = {"grad": grad.to(TYPES[case["grad"]]), "grad_scale": torch.tensor([0.37], device=DEV), "step": STEP,
         "places": places, "no_decay": no_decay}
    w = (_randn(g, n // BLOCK, BLOCK) * 0.02).mul_(used).view(-1)
    s["param"] = w.to(TYPES[case["param"]])
    s["master"] = w if case["master"] else None
    m = (_randn(g, n // BLOCK, BLOCK) * size * 3e-4).mul_(used)
    v = ((_randn(g, n // BLOCK, BLOCK) * size * 4e-4) ** 2).mul_(used)
    if case["state"] == 32:
        s["m"], s["v"] = m.view(-1), v.view(-1)
        s["m_scale"] = s["v_scale"] = None
    else:
        s["m"], s["m_scale"] = _encode(m, False)
        s["v"], s["v_scale"] = _encode(v.sqrt(), True)
    return s


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("logprob", "logprob_grad"):
        rows = case["rows"]
        s["logits"], s["token"] = _logits(case, g)
        s["mask"] = _mask(case, g)
        if kind == "logprob_grad":
            m = s["logits"].amax(1, keepdim=True).double()
            z = s["logits"].double().sub_(m).div_(case["temperature"])
            e = z.exp()
            total = e.sum(1)
            s["stat"] = torch.stack([m[:, 0], total.log()], 1).float()
            s["entropy"] = (total.log() - e.mul_(z).sum(1) / total).float()
            del z, e
            s["grad_logprob"] = _randn(g, rows) * 0.1
            s["grad_entropy"] = _randn(g, rows) * 0.01 if case["entropy"] else None
            s["grad_logits"] = torch.empty_like(s["logits"])
        else:
            top = case["top"]
            s["logprob"] = torch.empty(rows, device=DEV)
            s["stat"] = torch.empty(rows, 2, device=DEV)
            s["entropy"] = torch.empty(rows, device=DEV) if case["entropy"] else None
            s["top_token"] = torch.empty(rows, top, dtype=torch.int32, device=DEV) if top else None
            s["top_logprob"] = torch.empty(rows, top, device=DEV) if top else None
    elif kind == "embedding":
        s["token"] = _tokens(case, g)
        s["weight"] = (_randn(g, case["vocab"], case["dim"]) * 0.02).to(TYPES[case["weight"]])
        s["out"] = torch.empty(case["tokens"], case["dim"], dtype=TYPES[case["act"]], device=DEV)
    elif kind == "embedding_grad":
        s["token"] = _tokens(case, g)
        s["grad_out"] = (_randn(g, case["tokens"], case["dim"]) * 0.1).to(TYPES[case["act"]])
        s["grad_weight"] = (_randn(g, case["vocab"], case["dim"]) * 0.1).to(TYPES[case["weight"]])
    else:
        s.update(_adamw_inputs(case, g))
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the framework makes once: the status word, workspaces, the optimizer's table."""
    from paper_2507_13833_amd import binding as B
    case = s["case"]
    s["B"], s["status"] = B, torch.zeros(1, dtype=torch.int32, device=DEV)
    n = 0
    if case["kind"] == "logprob":
        n = B.dc_token_logprob_workspace_bytes(B.make_matrix(s["logits"]), case["top"])
    elif case["kind"] == "embedding_grad":
        n = B.dc_embedding_backward_workspace_bytes(B.make_matrix(s["grad_out"]), B.make_matrix(s["grad_weight"]))
    elif case["kind"] == "adamw":
        part = lambda name, at, n: None if s[name] is None else s[name][at:at + n]  # noqa: E731
        s["tensors"] = B.AdamwTensors([
            dict(param=part("param", at, n), master=part("master", at, n), grad=part("grad", at, n),
                 exp_avg=part("m", at, n), exp_avg_sq=part("v", at, n),
                 exp_avg_scale=part("m_scale", at // BLOCK, -(-n // BLOCK)),
                 exp_avg_sq_scale=part("v_scale", at // BLOCK, -(-n // BLOCK)), weight_decay=DECAY if decay else 0.0)
            for at, n, decay in s["places"]])
        n = B.dc_adamw_table_bytes(s["tensors"])
    s["ws_bytes"] = n
    s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    if case["kind"] == "adamw":
        B.dc_adamw_table(s["tensors"], s["ws"], n)


def run(state):
    return _RUN[state["case"]["kind"]][1 if own else 0](state)


# ---- the framework's operators ----

def _own_logprob(s):
    B, case = s["B"], s["case"]
    B.dc_token_logprob(B.make_matrix(s["logits"]), case["temperature"], s["token"], s["mask"], case["top"], s["logprob"],
                       s["stat"], s["entropy"], s["top_token"], s["top_logprob"], s["ws"], s["ws_bytes"], s["status"])
    return {k: s[k] for k in ("logprob", "stat", "entropy", "top_token", "top_logprob")}


def _own_logprob_grad(s):
    B, case = s["B"], s["case"]
    B.dc_token_logprob_backward(B.make_matrix(s["logits"]), case["temperature"], s["token"], s["mask"], s["stat"], s["entropy"],
                                s["grad_logprob"], s["grad_entropy"], B.make_matrix(s["grad_logits"]), s["status"])
    return {"grad_logits": s["grad_logits"]}


def _own_embedding(s):
    B, case = s["B"], s["case"]
    B.dc_embedding(B.make_matrix(s["weight"]), s["token"], math.sqrt(case["dim"]), B.make_matrix(s["out"]), s["status"])
    return {"out": s["out"]}


def _own_embedding_grad(s):
    B, case = s["B"], s["case"]
    B.dc_embedding_backward(B.make_matrix(s["grad_out"]), s["token"], math.sqrt(case["dim"]), case["accumulate"],
                            B.make_matrix(s["grad_weight"]), s["ws"], s["ws_bytes"], s["status"])
    return {"grad_weight": s["grad_weight"]}


def _own_adamw(s):
    B = s["B"]
    B.dc_adamw(s["tensors"], B.make_adamw(LR, *BETAS, EPS, s["step"]), s["grad_scale"], s["ws"], s["ws_bytes"], s["status"])
    s["step"] += 1
    return _adamw_outputs(s)


# ---- the plain form ----

def _top(x, n):
    """The n largest of every row and their columns, ties to the lowest column: one integer that sorts as (value, -column)."""
    bits = (x + 0.0).view(torch.int32)                       # (a zero's sign does not count)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
    key += 0xFFFFFFFF - torch.arange(x.shape[1], device=x.device)
    column = 0xFFFFFFFF - (torch.topk(key, n, dim=1).values & 0xFFFFFFFF)
    return column, torch.gather(x, 1, column)


def _plain_logprob(s):
    case = s["case"]
    x = s["logits"].float()
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
        out["entropy"] = (log_sum - (e * z.clamp(min=-1e4)).sum(1) / total).where(keep, 0.0)
    if case["top"]:
        column, value = _top(x, case["top"])
        out["top_token"] = column.where(keep[:, None], -1).to(torch.int32)
        out["top_logprob"] = ((value - m) / case["temperature"] - log_sum[:, None]).where(keep[:, None], 0.0)
    return out


def _plain_logprob_grad(s):
    case = s["case"]
    logp = (s["logits"].float() - s["stat"][:, :1]) / case["temperature"] - s["stat"][:, 1:]
    p = logp.exp()
    gl = s["grad_logprob"][:, None]
    d = -gl * p
    if s["grad_entropy"] is not None:
        d -= s["grad_entropy"][:, None] * p * (logp + s["entropy"][:, None])
    d.scatter_add_(1, s["token"].long()[:, None], gl)
    d /= case["temperature"]
    if s["mask"] is not None:
        d = d.where(s["mask"][:, None] != 0, 0.0)
    s["grad_logits"].copy_(d)
    return {"grad_logits": s["grad_logits"]}


def _plain_embedding(s):
    out = s["weight"][s["token"].long()].float() * math.sqrt(s["case"]["dim"])
    s["out"].copy_(out)
    return {"out": s["out"]}


def _plain_embedding_grad(s):
    case = s["case"]
    total = torch.zeros(case["vocab"], case["dim"], device=DEV)
    total.index_add_(0, s["token"].long(), s["grad_out"].float())
    total *= math.sqrt(case["dim"])
    if case["accumulate"]:
        total += s["grad_weight"].float()
    s["grad_weight"].copy_(total)
    return {"grad_weight": s["grad_weight"]}


def _divided(a, b):
    """a / b, rounded once to 32 bits: a code next to a border must not go by how a division is made."""
    return (a.double() / b.double()).float()


def _decode(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _encode(y, keep):
    """Blocks [n, BLOCK] of 32-bit values as 8-bit ones and a scale each.  `keep`: a value that is not zero stays one that
    is not (a root that is divided by)."""
    scale = _divided(y.abs().amax(1), torch.tensor(FP8_MOST, device=DEV))
    scale = scale.where(scale >= 2.0 ** -120, 0.0)
    inverse = _divided(torch.ones_like(scale), scale).where(scale > 0, 0.0)
    a = y * inverse[:, None]
    if keep:
        a = torch.where(a > 0, a.clamp(min=FP8_LEAST), a)
    return a.to(FP8).view(-1), scale


def _adamw_outputs(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale")}


def _plain_adamw(s):
    case, t = s["case"], s["step"]
    b1, b2 = BETAS
    g = s["grad"].float() * s["grad_scale"]
    if case["state"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, root = _decode(s["m"], s["m_scale"]), _decode(s["v"], s["v_scale"])
        v = root * root
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    root = v.double().sqrt().float()
    w = (s["param"].float() if s["master"] is None else s["master"]).clone()
    w[: s["no_decay"]] *= 1 - LR * DECAY
    w -= LR / (1 - b1 ** t) * (m / (root * (1 / math.sqrt(1 - b2 ** t)) + EPS))
    s["param"].copy_(w)
    if s["master"] is not None:
        s["master"].copy_(w)
    if case["state"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for name, x in (("m", m), ("v", root)):
            code, scale = _encode(x.view(-1, BLOCK), name == "v")
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
    s["step"] = t + 1
    return _adamw_outputs(s)


_RUN = {"logprob": (_plain_logprob, _own_logprob), "logprob_grad": (_plain_logprob_grad, _own_logprob_grad),
        "embedding": (_plain_embedding, _own_embedding), "embedding_grad": (_plain_embedding_grad, _own_embedding_grad),
        "adamw": (_plain_adamw, _own_adamw)}


# ---- what a pass cannot do without ----

def _touched(case):
    """How many ids of the vocabulary a draw of _tokens names, on average."""
    v, n, k = case["vocab"], case["tokens"], case["skew"]
    steps = 2000                                              # id = v u^k: the share of draws below x is (x / v)^(1/k)
    total, before = 0.0, 0.0
    for i in range(1, steps + 1):
        upto = i / steps
        share = (upto ** (1 / k) - before ** (1 / k)) / max(1.0, v / steps)
        total += (upto - before) * v * -math.expm1(n * math.log1p(-min(share, 1 - 1e-12)))
        before = upto
    return min(total, n, v)


def work(case):
    kind = case["kind"]
    if kind in ("logprob", "logprob_grad"):
        live, size = case["rows"] * case["loss_share"], SIZE[case["type"]]
        if kind == "logprob":
            out = 4 + 8 + 4 * case["entropy"] + 8 * case["top"]
            return {"bytes": live * case["vocab"] * size + case["rows"] * (out + 4),
                    "flops": live * case["vocab"] * (5 + 2 * case["entropy"])}
        return {"bytes": live * case["vocab"] * size + case["rows"] * (case["vocab"] * size + 24),
                "flops": live * case["vocab"] * (6 + 3 * case["entropy"])}
    if kind in ("embedding", "embedding_grad"):
        n, d, w, a = case["tokens"], case["dim"], SIZE[case["weight"]], SIZE[case["act"]]
        touched = _touched(case)
        if kind == "embedding":
            return {"bytes": n * (4 + d * a) + touched * d * w, "flops": n * d}
        rows = 2 * touched if case["accumulate"] else case["vocab"]
        return {"bytes": n * (4 + d * a) + rows * d * w, "flops": 2 * n * d}
    n = sum(count for count, _ in _shapes(case))
    p = 2 * SIZE[case["param"]] if not case["master"] else SIZE[case["param"]] + 8
    state = 16 if case["state"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (p + SIZE[case["grad"]] + state), "flops": 16 * n}


# ---- the definition in 64 bits ----

def _eight_bits(y, keep):
    """What blocks of 64-bit values are in 8 bits, by looking each up between the midpoints of what 8 bits can hold."""
    held = torch.tensor([math.ldexp(c, -9) if c < 8 else math.ldexp(8 + c % 8, c // 8 - 10) for c in range(127)],
                        dtype=torch.float64, device=DEV)
    y = y.view(-1, BLOCK)
    scale = y.abs().amax(1, keepdim=True) / FP8_MOST
    scale = torch.where(scale >= 2.0 ** -120, scale, 0.0)
    a = torch.where(scale > 0, y.abs() / scale, 0.0)
    code = torch.searchsorted((held[1:] + held[:-1]) / 2, a)
    if keep:
        code = torch.where(a > 0, code.clamp(min=1), code)
    return (held[code] * y.sign()).to(FP8).view(-1), scale[:, 0]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f64 = torch.float64
    kind = case["kind"]
    if kind in ("logprob", "logprob_grad"):
        x = s["logits"].to(f64)
        live = torch.ones(x.shape[0], dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].bool()
        logp = torch.log_softmax(x / case["temperature"], 1)
        p = logp.exp()
        token = s["token"].long()
        at = torch.arange(x.shape[0], device=DEV)
        entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
        if kind == "logprob_grad":
            d = p.neg().mul_(s["grad_logprob"].to(f64)[:, None])
            d[at, token] += s["grad_logprob"].to(f64)
            if case["entropy"]:
                d -= logp.add_(entropy[:, None]).mul_(p).mul_(s["grad_entropy"].to(f64)[:, None])
            d /= case["temperature"]
            d[~live] = 0.0
            return {"grad_logits": d}
        dead = ~live
        out = {"logprob": logp[at, token].masked_fill(dead, 0.0), "entropy": None, "top_token": None, "top_logprob": None}
        high = x.max(1).values
        out["stat"] = torch.stack([high, torch.logsumexp((x - high[:, None]) / case["temperature"], 1)], 1)
        out["stat"][dead] = 0.0
        if case["entropy"]:
            out["entropy"] = entropy.masked_fill(dead, 0.0)
        if case["top"]:
            best, where = x.sort(dim=1, descending=True, stable=True)
            where = where[:, : case["top"]]
            out["top_token"] = where.masked_fill(dead[:, None], -1).to(torch.int32)
            out["top_logprob"] = logp.gather(1, where).masked_fill(dead[:, None], 0.0)
        return out
    if kind == "embedding":
        return {"out": torch.index_select(s["weight"].to(f64), 0, s["token"].long()) * case["dim"] ** 0.5}
    if kind == "embedding_grad":
        base = s["grad_weight"].to(f64) * (1.0 if case["accumulate"] else 0.0)
        return {"grad_weight": base.index_add(0, s["token"].long(), s["grad_out"].to(f64), alpha=case["dim"] ** 0.5)}
    b1, b2 = BETAS
    g = s["grad"].to(f64) * float(s["grad_scale"])
    if case["state"] == 32:
        m, v = s["m"].to(f64), s["v"].to(f64)
    else:
        m, root = (s[k].to(f64) * s[k + "_scale"].to(f64).repeat_interleave(BLOCK) for k in ("m", "v"))
        v = root ** 2
    m.mul_(b1).add_(g, alpha=1 - b1)
    v.mul_(b2).addcmul_(g, g, value=1 - b2)
    w = (s["param"] if s["master"] is None else s["master"]).to(f64)
    shrink = torch.ones_like(w)
    shrink[: s["no_decay"]] -= LR * DECAY
    rate = LR * m / (1 - b1 ** STEP)
    w = w * shrink - rate / ((v / (1 - b2 ** STEP)).sqrt() + EPS)
    out = {"param": w, "master": w if case["master"] else None, "m_scale": None, "v_scale": None}
    if case["state"] == 32:
        return {**out, "m": m, "v": v}
    out["m"], out["m_scale"] = _eight_bits(m, False)
    out["v"], out["v_scale"] = _eight_bits(v.sqrt(), True)
    return out
