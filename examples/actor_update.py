"""The actor's update on a repacked GRPO batch, from end to end on one GPU.

A rollout batch goes through the reshard (balance, advantages, plan, gather); one data-parallel rank's micro-batches then
go through a small actor: the embedding of their token ids, a linear block whose normed result joins the residual stream, the
stream normed for the head, the log-probabilities of the next tokens without a matrix of logits (or, with --keep-logits, from a
matrix of them, which a program that does more with its logits has anyway), the clipped policy objective
with an entropy bonus, and back, and AdamW with 8-bit states steps on 32-bit master weights.
The actor is a bigram model (the next token's logits come from the current token's embedding alone): what it learns is not
the point, what it calls is.

    python examples/actor_update.py [--keep-logits]
"""
from __future__ import annotations

import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

from paper_2507_13833_amd import binding as B
from paper_2507_13833_amd import runner, workloads


class Actor:
    """Weights, gradients and optimizer states of the model, and the calls of its forward and backward pass."""

    def __init__(self, vocab: int, dim: int, max_tokens: int, device: str = "cuda:0", seed: int = 0, keep_logits: bool = False):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.dim, self.scale = dim, dim ** 0.5
        self.items = []

        def item(rows, std, mean=0.0, decay=0.01):
            master = mean + torch.randn(rows, dim, generator=gen, device=device) * std
            n, blocks = rows * dim, -(-rows * dim // B.DC_STATE_BLOCK)
            state = lambda: torch.zeros(n, dtype=torch.float8_e4m3fn, device=device)  # noqa: E731
            self.items.append(dict(param=master.bfloat16(), master=master, grad=torch.zeros(rows, dim, device=device),
                                   exp_avg=state(), exp_avg_sq=state(), exp_avg_scale=torch.zeros(blocks, device=device),
                                   exp_avg_sq_scale=torch.zeros(blocks, device=device), weight_decay=decay))
            return self.items[-1]

        self.embed, self.head = item(vocab, 0.3 / self.scale), item(vocab, 0.3 / self.scale)
        self.block = item(dim, 1.0 / self.scale)
        self.post, self.pre = item(1, 0.0, 1.0, 0.0), item(1, 0.0, 1.0, 0.0)   # the norms' weights
        self.norm = B.make_norm(1e-6, 1.0, 0.5)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        # what the calls need is laid out once: the optimizer's table, activations and workspaces for the largest micro-batch
        self.tensors = B.AdamwTensors(self.items)
        self.table_bytes = B.dc_adamw_table_bytes(self.tensors)
        self.table = torch.empty(self.table_bytes, dtype=torch.uint8, device=device)
        B.dc_adamw_table(self.tensors, self.table, self.table_bytes)
        new = lambda dtype, cols=dim: torch.empty(max_tokens, cols, dtype=dtype, device=device)  # noqa: E731
        self.act = {"embed": new(torch.bfloat16), "block": new(torch.bfloat16), "stream": new(torch.bfloat16),
                    "normed": new(torch.bfloat16), "stat": new(torch.float32, 2)}
        self.grad = {k: new(torch.bfloat16) for k in ("normed", "block", "stream")}
        m = B.make_matrix
        normed, head = m(self.act["normed"]), m(self.head["param"])
        self.logits = new(torch.bfloat16, vocab) if keep_logits else None
        of_head = [B.dc_token_logprob_workspace_bytes(m(self.logits), 5)] if keep_logits else \
            [B.dc_head_logprob_workspace_bytes(normed, head, 5),
             B.dc_head_logprob_backward_workspace_bytes(normed, head, m(self.head["grad"]))]
        self.ws_bytes = max(*of_head, B.dc_residual_norm_backward_workspace_bytes(normed),
                            B.dc_embedding_backward_workspace_bytes(normed, m(self.embed["grad"])))
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.steps = 0

    def hidden(self, ids: torch.Tensor) -> torch.Tensor:
        """The normed residual stream of the tokens behind ids[:-1]; row t is for ids[t + 1]."""
        n, m = ids.numel() - 1, B.make_matrix
        a = self.a = {k: v[:n] for k, v in self.act.items()}
        B.dc_embedding(m(self.embed["param"]), ids, self.scale, m(a["embed"]), self.status)
        torch.mm(a["embed"], self.block["param"], out=a["block"])
        B.dc_residual_norm(m(a["block"]), m(self.post["param"]), None, m(a["embed"]), m(self.pre["param"]), self.norm,
                           m(a["stream"]), m(a["normed"]), a["stat"])
        return a["normed"]

    def logprob(self, hidden, temperature, *rest) -> None:
        """The head's log-probabilities of rows of hidden states: what follows is dc_token_logprob's."""
        m = B.make_matrix
        if self.logits is None:
            B.dc_head_logprob(m(hidden), m(self.head["param"]), temperature, *rest, self.ws, self.ws_bytes, self.status)
        else:
            logits = self.logits[:hidden.shape[0]]
            torch.mm(hidden, self.head["param"].t(), out=logits)
            B.dc_token_logprob(m(logits), temperature, *rest, self.ws, self.ws_bytes, self.status)

    def score(self, hidden, ids, mask, temperature: float):
        """log-probability and entropy of every next token whose mask byte is set (0 elsewhere), and what their gradient needs."""
        n = hidden.shape[0]
        logprob, entropy = torch.empty(n, device=hidden.device), torch.empty(n, device=hidden.device)
        stat = torch.empty(n, 2, device=hidden.device)
        self.logprob(hidden, temperature, ids[1:], mask[1:], 0, logprob, stat, entropy, None, None)
        return logprob, entropy, stat

    def backward(self, hidden, ids, mask, temperature, stat, entropy, grad_logprob, grad_entropy, first: bool) -> None:
        """Gradients of all weights, added to those of the micro-batches before unless this is the first."""
        n, m, a = hidden.shape[0], B.make_matrix, self.a
        g = {k: v[:n] for k, v in self.grad.items()}
        if self.logits is None:
            B.dc_head_logprob_backward(m(hidden), m(self.head["param"]), temperature, ids[1:], mask[1:], stat, entropy, grad_logprob,
                                       grad_entropy, m(g["normed"]), not first, m(self.head["grad"]), self.ws, self.ws_bytes,
                                       self.status)
        else:                                                                  # the logits' gradient takes their place
            logits = self.logits[:n]
            B.dc_token_logprob_backward(m(logits), temperature, ids[1:], mask[1:], stat, entropy, grad_logprob, grad_entropy,
                                        m(logits), self.status)
            torch.mm(logits, self.head["param"], out=g["normed"])
            if first:
                self.head["grad"].zero_()
            self.head["grad"] += torch.mm(logits.t(), hidden)
        B.dc_residual_norm_backward(m(a["block"]), m(self.post["param"]), None, m(a["stream"]), m(self.pre["param"]), self.norm, a["stat"],
                                    None, m(g["normed"]), m(g["block"]), m(g["stream"]), not first, m(self.post["grad"]), None,
                                    m(self.pre["grad"]), self.ws, self.ws_bytes)
        if first:
            self.block["grad"].zero_()
        self.block["grad"] += torch.mm(a["embed"].t(), g["block"])
        grad_embed = torch.addmm(g["stream"], g["block"], self.block["param"].t())
        B.dc_embedding_backward(m(grad_embed), ids, self.scale, not first, m(self.embed["grad"]), self.ws, self.ws_bytes, self.status)

    def step(self, lr: float, max_norm: float = 1.0) -> None:
        """AdamW on gradients whose norm is cut to max_norm; the factor stays on the device."""
        self.steps += 1
        norm = torch.sqrt(sum(it["grad"].square().sum() for it in self.items))
        factor = (max_norm / (norm + 1e-6)).clamp(max=1.0).reshape(1)
        B.dc_adamw(self.tensors, B.make_adamw(lr, 0.9, 0.95, 1e-8, self.steps), factor, self.table, self.table_bytes, self.status)


def micro_batches(d: runner.DeviceBatch, shard: int):
    """Token ranges of a shard's micro-batches in the arenas."""
    n_mb = int(d.n_mb.item())
    mb = d.mb_seq_off[: n_mb + 1].tolist()
    tok = d.dst_tok_off.tolist()
    ends = d.shard_tok_off.tolist()
    lo, hi = d.shard_mb_off[shard].item(), d.shard_mb_off[shard + 1].item()
    first_slot = d.shard_seq_off.tolist()
    return [(tok[mb[m]], tok[mb[m + 1]] if mb[m + 1] < first_slot[shard + 1] else ends[shard + 1]) for m in range(lo, hi)]


def main(prompts: int = 16, epochs: int = 4, dim: int = 64, lr: float = 3e-3, clip: float = 0.2, entropy_coef: float = 1e-3,
         temperature: float = 1.0, verbose: bool = True, keep_logits: bool = False):
    vocab = 32000                                                              # workload 1's
    w = workloads.make_workload(1, prompts=prompts)
    d = runner.DeviceBatch(w)
    d.step_two_calls()                                                         # balance, advantages, plan; gather
    spans = micro_batches(d, 0)
    ids, mask = d.dst_fields["token_id"], d.dst_fields["mask"]
    adv = d.dst_fields["adv_tok"].view(torch.float32)
    actor = Actor(vocab, dim, max(b - a for a, b in spans), keep_logits=keep_logits)
    n_loss = max(1, sum(int(mask[a + 1:b].ne(0).sum()) for a, b in spans))
    old, history = {}, []
    for epoch in range(epochs):
        objective = entropy_sum = 0.0
        for m, (a, b) in enumerate(spans):
            t, k, adv_m = ids[a:b], mask[a:b], adv[a + 1:b]
            hidden = actor.hidden(t)
            logprob, entropy, stat = actor.score(hidden, t, k, temperature)
            if epoch == 0:
                old[m] = logprob.clone()                                       # the policy that the batch is scored with
            ratio = torch.exp(logprob - old[m])
            kept = torch.where(adv_m >= 0, ratio <= 1 + clip, ratio >= 1 - clip)
            objective += float((torch.minimum(ratio * adv_m, ratio.clamp(1 - clip, 1 + clip) * adv_m) * (k[1:] != 0)).sum())
            entropy_sum += float(entropy.sum())
            # what is made smaller: -(objective + entropy_coef * entropy) / tokens
            actor.backward(hidden, t, k, temperature, stat, entropy, -ratio * adv_m * kept / n_loss,
                           torch.full_like(entropy, -entropy_coef / n_loss), first=m == 0)
        actor.step(lr)
        history.append((objective / n_loss, entropy_sum / n_loss))
        if verbose:
            print(f"epoch {epoch}: objective {history[-1][0]:+.5f}  entropy {history[-1][1]:.4f}", flush=True)
    torch.cuda.synchronize()
    assert d.read_status() == 0 and int(actor.status) == 0
    if verbose:
        # the serving form: the next token behind the last one, with its likeliest alternatives
        hidden = actor.hidden(ids[spans[-1][1] - 2:spans[-1][1]])
        top, top_lp = torch.empty(1, 5, dtype=torch.int32, device=hidden.device), torch.empty(1, 5, device=hidden.device)
        actor.logprob(hidden, temperature, None, None, 5, None, None, None, top, top_lp)
        print("alternatives:", [(i, round(p, 4)) for i, p in zip(top[0].tolist(), top_lp[0].tolist())])
    return history


if __name__ == "__main__":
    main(keep_logits="--keep-logits" in sys.argv[1:])
