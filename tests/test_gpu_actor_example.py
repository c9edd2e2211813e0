"""The example's gradients against torch's own differentiation in 64 bits."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_actor_update_gradients():
    import torch
    spec = importlib.util.spec_from_file_location("actor_update", os.path.join(ROOT, "examples", "actor_update.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    vocab, dim, n = 700, 64, 201
    actor = m.Actor(vocab, dim, 400)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = [torch.randint(0, vocab, (n,), generator=g, device="cuda").to(torch.int32) for _ in range(2)]
    masks = [(torch.rand(n, generator=g, device="cuda") < 0.7).to(torch.uint8) for _ in range(2)]
    a = [torch.randn(n - 1, generator=g, device="cuda") * 0.3 for _ in range(2)]
    b = [torch.randn(n - 1, generator=g, device="cuda") * 0.1 for _ in range(2)]
    for k in range(2):                                        # two micro-batches, the second one's gradients added
        hidden = actor.hidden(ids[k])
        logprob, entropy, stat = actor.score(hidden, ids[k], masks[k], 0.9)
        actor.backward(hidden, ids[k], masks[k], 0.9, stat, entropy, a[k], b[k], first=k == 0)
    torch.cuda.synchronize()
    assert int(actor.status) == 0
    leaves = [it["param"].double().requires_grad_() for it in (actor.embed, actor.head, actor.block, actor.post, actor.pre)]
    e, h, w, post, pre = leaves
    loss = 0.0
    for k in range(2):
        x = e[ids[k][:-1].long()] * actor.scale
        y = x @ w
        s = x + 0.5 * y * (y.square().mean(1, keepdim=True) + 1e-6).rsqrt() * post
        lp = torch.log_softmax(s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * pre @ h.t() / 0.9, 1)
        live = masks[k][1:].double()
        loss = loss + (live * (lp[torch.arange(n - 1), ids[k][1:].long()] * a[k].double() - (lp.exp() * lp).sum(1) * b[k].double())).sum()
    want = torch.autograd.grad(loss, leaves)
    for it, ref in zip((actor.embed, actor.head, actor.block, actor.post, actor.pre), want):
        # a value on the way is rounded to 16 bits (2^-8 of it at most) no more than eight times: embedding, block, stream, its norm,
        # three gradients and their sum
        assert float((it["grad"].double() - ref).norm() / ref.norm()) < 8 * 2.0 ** -8


def example():
    spec = importlib.util.spec_from_file_location("actor_update", os.path.join(ROOT, "examples", "actor_update.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
def test_actor_update_gradients_with_logits_kept():
    """As without: a matrix of logits and one of their gradient are two roundings to 16 bits more than the eight of the test above."""
    import torch
    m = example()
    vocab, dim, n = 700, 64, 201
    actors = [m.Actor(vocab, dim, 400, keep_logits=k) for k in (False, True)]
    g = torch.Generator(device="cuda").manual_seed(4)
    for k in range(2):
        ids = torch.randint(0, vocab, (n,), generator=g, device="cuda").to(torch.int32)
        mask = (torch.rand(n, generator=g, device="cuda") < 0.7).to(torch.uint8)
        a, b = torch.randn(n - 1, generator=g, device="cuda") * 0.3, torch.randn(n - 1, generator=g, device="cuda") * 0.1
        for actor in actors:
            hidden = actor.hidden(ids)
            logprob, entropy, stat = actor.score(hidden, ids, mask, 0.9)
            actor.backward(hidden, ids, mask, 0.9, stat, entropy, a, b, first=k == 0)
    torch.cuda.synchronize()
    for x, y in zip(*(actor.items for actor in actors)):
        assert float((x["grad"] - y["grad"]).norm() / x["grad"].norm()) < (8 + 10) * 2.0 ** -8
    assert all(int(actor.status) == 0 for actor in actors)


@pytest.mark.gpu
@pytest.mark.parametrize("keep_logits", [False, True])
def test_actor_update_runs(keep_logits):
    history = example().main(prompts=2, epochs=2, keep_logits=keep_logits)
    assert len(history) == 2 and all(abs(x) < float("inf") for step in history for x in step)
