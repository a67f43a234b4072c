"""The example's gradients against autograd of the same layer in float64, and that it runs with what it keeps in 8 bits.

Tolerance, in norms: between the weights and a gradient lie at most 8 roundings to bf16 (2^-8 of a value each, at random signs), which
gives 2^-5; with keep8 the kept values are off by half a step, a block's largest over 127.5 or half of that: below 2^-6 of a
normal block's size. The router's gradient is a difference of the experts' shares, whose errors stay: twice that.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def plain(model, tokens, targets, chosen, dloss):
    """Losses and gradients in float64, for a given choice of experts."""
    w = {n: t.double().requires_grad_() for n, t in model.w.items()}
    x = w["embed"][tokens]
    score = torch.sigmoid(x @ w["router"])
    idx = chosen.long()
    picked = score.gather(1, idx)
    weights = picked / picked.sum(1, keepdim=True)
    out = x
    for j in range(idx.shape[1]):
        h = torch.einsum("td,tdf->tf", x, w["up"][idx[:, j]])
        a = h * torch.sigmoid(h) if model.keep8 else torch.relu(h)
        out = out + weights[:, j:j + 1] * torch.einsum("tf,tfd->td", a, w["down"][idx[:, j]])
    logp = torch.log_softmax(out @ w["head"], -1)
    loss = -logp.gather(1, targets[:, None]).squeeze(1)
    loss.backward(dloss.double())
    return loss.detach(), {n: t.grad for n, t in w.items()}


@pytest.mark.parametrize("keep8", [False, True])
def test_gradients(keep8):
    import train_moe
    model = train_moe.Model(vocab=512, d=64, f=96, experts=4, seed=3, keep8=keep8)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens, targets = (torch.randint(0, 512, (200,), generator=g, device="cuda") for _ in range(2))
    dloss = torch.rand(200, generator=g, device="cuda") / 200
    loss, s = model.forward(tokens, targets)
    model.backward(s, dloss)
    want_loss, want = plain(model, tokens, targets, s["chosen"], dloss)
    assert float((loss.double() - want_loss).abs().max()) < 2.0**-5
    bound = 2.0**-5 + (2.0**-6 if keep8 else 0.0)
    for n, grad in model.g.items():
        error = float((grad.double() - want[n]).norm() / want[n].norm())
        assert error < (2 * bound if n == "router" else bound), (n, error)
    model.opt.close()


def test_runs_with_what_it_keeps_in_8_bits():
    import train_moe
    first, last = train_moe.train(steps=20, tokens=512, log=lambda s: print(s, flush=True), keep8=True)
    assert first > 0 and last > 0
