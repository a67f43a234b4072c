"""The example's gradients in a later step, after the optimizer has moved the weights and with what an earlier batch left in every buffer,
against autograd in float64 at the weights of that step. Tolerance as in test_gpu_example.py."""
import pytest
import torch

from test_gpu_example import plain   # (puts examples/ on the path)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep8", [False, True])
def test_gradients_of_a_later_step(keep8):
    import train_moe
    model = train_moe.Model(vocab=512, d=64, f=96, experts=4, seed=5, keep8=keep8)
    g = torch.Generator(device="cuda").manual_seed(2)
    bound = 2.0**-5 + (2.0**-6 if keep8 else 0.0)
    before = {n: w.clone() for n, w in model.w.items()}
    for step, n in enumerate((333, 200, 57), 1):   # batches of other sizes
        tokens, targets = (torch.randint(0, 512, (n,), generator=g, device="cuda") for _ in range(2))
        dloss = torch.rand(n, generator=g, device="cuda") / n
        loss, s = model.forward(tokens, targets)
        model.backward(s, dloss)
        assert bool(loss.isfinite().all())
        want_loss, want = plain(model, tokens, targets, s["chosen"], dloss)
        assert float((loss.double() - want_loss).abs().max()) < 2.0**-5
        for name, grad in model.g.items():
            error = float((grad.double() - want[name]).norm() / want[name].norm())
            assert error < (2 * bound if name == "router" else bound), (step, name, error)
        model.balance(s["plan"])
        model.opt.step(step, lr=0.01, max_grad_norm=1.0)
    torch.cuda.synchronize()
    assert all(not torch.equal(w, before[n]) for n, w in model.w.items())
    model.opt.close()
