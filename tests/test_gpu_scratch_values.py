"""What lies in memory before a call has no part in its result: the scratch and the outputs come from blocks that held NaN."""
import pytest
import torch

import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def dirty():
    """NaN (all bits set) in the allocator's free blocks."""
    torch.cuda.synchronize()
    blocks = [torch.full((n,), -1, dtype=torch.int32, device=DEV) for n in [64, 256, 4096, 1 << 16, 1 << 18] * 6 + [1 << 22, 1 << 24, 1 << 26] * 4]
    del blocks


LOSS = [(1, 40, 100), (3, 33, 17), (70, 31, 257), (5, 64, 20003), (300, 130, 777), (600, 1000, 905), (700, 2033, 377), (2048, 520, 1001),
        (1100, 1024, 4096)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", LOSS, ids=lambda c: "x".join(map(str, c)))
def test_loss(case, tied):
    T, d, V = case
    g = torch.Generator(device=DEV).manual_seed(T)
    x, w = torch.randn(T, d, generator=g, device=DEV).to(BF), (torch.randn(V, d, generator=g, device=DEV) * 0.05).to(BF)
    w = w if tied else w.T.contiguous()
    targets = torch.randint(-1, V, (T,), generator=g, device=DEV)
    dloss = torch.rand(T, generator=g, device=DEV)

    def run():
        loss, lse = P.head_loss(x, w, targets, tied=tied)
        return (loss, lse, *P.head_loss_backward(x, w, targets, lse, dloss, tied=tied))
    want = [t.clone() for t in run()]
    assert all(bool(t.isfinite().all()) for t in want)
    for _ in range(2):
        dirty()
        assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize("dy_type", [BF, F32])
@pytest.mark.parametrize("case", [(40, 3, 2, 33, 17), (300, 8, 2, 1000, 264), (500, 4, 1, 1031, 301)], ids=lambda c: "x".join(map(str, c)))
def test_weights_gradient_from_kept_rows(case, dy_type):
    T, E, k, n, m = case
    g = torch.Generator(device=DEV).manual_seed(T)
    experts = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].int().contiguous()
    experts[::7] = -1
    x, dy = torch.randn(T, n, generator=g, device=DEV).to(BF), torch.randn(T * k, m, generator=g, device=DEV).to(dy_type)

    def run():
        plan = P.expert_rows(experts, E)
        kept = P.keep8(x)
        return P.restore8(kept), P.expert_matmul_grad(kept, dy, plan, gather=True)
    want = [t.clone() for t in run()]
    assert all(bool(t.isfinite().all()) for t in want)
    for _ in range(2):
        dirty()
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
