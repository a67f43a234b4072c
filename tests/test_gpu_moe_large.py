"""The experts' products at the sizes where larger tiles, shared contractions and long lists take over, and all operators
where offsets pass 32 bits: against float64 (tests/moe_ref.py), with the bounds of tests/test_gpu_moe.py; and the
example, which runs the operators together with the optimizer."""
import os
import sys

import pytest
import torch

import moe_ref as ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = (got - want).abs() > bound
    assert not bad.any() and not got.isnan().any(), (what, int(bad.sum()), float((got - want).abs().max()))


def bound(K, size, want, dtype):
    return 2 * (K + 8) * ref.U32 * size + want.abs() * (ref.UBF if dtype == BF else ref.U32) + 1e-38


# T, E, k, n, m (the contraction runs over n forward, over m backward): tiles of 256 x 256, 128 x 256, 64 x 256, and shared
# contractions; then rows of any length
FORWARD = [(4096, 2, 2, 72, 4104), (4096, 2, 2, 64, 4104), (2100, 16, 2, 168, 4104), (1000, 64, 1, 96, 2056),
           (3, 4, 2, 2104, 136), (1, 2, 1, 8192, 64), (1500, 4, 1, 37, 5501), (3, 4, 2, 2101, 131), (40, 4, 2, 4100, 33)]


@pytest.mark.parametrize("transpose", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("case", FORWARD, ids=lambda c: "x".join(map(str, c)))
def test_large_matmul(case, transpose):
    T, E, k, K, cols = case
    n, m = (cols, K) if transpose else (K, cols)
    g = torch.Generator().manual_seed(T + K)
    experts = ref.draw_experts(T, E, k, g, none=0.03)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    w = torch.randn(E, n, m, generator=g).to(BF)
    scale = torch.randn(T, k, generator=g)
    for gather, dtype, s in ((True, BF, None), (False, F32, scale)):
        x = torch.randn(T if gather else T * k, K, generator=g).to(BF)
        kw = dict(gather=gather, transpose=transpose, scale=s)
        want, size = ref.matmul(x, w, off, row, k, **kw), ref.matmul(x, w, off, row, k, absolute=True, **kw)
        args = (x.to(DEV), w.to(DEV), plan)
        kw = dict(gather=gather, transpose=transpose, scale=None if s is None else s.to(DEV), dtype=dtype)
        got = P.expert_matmul(*args, **kw)
        near(got, want, bound(K, size, want, dtype), (gather, dtype))
        assert torch.equal(got, P.expert_matmul(*args, **kw))


# T, E, k, n, m: tiles of 256 x 256, 128 x 256, 64 x 128 with more places than one list holds; rows of any length
WEIGHTS = [(1100, 3, 1, 3000, 3800), (420, 8, 2, 1024, 2056), (2500, 1, 1, 64, 72), (1400, 2, 2, 72, 136),
           (500, 4, 1, 1031, 2001), (2500, 1, 1, 65, 71), (300, 70, 2, 130, 264)]


@pytest.mark.parametrize("case", WEIGHTS, ids=lambda c: "x".join(map(str, c)))
def test_large_matmul_grad(case):
    T, E, k, n, m = case
    g = torch.Generator().manual_seed(T + n)
    experts = ref.draw_experts(T, E, k, g, none=0.03)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    K = int((off[1:] - off[:-1]).max())
    dy = torch.randn(T * k, m, generator=g).to(BF)
    for gather in (False, True):
        x = torch.randn(T if gather else T * k, n, generator=g).to(BF)
        want, size = (ref.matmul_grad(x, dy, off, row, k, gather, absolute=a) for a in (False, True))
        got = P.expert_matmul_grad(x.to(DEV), dy.to(DEV), plan, gather=gather)
        near(got, want, bound(K, size, want, BF), gather)
        assert torch.equal(got, P.expert_matmul_grad(x.to(DEV), dy.to(DEV), plan, gather=gather))


def test_results_do_not_depend_on_other_experts_rows():
    """The same tokens with more tokens for another expert: their rows have the same bits while the kernel is the same."""
    g = torch.Generator().manual_seed(3)
    w = torch.randn(3, 256, 512, generator=g).to(BF).to(DEV)
    x = torch.randn(900, 256, generator=g).to(BF).to(DEV)
    experts = (torch.arange(900) % 3).int()[:, None]
    base = P.expert_matmul(x, w, P.expert_rows(experts.to(DEV), 3), gather=True)
    experts[600:, 0] = 2
    plan = P.expert_rows(experts.to(DEV), 3)
    other = P.expert_matmul(x, w, plan, gather=True)
    first = P.expert_rows((torch.arange(900) % 3).int()[:, None].to(DEV), 3).slots[:600, 0].long()
    assert torch.equal(base[first], other[plan.slots[:600, 0].long()])


def test_offsets_beyond_32_bits():
    """Weights, token rows, results and tables of more than 2^32 bytes; what lies at their ends is checked."""
    g = torch.Generator(device=DEV).manual_seed(1)

    def normal(*shape):
        return torch.empty(shape, dtype=BF, device=DEV).normal_(generator=g)

    E, n, m, T = 9, 8192, 32768, 40                       # W: 4.8e9 bytes
    w = normal(E, n, m)
    experts = torch.full((T, 1), E - 1, dtype=torch.int32, device=DEV)
    plan = P.expert_rows(experts, E)
    x, last = normal(T, n), w[E - 1].cpu().double()
    want, size = x.cpu().double() @ last, x.cpu().double().abs() @ last.abs()
    near(P.expert_matmul(x, w, plan, gather=True), want, bound(n, size, want, BF), "forward")
    d = normal(T, m)
    want, size = d.cpu().double() @ last.T, d.cpu().double().abs() @ last.T.abs()
    near(P.expert_matmul(d, w, plan, gather=True, transpose=True), want, bound(m, size, want, BF), "backward")
    dw = P.expert_matmul_grad(x, d, plan, gather=True, out=w)
    want = x.cpu().double().T @ d.cpu().double()
    near(dw[E - 1], want, bound(T, x.cpu().double().abs().T @ d.cpu().double().abs(), want, BF), "weights")
    assert not dw[:E - 1].any()
    del w, dw

    T, n, m, tail = 70000, 32768, 24, slice(69992, 70000)   # rows: 4.6e9 bytes
    x, w = normal(T, n), normal(2, n, m)
    experts = (torch.arange(T, device=DEV) >= T // 2).int()[:, None]
    plan = P.expert_rows(experts, 2)
    want, size = (x[tail].cpu().double() @ w[1].cpu().double(), x[tail].cpu().double().abs() @ w[1].cpu().double().abs())
    for gather in (True, False):   # the order is the tokens' own here
        near(P.expert_matmul(x, w, plan, gather=gather)[tail], want, bound(n, size, want, BF), gather)
    d = normal(T, m)
    y = P.expert_matmul(d, w, plan, transpose=True)          # the result: 4.6e9 bytes
    want = d[tail].cpu().double() @ w[1].cpu().double().T
    near(y[tail], want, bound(m, d[tail].cpu().double().abs() @ w[1].cpu().double().T.abs(), want, BF), "rows")
    zero = torch.zeros_like(d)
    zero[tail] = d[tail]
    got = P.expert_matmul_grad(x, zero, plan)
    want = x[tail].cpu().double().T @ d[tail].cpu().double()
    near(got[1], want, bound(8, x[tail].cpu().double().abs().T @ d[tail].cpu().double().abs(), want, BF), "weights")
    out = P.expert_combine(y, plan)
    assert torch.equal(out[tail], y[tail])
    del y, out, got, zero

    ids = torch.tensor([69999, 5, 69999, -1, 69998], device=DEV)
    assert torch.equal(P.embed(ids, x)[[0, 1, 2, 4]], x[ids[[0, 1, 2, 4]]])
    dout = normal(5, n)
    dt = P.embed_grad(ids, dout, T, out=x)
    assert torch.equal(dt[69998], dout[4]) and torch.equal(dt[5], dout[1])
    assert torch.equal(dt[69999], (dout[0].float() + dout[2].float()).to(BF))
    assert int(dt.any(1).sum()) == 3


def test_example_learns():
    """The example's loss falls from near log(512) = 6.24 towards the chain's entropy (about 2)."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_moe
    first, last = train_moe.train(steps=60, log=lambda s: print(s, flush=True))
    assert last < first - 1.0, (first, last)
