"""How often a value is rounded on its way through the operators: against float64 (tests/moe_ref.py)."""
import pytest
import torch

import moe_ref as ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
SPLIT = 2.0**-16   # what two bf16 parts of a float32 leave out, relative: 8 bits each, the first one cut off


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = (got - want).abs() > bound
    assert not bad.any() and not got.isnan().any(), (what, int(bad.sum()), float((got - want).abs().max()))


# T, E, k, n, m: tiles through registers and straight to LDS, one row to more than one list of them, odd widths
CASES = [(1, 2, 1, 8, 8), (3, 4, 2, 33, 17), (40, 3, 2, 128, 200), (420, 8, 2, 1024, 2056), (300, 70, 2, 130, 264),
         (1400, 2, 2, 72, 136), (500, 4, 1, 1031, 2001), (1100, 3, 1, 1200, 1800)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_weights_gradient_of_a_weighted_sum_is_rounded_once(case):
    """From dout (bf16) and the weights (float32) to dW (bf16): the rows in between keep float32's accuracy. A bound
    of one rounding of dW, K products' float32 sum and the two parts' remainder."""
    T, E, k, n, m = case
    g = gen(T + n)
    experts = ref.draw_experts(T, E, k, g)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    x, y = torch.randn(T * k, n, generator=g).to(BF), torch.randn(T * k, m, generator=g).to(BF)
    dout, weights = torch.randn(T, m, generator=g).to(BF), torch.rand(T, k, generator=g)
    dy, _ = P.expert_combine_backward(dout.to(DEV), y.to(DEV), plan, weights.to(DEV))
    got = P.expert_matmul_grad(x.to(DEV), dy, plan)
    held = int(off[-1])
    exact = torch.zeros(T * k, m, dtype=torch.float64)
    pair = row[:held].long()
    exact[:held] = dout.double()[pair // k] * weights.double().reshape(-1)[pair][:, None]
    K = int((off[1:] - off[:-1]).max())
    want, size = (ref.matmul_grad(x, exact, off, row, k, absolute=a) for a in (False, True))
    near(got, want, ref.UBF * want.abs() + (SPLIT + (4 * K + 16) * ref.U32) * size + 1e-38, case)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_weights_gradient_of_float32_rows(case, gather):
    T, E, k, n, m = case
    g = gen(T + m)
    experts = ref.draw_experts(T, E, k, g)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = ref.rows(experts, E)
    K = int((off[1:] - off[:-1]).max())
    x, dy = torch.randn(T if gather else T * k, n, generator=g).to(BF), torch.randn(T * k, m + 5, generator=g)[:, 3:3 + m]
    want, size = (ref.matmul_grad(x, dy, off, row, k, gather, absolute=a) for a in (False, True))
    bound = ref.UBF * want.abs() + (SPLIT + (4 * K + 16) * ref.U32) * size + 1e-38
    wide = torch.full((T * k, m + 5), float("nan"))
    wide[:, 3:3 + m] = dy
    for d in (dy.contiguous().to(DEV), wide.to(DEV)[:, 3:3 + m]):
        got = P.expert_matmul_grad(x.to(DEV), d, plan, gather=gather)
        near(got, want, bound, case)
        assert torch.equal(got, P.expert_matmul_grad(x.to(DEV), d, plan, gather=gather))


def test_float32_rows_keep_their_special_values():
    """The largest and the smallest normal numbers, infinities and NaN: a column of dW each, by one row alone."""
    top, low = torch.finfo(F32).max, 2.0**-120
    values = [top, -top, low, float("inf"), -float("inf"), float("nan"), 0.0, 1 + 2.0**-9]
    plan = P.expert_rows(torch.zeros(1, 1, dtype=torch.int32, device=DEV), 2)
    got = P.expert_matmul_grad(torch.ones(1, 8, dtype=BF, device=DEV), torch.tensor([values], device=DEV), plan).cpu()
    want = torch.tensor(values).to(BF).float()
    assert torch.equal(got[0, :, 5].isnan(), torch.ones(8, dtype=torch.bool)) and not got[1].any()
    for i in (0, 1, 2, 3, 4, 6, 7):
        assert (got[0, :, i].float() == want[i]).all(), i


def test_type_of_the_rows_and_no_tokens():
    experts = torch.zeros(4, 2, dtype=torch.int32, device=DEV)
    experts[:, 1] = 1
    plan = P.expert_rows(experts, 2)
    y, dout = torch.randn(8, 16, device=DEV), torch.randn(4, 16, device=DEV).to(BF)
    w = torch.rand(4, 2, device=DEV)
    wide, dw = P.expert_combine_backward(dout, y, plan, w)
    narrow, dw2 = P.expert_combine_backward(dout, y, plan, w, dtype=BF)
    assert wide.dtype == F32 and narrow.dtype == BF and torch.equal(wide.to(BF), narrow) and torch.equal(dw, dw2)
    with pytest.raises(TypeError):
        P.expert_combine_backward(dout, y, plan, w, dtype=torch.float16)
    none = P.expert_rows(torch.empty(0, 2, dtype=torch.int32, device=DEV), 3)
    x, dy = torch.empty(0, 8, dtype=BF, device=DEV), torch.empty(0, 16, device=DEV)
    assert not P.expert_matmul_grad(x, dy, none, out=torch.ones(3, 8, 16, dtype=BF, device=DEV)).any()
    closed = P.expert_rows(torch.full((5, 2), -1, dtype=torch.int32, device=DEV), 3)
    x, dy = torch.ones(10, 8, dtype=BF, device=DEV), torch.ones(10, 16, device=DEV)
    assert not P.expert_matmul_grad(x, dy, closed, out=torch.ones(3, 8, 16, dtype=BF, device=DEV)).any()


def test_infinite_rows_stay_infinite():
    """An infinity of x times a finite value, or an infinity, is an infinity, whether or not the value is a bf16 number."""
    inf = float("inf")
    x = torch.tensor([[inf, -inf, 1.0, 0.0, 2.0, -1.0, 0.5, 3.0]])
    d = torch.tensor([[1.0, -1.0, 1 + 2.0**-9, -(1 + 2.0**-20), 2.0**-60, inf, -inf, 0.0]])
    plan = P.expert_rows(torch.zeros(1, 1, dtype=torch.int32, device=DEV), 1)
    got = P.expert_matmul_grad(x.to(BF).to(DEV), d.to(DEV), plan).cpu()[0].float()
    want = (x.double().T @ d.double()).to(BF).float()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[~want.isnan()], want[~want.isnan()])
