"""Offsets beyond 2^31 elements and 2^32 bytes: the head's loss with a large vocabulary, rows kept in 8 bits, the activation and the weights'
gradient of many rows. Inputs repeat with a short period where that tells what the far ones have to be."""
import pytest
import torch

import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("tied", [False, True])
def test_head_of_many_words(tied):
    """2.46e9 weights. The vocabulary is one of 600 words 1000 times over: lse is log(1000) more than with 600, and a word's gradient
    that of its first copy where neither is a target."""
    d, few, times, T = 4096, 600, 1000, 40
    g = torch.Generator(device=DEV).manual_seed(0)
    small = (torch.randn(few, d, generator=g, device=DEV) * d**-0.5).to(BF)
    x = torch.randn(T, d, generator=g, device=DEV).to(BF)
    w = small.repeat(times, 1) if tied else small.T.repeat(1, times)
    assert w.numel() > 2**31
    V = few * times
    targets = torch.randint(V - few, V, (T,), generator=g, device=DEV)   # among the last copies
    loss, lse = P.head_loss(x, w, targets, tied=tied)
    z = x.double() @ small.double().T
    want = torch.logsumexp(z, 1) + torch.log(torch.tensor(float(times), dtype=torch.float64))
    # float32 sums of 4096 products of numbers below 5 and 1: below 1e-5; lse of 14 and 60 roundings of it in the sums: 1e-4
    assert float((lse.double() - want).abs().max()) < 1e-4
    mine = z.gather(1, (targets % few)[:, None]).squeeze(1)
    assert float((loss.double() - (want - mine)).abs().max()) < 1e-4
    dloss = torch.rand(T, generator=g, device=DEV) + 0.5
    dx, dw = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied)
    p = torch.exp(z - want[:, None])
    G = p * dloss.double()[:, None]
    wx = times * (G @ small.double()) - dloss.double()[:, None] * small.double()[targets % few]
    assert float((dx.double() - wx).norm() / wx.norm()) < 2.0**-8
    base = G.T.contiguous() @ x.double()
    last = base.index_add(0, targets % few, -dloss.double()[:, None] * x.double())
    rows = dw if tied else dw.T
    for at, want in ((0, base), (V - 2 * few, base), (V - few, last)):
        got = rows[at:at + few].double()
        assert float((got - want).norm() / want.norm()) < 2.0**-8, at


def test_rows_kept_in_8_bits():
    """5e9 values in rows of odd length. Rows repeat every 1000."""
    R, C, period = 70001, 71003, 1000
    g = torch.Generator(device=DEV).manual_seed(1)
    part = torch.randn(period, C, generator=g, device=DEV).to(BF)
    x = part.repeat(R // period + 1, 1)[:R]
    kept, want = P.keep8(x), P.keep8(part)
    back = P.restore8(want)
    for r in range(0, R, 9973):
        n = min(period, R - r)
        i = (torch.arange(r, r + n, device=DEV) % period)
        assert torch.equal(kept.codes[r:r + n], want.codes[i]) and torch.equal(kept.scales[r:r + n], want.scales[i])
    del x
    values = P.restore8(kept)
    for r in (0, 30000, 60000, R - 500):
        i = torch.arange(r, r + 500, device=DEV) % period
        assert torch.equal(values[r:r + 500], back[i])


def test_activation_of_many_values():
    R, C, period = 70001, 65544, 500
    g = torch.Generator(device=DEV).manual_seed(2)
    part = torch.randn(period, C, generator=g, device=DEV).to(BF)
    x = part.repeat(R // period + 1, 1)[:R]
    a, kept = P.expert_act(x, x, keep=True)
    want, few = P.expert_act(part, part, keep=True)
    again, dg, du = P.expert_act_backward(a, kept)
    want2, wg, wu = P.expert_act_backward(want, few)
    for r in (0, 32768, 65535, R - 300):
        i = torch.arange(r, r + 300, device=DEV) % period
        for got, ref in ((a, want), (again, want2), (dg, wg), (du, wu)):
            assert torch.equal(got[r:r + 300], ref[i])


@pytest.mark.parametrize("gather", [False, True])
def test_weights_gradient_of_many_kept_rows(gather):
    """The restored rows pass 2^32 bytes; rows repeat every 2000, half of them to each expert. The first rows' sums alone give the result."""
    T, n, m, E = 600000, 4096, 64, 2
    period = 2000
    g = torch.Generator(device=DEV).manual_seed(3)
    part = torch.randn(period, n, generator=g, device=DEV).to(BF)
    few = P.keep8(part)
    codes, scales = (t.repeat(T // period, 1) for t in (few.codes, few.scales))
    experts = (torch.arange(T, device=DEV) % period >= period // 2).int()[:, None].contiguous()
    plan = P.expert_rows(experts, E)
    dy_part = torch.randn(period, m, generator=g, device=DEV).to(BF)
    pair = plan.rows.long()
    kept = P.Kept8(codes, scales, n) if gather else P.Kept8(codes[pair].contiguous(), scales[pair].contiguous(), n)
    dw = P.expert_matmul_grad(kept, dy_part[pair % period].contiguous(), plan, gather=gather)
    v = P.restore8(few, dtype=F32).double()
    for e in range(E):
        rows = slice(e * (period // 2), (e + 1) * (period // 2))
        want = (v[rows].T.contiguous() @ dy_part[rows].double()) * (T // period)
        # sums of 300000 products in float32: 2 * 300000 half ulps of sums of magnitudes some 500 times the result at most, far less at random
        assert float((dw[e].double() - want).norm() / want.norm()) < 2.0**-7
