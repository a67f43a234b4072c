"""The weights' gradient from kept rows on each of its tiles, against float64 on the GPU. Which sizes take which tile is the host's rule, which
tests/test_kept_tiles_cpu.py follows. Tolerance as in test_gpu_kept.py: 4 K + 16 half ulps of float32 of the sum of absolute values, and the
rounding to bf16."""
import pytest
import torch

import paper_2607_19058_amd as P
from kept_ref import U32, UBF

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32

# tile, tokens, experts, choices, n, m: results in whole chunks of 8, and not
CASES = [(2, 500, 9, 2, 320, 136), (2, 500, 9, 2, 333, 131), (1, 2000, 64, 2, 1024, 264), (1, 2000, 64, 2, 1031, 261), (1, 1001, 70, 1, 1000, 513),
         (0, 8192, 16, 2, 2048, 1032), (0, 8192, 16, 2, 2048, 1031), (0, 8200, 16, 2, 2041, 1033), (0, 6144, 32, 2, 2040, 2048),
         (0, 6145, 32, 2, 2033, 2001)]


def plan_of(T, E, k, g):
    """Pairs whose experts have 0, 1, 31, 32, 33, 64, 65 rows, the others the rest; a share of the pairs has none. (An expert may be twice a
    token's, which the products do not mind.)"""
    few = [0, 1, 31, 32, 33, 64, 65][:E - 2]
    rest = torch.arange(len(few), E, device=DEV).repeat(T * k // (E - len(few)) + 1)
    key = torch.cat([torch.full((n,), e, device=DEV) for e, n in enumerate(few)] + [torch.full((T // 20,), -1, device=DEV), rest])[:T * k]
    return P.expert_rows(key[torch.randperm(T * k, generator=g, device=DEV)].view(T, k).int().contiguous(), E)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[1:])) + f"-tile{c[0]}")
def test_tile(case, gather):
    _, T, E, k, n, m = case
    g = torch.Generator(device=DEV).manual_seed(T + n)
    plan = plan_of(T, E, k, g)
    kept = P.keep8(torch.randn(T if gather else T * k, n, generator=g, device=DEV).to(BF))
    dy = torch.randn(T * k, m, generator=g, device=DEV).to(BF)
    out = torch.full((E, n, m + 8), 7.0, dtype=BF, device=DEV)
    got = P.expert_matmul_grad(kept, dy, plan, gather=gather)
    P.expert_matmul_grad(kept, dy, plan, gather=gather, out=out[:, :, :m])
    assert torch.equal(out[:, :, :m], got) and bool((out[:, :, m:] == 7).all())
    x = P.restore8(kept, dtype=F32).double()
    off = plan.offsets.tolist()
    assert off[-1] < T * k and {0, 1, 31, 32, 33} <= set(b - a for a, b in zip(off, off[1:]))
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        a = x[plan.rows[lo:hi].long() // k] if gather else x[lo:hi]
        at, d = a.T.contiguous(), dy[lo:hi].double()
        want, size = at @ d, at.abs() @ d.abs()
        bad = ~((got[e].double() - want).abs() <= UBF * want.abs() + (4 * (hi - lo) + 16) * U32 * size + 1e-38)
        assert not bad.any(), (e, hi - lo, int(bad.sum()))
