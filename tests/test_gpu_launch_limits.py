"""The largest rows kept in 8 bits that are taken: 2^31 - 128 blocks, one value each (the codes are 64 GiB)."""
import pytest
import torch

import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def test_most_blocks():
    R, period = 2**31 - 128, 2**20
    part = torch.randn(period, 1, generator=torch.Generator(device=DEV).manual_seed(0), device=DEV).to(BF)
    x = part.repeat(R // period + 1, 1)[:R]
    kept, want = P.keep8(x), P.keep8(part)
    del x
    for r in (0, 2**30, R - 5000):
        i = torch.arange(r, r + 5000, device=DEV) % period
        assert torch.equal(kept.codes[r:r + 5000], want.codes[i]) and torch.equal(kept.scales[r:r + 5000], want.scales[i])
    values, back = P.restore8(kept), P.restore8(want)
    for r in (0, 2**30, R - 5000):
        assert torch.equal(values[r:r + 5000], back[torch.arange(r, r + 5000, device=DEV) % period])


def test_zeros_of_a_large_head_without_tokens():
    """dw of 2^35 + 2^20 elements, more than one launch fills."""
    d, V = 2**20, 2**15 + 1
    x, w = torch.empty(0, d, dtype=BF, device=DEV), torch.empty(V, d, dtype=BF, device=DEV)
    out = torch.full((V, d), 7.0, dtype=BF, device=DEV)
    none = torch.empty(0, device=DEV)
    dx, dw = P.head_loss_backward(x, w, torch.empty(0, dtype=torch.int64, device=DEV), none, none, tied=True, out=out)
    assert dx.shape == (0, d) and dw is out
    for r in range(0, V, 1024):
        assert not out[r:r + 1024].any(), r
