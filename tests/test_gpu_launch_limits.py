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
