"""Edges that include/skew_loss.h states: rows that are no token beside weights that are not finite."""
import math

import pytest
import torch

import paper_2607_19058_amd as P
from test_gpu_loss import inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# few tokens (two bf16 numbers, shared contractions), many (float16 operands), two pieces of the vocabulary
NONE = [(3, 33, 17), (40, 64, 300), (300, 130, 777), (2048, 128, 512), (600, 1000, 904), (2100, 1031, 999), (4100, 24, 66010)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", NONE, ids=lambda c: "x".join(map(str, c)))
def test_rows_that_are_no_token_are_zeros_whatever_w_holds(case, tied):
    x, w, targets, dloss, dlse = inputs(*case, tied=tied, none=0.3)
    targets[0] = -1
    there = (targets >= 0) & (targets < case[2])
    words = w if tied else w.T
    words[1, 2], words[case[2] - 1, 0], words[5] = math.nan, math.inf, -math.inf
    loss, lse = P.head_loss(x, w, targets, tied=tied)
    assert not loss[~there].any() and not lse[~there].any() and bool(loss[there].isnan().all())
    for dtype in (BF, F32):
        dx, _ = P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied, dtype=dtype)
        assert not dx[~there].any() and bool(dx[there].isnan().all())
    none = torch.full_like(targets, case[2])
    loss, lse = P.head_loss(x, w, none, tied=tied)
    dx, dw = P.head_loss_backward(x, w, none, lse, dloss, dlse=dlse, tied=tied)
    assert not loss.any() and not lse.any() and not dx.any() and not dw.any()


@pytest.mark.parametrize("tied", [False, True])
def test_outputs_that_share_memory_with_inputs_are_refused(tied):
    T, d, V = 40, 64, 100
    x, w, targets, dloss, _ = inputs(T, d, V, tied=tied, none=0.0)
    _, lse = P.head_loss(x, w, targets, tied=tied)
    _, want = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied)
    n, m = w.shape
    both = torch.zeros(n + 1, 2 * m, dtype=BF, device="cuda")
    flat = torch.zeros(2 * n * m + T * d, dtype=BF, device="cuda")
    wide, rows, shared = both[:n, :m], flat[:n * m].view(n, m), flat[:T * d].view(T, d)
    for v, t in ((wide, w), (rows, w)):
        v.copy_(t)
    for out, xv, wv in ((wide, x, wide), (both[1:, :m], x, wide), (both[:n, 1:m + 1], x, wide), (both[:n, m - 1:2 * m - 1], x, wide), (rows, x, rows),
                        (flat[n * m - 1:2 * n * m - 1].view(n, m), x, rows), (rows, shared, w)):
        with pytest.raises(ValueError, match="shares memory"):
            P.head_loss_backward(xv, wv, targets, lse, dloss, tied=tied, out=out)
    for out, wv in ((both[:n, m:], wide), (flat[n * m:2 * n * m].view(n, m), rows)):   # beside it, and behind it
        _, dw = P.head_loss_backward(x, wv, targets, lse, dloss, tied=tied, out=out)
        assert dw is out and torch.equal(dw, want) and torch.equal(wv, w)
