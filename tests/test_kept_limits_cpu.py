"""Rows kept in 8 bits at the largest sizes: a work-group takes 128 blocks of 32, and a launch has fewer than 2^32 threads, so there are at most
2^31 - 128 blocks. What is beyond is refused before any launch."""
import ctypes

import pytest

from paper_2607_19058_amd import kept
from paper_2607_19058_amd.skewadam import SKEW_EINVAL, SKEW_OK
from test_kept_cpu import A, _act

MOST = 2**31 - 128
BEYOND = [(MOST + 1, 32), (2**31 - 1, 1), ((MOST + 3) // 3 + 1, 96)]


@pytest.mark.parametrize("rows, cols", BEYOND, ids=str)
def test_refused(rows, cols):
    L = kept._lib()
    assert L.skew_keep8(A, 0, rows, cols, cols, A, A, None) == SKEW_EINVAL
    assert L.skew_restore8(A, A, rows, cols, A, 0, cols, None) == SKEW_EINVAL
    ld = dict.fromkeys(("ldg", "ldu", "ldda", "lda", "lddg", "lddu"), cols)
    d = _act(rows=rows, cols=cols, **ld)
    assert L.skew_expert_act(ctypes.byref(d), None) == SKEW_EINVAL
    assert L.skew_expert_act_backward(ctypes.byref(d), None) == SKEW_EINVAL
    with pytest.raises(ValueError):
        kept._size(rows, cols)


@pytest.mark.parametrize("rows, cols", [(MOST, 32), (MOST, 1), (MOST // 3, 96), (0, 1 << 24), (4095, 1 << 24)], ids=str)
def test_sizes_that_are_taken(rows, cols):
    assert kept._size(rows, cols) == -(-cols // 32)


def test_weights_gradient_of_kept_rows():
    """The size query says what the call takes."""
    from paper_2607_19058_amd import moe
    L, n = kept._lib(), ctypes.c_size_t()
    for places, n_cols, want in ((2**31 - 1, 8, SKEW_EINVAL), (MOST, 8, SKEW_OK)):
        r = moe.RowsDesc(A, A, A, places, 1, 2)
        p = moe.ProductDesc(None, A, A, None, n_cols, 8, 0, 8, 8 * n_cols, 8, 0, moe.BF16)
        assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(n)) == want
