"""CPU checks of the float32 forms of the weighted sum's and the weights' gradient: refusals (before any launch) and scratch."""
import ctypes

import pytest

from paper_2607_19058_amd import moe
from paper_2607_19058_amd.skewadam import SKEW_EINVAL, SKEW_ENOSPACE, SKEW_OK
from test_moe_cpu import A, BAD_PRODUCT, BAD_ROWS, _product, _rows

IDS = dict(ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))


@pytest.mark.parametrize("bad", BAD_ROWS + BAD_PRODUCT + [dict(flags=2), dict(scale=A), dict(tokens=1 << 30, k=1)], **IDS)
def test_grad_of_float32_rows_refuses(bad):
    L, b = moe._lib(), ctypes.c_size_t()
    r = _rows(**{k: v for k, v in bad.items() if k in dict(moe.RowsDesc._fields_)})
    p = _product(**{k: v for k, v in bad.items() if k in dict(moe.ProductDesc._fields_)})
    assert L.skew_expert_matmul_grad_f32(ctypes.byref(r), ctypes.byref(p), A, 1 << 60, None) == SKEW_EINVAL
    if not set(bad) & {"x", "w", "y"}:   # (the size needs no buffers)
        assert L.skew_expert_matmul_grad_f32_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_EINVAL


def test_grad_of_float32_rows_scratch():
    L, b, r = moe._lib(), ctypes.c_size_t(), _rows()
    for m in (24, 25):
        p = _product(m=m, ldw=m, slice=16 * m, ldy=m)
        assert L.skew_expert_matmul_grad_f32_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_OK
        assert b.value >= 9 * 4 + 16 * 4 + 16 * m * 2   # offsets, rows, two bf16 rows a pair
        assert L.skew_expert_matmul_grad_f32(ctypes.byref(r), ctypes.byref(p), A, b.value - 1, None) == SKEW_ENOSPACE
        assert L.skew_expert_matmul_grad_f32(ctypes.byref(r), ctypes.byref(p), None, b.value, None) == SKEW_EINVAL
    assert L.skew_expert_matmul_grad_f32_bytes(ctypes.byref(r), ctypes.byref(p), None) == SKEW_EINVAL
    assert L.skew_expert_matmul_grad_f32_bytes(ctypes.byref(_rows(tokens=0)), ctypes.byref(p), ctypes.byref(b)) == SKEW_OK
    assert b.value == 0


@pytest.mark.parametrize("bad", BAD_ROWS, **IDS)
def test_combine_backward_to_float32_refuses(bad):
    L, r = moe._lib(), _rows(**bad)
    call = L.skew_expert_combine_backward_f32
    assert call(ctypes.byref(r), A, 16, A, 0, 16, None, A, 16, A, 16, None) == SKEW_EINVAL
    for k in range(4):   # dout, y, dy, dweights
        ptr = [A] * 4
        ptr[k] = None
        assert call(ctypes.byref(_rows()), ptr[0], 16, ptr[1], 0, 16, None, ptr[2], 16, ptr[3], 16, None) == SKEW_EINVAL
    assert call(ctypes.byref(_rows()), A, 16, A, 0, 16, None, A, 15, A, 16, None) == SKEW_EINVAL
    assert call(ctypes.byref(_rows(tokens=0)), None, 16, None, 0, 16, None, None, 16, None, 16, None) == SKEW_OK
