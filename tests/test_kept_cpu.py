"""CPU checks of the ABI of rows kept in 8 bits: exports, argument checks (they come before any launch), scratch sizes."""
import ctypes
import os
import re

import pytest
import torch

import kept_ref as ref
from paper_2607_19058_amd import kept, moe
from paper_2607_19058_amd.skewadam import LIB_PATH, SKEW_EINVAL, SKEW_ENOSPACE, SKEW_OK

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 4096   # an address that no call may touch


def test_library_exports_every_declared_function():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "skew_kept.h")).read(), flags=re.S)
    names = re.findall(r"^int\s+(skew_\w+)\s*\(", src, flags=re.M)
    assert sorted(names) == sorted(kept.EXPORTS)
    L = ctypes.CDLL(LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
    for name, value in kept.KINDS.items():
        assert re.search(rf"SKEW_ACT_{name.upper()} = {value}\b", src)
    assert re.search(rf"#define SKEW_KEPT_BLOCK {kept.BLOCK}\b", src)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(rows=-1), dict(cols=0), dict(cols=(1 << 24) + 1, ld=1 << 25), dict(ld=39),
                                 dict(x=None), dict(codes=None), dict(scales=None), dict(codes=A + 8),
                                 dict(rows=1 << 30), dict(rows=1 << 25, ld=1 << 36)], ids=str)
def test_keep_and_restore_refuse(bad):
    L, f = kept._lib(), dict(x=A, dtype=0, rows=4, cols=40, ld=40, codes=A, scales=A, **{})
    f.update(bad)
    assert L.skew_keep8(f["x"], f["dtype"], f["rows"], f["cols"], f["ld"], f["codes"], f["scales"], None) == SKEW_EINVAL
    assert L.skew_restore8(f["codes"], f["scales"], f["rows"], f["cols"], f["x"], f["dtype"], f["ld"], None) == SKEW_EINVAL


def test_calls_without_rows():
    L = kept._lib()
    assert L.skew_keep8(None, 0, 0, 40, 40, None, None, None) == SKEW_OK
    assert L.skew_restore8(None, None, 0, 40, None, 1, 40, None) == SKEW_OK
    d = _act(rows=0, g=None, a=None, da=None, dg=None, du=None, codes_u=None, scales_u=None)
    assert L.skew_expert_act(ctypes.byref(d), None) == SKEW_OK
    assert L.skew_expert_act_backward(ctypes.byref(d), None) == SKEW_OK


def _act(**kw):
    f = dict(rows=4, cols=40, g=A, u=A, da=A, a=A, dg=A, du=A, ldg=40, ldu=40, ldda=40, lda=40, lddg=40, lddu=40, codes_g=A,
             codes_u=A, scales_g=A, scales_u=A, kind=1, in_dtype=0, out_dtype=1)
    f.update(kw)
    return kept.ActDesc(**f)


BOTH = [dict(rows=-1), dict(cols=0), dict(kind=3), dict(kind=-1), dict(in_dtype=2), dict(out_dtype=-1), dict(lda=39), dict(codes_g=None),
        dict(scales_g=None), dict(scales_u=None), dict(codes_g=A + 4), dict(codes_u=A + 8), dict(rows=1 << 30)]


@pytest.mark.parametrize("bad", BOTH + [dict(g=None), dict(a=None), dict(ldg=39), dict(ldu=39), dict(u=None),
                                        dict(codes_g=None, scales_g=None)], ids=str)
def test_activation_refuses(bad):
    assert kept._lib().skew_expert_act(ctypes.byref(_act(**bad)), None) == SKEW_EINVAL


@pytest.mark.parametrize("bad", BOTH + [dict(da=None), dict(dg=None), dict(du=None), dict(ldda=39), dict(lddg=39), dict(lddu=39),
                                        dict(codes_g=None, scales_g=None), dict(codes_u=None, scales_u=None)], ids=str)
def test_activation_backward_refuses(bad):
    assert kept._lib().skew_expert_act_backward(ctypes.byref(_act(**bad)), None) == SKEW_EINVAL


def test_null_descriptors():
    L = kept._lib()
    assert L.skew_expert_act(None, None) == L.skew_expert_act_backward(None, None) == SKEW_EINVAL
    assert L.skew_expert_matmul_grad_kept_bytes(None, None, None) == SKEW_EINVAL


def _grad(rows=None, **kw):
    r = dict(offsets=A, rows=A, slots=A, tokens=4, k=2, experts=8)
    r.update(rows or {})
    p = dict(x=None, w=A, y=A, scale=None, n=40, m=24, ldx=0, ldw=24, slice=960, ldy=24, flags=0, out_dtype=0)
    p.update(kw)
    return moe.RowsDesc(**r), moe.ProductDesc(**p)


def test_weights_gradient_scratch():
    L, b = kept._lib(), ctypes.c_size_t()
    for flags, rows in ((0, 8), (1, 4)):
        r, p = _grad(flags=flags)
        assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_OK
        assert b.value >= rows * 64 * 2
        assert L.skew_expert_matmul_grad_kept(ctypes.byref(r), ctypes.byref(p), A, A, A, b.value - 1, None) == SKEW_ENOSPACE
        assert L.skew_expert_matmul_grad_kept(ctypes.byref(r), ctypes.byref(p), A, A, None, b.value, None) == SKEW_EINVAL
        small = b.value
        r, p = _grad(flags=flags, out_dtype=1)
        assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_OK
        assert b.value > small
    # more rows than 2^31 bytes hold
    r, p = _grad(rows=dict(tokens=1 << 22, k=16), n=4096, slice=4096 * 24)
    assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_EINVAL
    r, p = _grad(rows=dict(tokens=1 << 20, k=16), n=4064, slice=4064 * 24)
    assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_OK
    assert b.value >= (1 << 24) * 4064 * 2


@pytest.mark.parametrize("bad", [dict(x=A), dict(n=0), dict(m=0), dict(ldw=23), dict(slice=959), dict(ldy=23), dict(flags=2), dict(scale=A),
                                 dict(out_dtype=2), dict(rows=dict(k=0)), dict(rows=dict(experts=0)), dict(rows=dict(offsets=None)),
                                 dict(rows=dict(tokens=1 << 30, k=1), out_dtype=1, n=1)], ids=str)
def test_weights_gradient_refuses(bad):
    L, b = kept._lib(), ctypes.c_size_t()
    r, p = _grad(**bad)
    assert L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(b)) == SKEW_EINVAL
    assert L.skew_expert_matmul_grad_kept(ctypes.byref(r), ctypes.byref(p), A, A, A, 1 << 40, None) == SKEW_EINVAL


def test_weights_gradient_null_pointers():
    L = kept._lib()
    for kw, codes, scales in ((dict(w=None), A, A), (dict(y=None), A, A), ({}, None, A), ({}, A, None), ({}, A + 1, A)):
        r, p = _grad(**kw)
        assert L.skew_expert_matmul_grad_kept(ctypes.byref(r), ctypes.byref(p), codes, scales, A, 1 << 40, None) == SKEW_EINVAL


def test_the_reference_keeps_within_half_a_step():
    x = torch.randn(50, 70, generator=torch.Generator().manual_seed(0)) * 10
    codes, scales = ref.keep(x)
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :70]
    assert bool(((ref.restore(codes, scales, 70) - x.double()).abs() <= step / 2).all())
