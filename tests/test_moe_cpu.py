"""CPU checks of the mixture-of-experts ABI: exports, argument checks (they come before any launch, so they need no
GPU), scratch sizes, and the binding's own refusals."""
import ctypes
import os
import re

import pytest
import torch

import paper_2607_19058_amd as P
from paper_2607_19058_amd import moe
from paper_2607_19058_amd.skewadam import LIB_PATH, SKEW_EINVAL, SKEW_ENOSPACE, SKEW_OK

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 4096   # an address that no call may touch


def test_library_exports_every_declared_function():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "skew_moe.h")).read(), flags=re.S)
    names = re.findall(r"^int\s+(skew_\w+)\s*\(", src, flags=re.M)
    assert sorted(names) == sorted(moe.EXPORTS)
    L = ctypes.CDLL(LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
    for name, value in (("SKEW_MAX_EXPERTS", moe.MAX_EXPERTS), ("SKEW_MAX_CHOICES", moe.MAX_CHOICES),
                        ("SKEW_MAX_GROUPS", moe.MAX_GROUPS)):
        assert re.search(rf"#define {name} {value}\b", src)


def _route(**kw):
    f = dict(tokens=4, ld=8, experts=8, k=2, dtype=1, score=0, groups=1, top_groups=1, group_sum=1, renormalize=1,
             scale=1.0)
    f.update(kw)
    return moe.RouteDesc(**f)


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(ld=7), dict(experts=0), dict(experts=1025, ld=1025), dict(k=0), dict(k=9),
                                 dict(experts=64, ld=64, k=17), dict(dtype=2), dict(score=2), dict(groups=3), dict(groups=0),
                                 dict(groups=4, top_groups=5), dict(groups=4, top_groups=0), dict(group_sum=3),
                                 dict(groups=8, top_groups=1), dict(experts=1024, ld=1024, groups=128), dict(group_sum=2),
                                 dict(renormalize=2), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(tokens=1 << 31), dict(tokens=1 << 28, ld=1 << 40)],
                         ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_route_refuses(bad):
    L, d = moe._lib(), _route(**bad)
    assert L.skew_route(ctypes.byref(d), A, None, A, A, None) == SKEW_EINVAL
    if not set(bad) & {"groups", "top_groups", "group_sum"}:
        assert L.skew_route_backward(ctypes.byref(d), A, A, A, A, None) == SKEW_EINVAL


def test_null_pointers_and_empty_calls():
    L, d = moe._lib(), _route()
    assert L.skew_route(None, A, None, A, A, None) == SKEW_EINVAL
    for k in range(3):
        ptr = [A, A, A]
        ptr[k] = None
        assert L.skew_route(ctypes.byref(d), ptr[0], None, ptr[1], ptr[2], None) == SKEW_EINVAL
    assert L.skew_route(ctypes.byref(_route(tokens=0)), None, None, None, None, None) == SKEW_OK
    assert L.skew_route_backward(ctypes.byref(_route(tokens=0)), None, None, None, None, None) == SKEW_OK
    assert L.skew_embed(None, 8, 0, None, 5, 4, 4, None, 4, 0, 1.0, None) == SKEW_OK


def test_order_bytes():
    L, b = moe._lib(), ctypes.c_size_t()
    for n, keys, cols in ((0, 1, 0), (1, 8, 0), (16384, 128, 0), (16385, 1024, 0), (8192, 50304, 2048), (1 << 20, 1 << 30, 64)):
        assert L.skew_order_bytes(n, keys, cols, ctypes.byref(b)) == SKEW_OK
        assert 16 * n <= b.value   # two key and two index arrays
    for n, keys, cols in ((-1, 1, 0), (1, 0, 0), (1 << 31, 8, 0), (1, 1 << 31, 0), (1, 8, -1), (1, 8, 1 << 27)):
        assert L.skew_order_bytes(n, keys, cols, ctypes.byref(b)) == SKEW_EINVAL
    assert L.skew_order_bytes(1, 1, 0, None) == SKEW_EINVAL
    assert L.skew_order_bytes(64, 8, 0, ctypes.byref(b)) == SKEW_OK
    assert L.skew_expert_rows(A, 64, 8, A, A, A, A, b.value - 1, None) == SKEW_ENOSPACE
    assert L.skew_expert_rows(A, 64, 8, A, A, A, None, b.value, None) == SKEW_EINVAL
    assert L.skew_expert_rows(A, 64, 1025, A, A, A, A, b.value, None) == SKEW_EINVAL
    assert L.skew_expert_rows(A, 64, 8, None, A, A, A, b.value, None) == SKEW_EINVAL


def _rows(**kw):
    f = dict(offsets=A, rows=A, slots=A, tokens=4, k=2, experts=8)
    f.update(kw)
    return moe.RowsDesc(**f)


def _product(**kw):
    f = dict(x=A, w=A, y=A, scale=None, n=16, m=24, ldx=16, ldw=24, slice=16 * 24, ldy=24, flags=0, out_dtype=0)
    f.update(kw)
    return moe.ProductDesc(**f)


BAD_ROWS = [dict(tokens=-1), dict(k=0), dict(k=17), dict(experts=0), dict(experts=1025), dict(offsets=None), dict(rows=None),
            dict(slots=None), dict(tokens=1 << 31)]
BAD_PRODUCT = [dict(x=None), dict(w=None), dict(y=None), dict(n=0), dict(m=0), dict(n=(1 << 26) + 1), dict(ldx=15), dict(ldw=23),
               dict(slice=16 * 24 - 1), dict(ldy=23), dict(flags=4), dict(slice=1 << 60)]


@pytest.mark.parametrize("bad", BAD_ROWS + BAD_PRODUCT + [dict(flags=2), dict(out_dtype=2)],
                         ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_products_refuse(bad):
    L = moe._lib()
    r = _rows(**{k: v for k, v in bad.items() if k in dict(moe.RowsDesc._fields_)})
    p = _product(**{k: v for k, v in bad.items() if k in dict(moe.ProductDesc._fields_)})
    assert L.skew_expert_matmul(ctypes.byref(r), ctypes.byref(p), A, 1 << 40, None) == SKEW_EINVAL
    if "out_dtype" not in bad:
        assert L.skew_expert_matmul_grad(ctypes.byref(r), ctypes.byref(p), None) == SKEW_EINVAL


def test_grad_takes_no_scale_and_no_transpose():
    L, r = moe._lib(), _rows()
    for bad in (dict(scale=A), dict(flags=3)):
        assert L.skew_expert_matmul_grad(ctypes.byref(r), ctypes.byref(_product(**bad)), None) == SKEW_EINVAL


@pytest.mark.parametrize("bad", BAD_ROWS, ids=lambda b: ",".join(f"{k}={v}" for k, v in b.items()))
def test_combine_refuses(bad):
    L, r = moe._lib(), _rows(**bad)
    assert L.skew_expert_combine(ctypes.byref(r), A, 0, 16, None, A, 0, 16, 16, None) == SKEW_EINVAL
    assert L.skew_expert_combine_backward(ctypes.byref(r), A, 16, A, 0, 16, None, A, 16, A, 16, None) == SKEW_EINVAL


def test_combine_and_embed_refuse_shapes_and_types():
    L, r = moe._lib(), _rows()
    for bad in (dict(t=2), dict(ldy=15), dict(o=2), dict(ldo=15), dict(m=0)):
        f = dict(dict(t=0, ldy=16, o=0, ldo=16, m=16), **bad)
        assert L.skew_expert_combine(ctypes.byref(r), A, f["t"], f["ldy"], None, A, f["o"], f["ldo"], f["m"], None) == SKEW_EINVAL
    for bad in (dict(b=2), dict(n=-1), dict(v=0), dict(d=0), dict(ldt=15), dict(ldo=15), dict(t=2), dict(s=float("nan"))):
        f = dict(dict(b=8, n=4, v=5, d=16, ldt=16, ldo=16, t=0, s=1.0), **bad)
        assert L.skew_embed(A, f["b"], f["n"], A, f["v"], f["d"], f["ldt"], A, f["ldo"], f["t"], f["s"], None) == SKEW_EINVAL
        assert L.skew_embed_grad(A, f["b"], f["n"], A, f["ldo"], A, f["v"], f["d"], f["ldt"], f["t"], f["s"], A, 1 << 40,
                                 None) == SKEW_EINVAL
    assert L.skew_embed_grad(A, 8, 4, A, 16, A, 5, 16, 16, 0, 1.0, A, 8, None) == SKEW_ENOSPACE


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, 8, 8, dtype=torch.bfloat16)
    i = torch.zeros(4, 1, dtype=torch.int32)
    plan = P.ExpertRows(torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), i)
    for call in (lambda: P.route(x, 2), lambda: P.expert_rows(i, 2), lambda: P.expert_matmul(x, w, plan),
                 lambda: P.expert_matmul_grad(x, x, plan), lambda: P.expert_combine(x, plan),
                 lambda: P.embed(i[:, 0], x), lambda: P.embed_grad(i[:, 0], x, 5),
                 lambda: P.route_backward(x, i, torch.zeros(4, 1))):
        with pytest.raises(TypeError, match="HIP device"):
            call()
    with pytest.raises(TypeError, match="bfloat16"):
        P.route(x.half(), 2)
