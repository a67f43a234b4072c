"""CPU checks of the head's loss ABI: exports, argument checks (they come before any launch), scratch sizes."""
import ctypes
import os
import re

import pytest

from paper_2607_19058_amd import loss
from paper_2607_19058_amd.skewadam import LIB_PATH, SKEW_EINVAL, SKEW_ENOSPACE, SKEW_OK

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 4096   # an address that no call may touch


def test_library_exports_every_declared_function():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "skew_loss.h")).read(), flags=re.S)
    names = re.findall(r"^int\s+(skew_\w+)\s*\(", src, flags=re.M)
    assert sorted(names) == sorted(loss.EXPORTS)
    L = ctypes.CDLL(LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
    for name, value in (("SKEW_MAX_LOSS_TOKENS", loss.MAX_TOKENS), ("SKEW_MAX_HEAD_WIDTH", loss.MAX_WIDTH)):
        assert re.search(rf"#define {name} {value}\b", src)


def head(**kw):
    f = dict(x=A, w=A, targets=A, tokens=4, d=40, vocab=100, ldx=40, ldw=100, target_bytes=8, flags=0, scale=1.0)
    f.update(kw)
    return loss.HeadDesc(**f)


def sizes(h):
    L, a, b = loss._lib(), ctypes.c_size_t(), ctypes.c_size_t()
    rc = L.skew_head_loss_bytes(ctypes.byref(h), ctypes.byref(a)), L.skew_head_loss_backward_bytes(ctypes.byref(h), ctypes.byref(b))
    return rc, a.value, b.value


def forward(h, out=A, lse=A, ws=A, nbytes=1 << 50):
    return loss._lib().skew_head_loss(ctypes.byref(h), out, lse, ws, nbytes, None)


def backward(h, lse=A, dloss=A, dlse=None, dx=A, dtype=0, lddx=40, dw=A, lddw=100, ws=A, nbytes=1 << 50):
    return loss._lib().skew_head_loss_backward(ctypes.byref(h), lse, dloss, dlse, dx, dtype, lddx, dw, lddw, ws, nbytes, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=(1 << 22) + 1), dict(d=0), dict(d=(1 << 20) + 1, ldx=1 << 21), dict(vocab=0),
                                 dict(vocab=(1 << 24) + 1, ldw=1 << 25), dict(ldx=39), dict(ldw=99), dict(flags=2, ldw=40), dict(flags=2),
                                 dict(flags=1), dict(flags=4), dict(target_bytes=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
                                 dict(scale=INF), dict(scale=1e-31), dict(ldx=1 << 58), dict(ldw=1 << 55)], ids=str)
def test_refuses(bad):
    h = head(**bad)
    if bad == dict(flags=2):   # w's rows of 40 may be 100 apart
        assert sizes(h)[0] == (SKEW_OK, SKEW_OK)
        return
    if bad == dict(flags=2, ldw=40):
        assert sizes(h)[0] == (SKEW_OK, SKEW_OK) and backward(h, lddw=39) == SKEW_EINVAL
        return
    assert sizes(h)[0] == (SKEW_EINVAL, SKEW_EINVAL)
    assert forward(h) == SKEW_EINVAL and backward(h) == SKEW_EINVAL


def test_null_pointers_and_small_workspaces():
    h = head()
    (rc, need, back) = sizes(h)
    assert rc == (SKEW_OK, SKEW_OK) and need > 0 and back > need
    for kw in (dict(x=None), dict(w=None), dict(targets=None)):
        assert forward(head(**kw)) == backward(head(**kw)) == SKEW_EINVAL
    for kw in (dict(out=None), dict(lse=None), dict(ws=None)):
        assert forward(h, **kw) == SKEW_EINVAL
    for kw in (dict(lse=None), dict(dloss=None), dict(dx=None), dict(dw=None), dict(ws=None), dict(dtype=2), dict(lddx=39), dict(lddw=99)):
        assert backward(h, **kw) == SKEW_EINVAL
    assert forward(h, nbytes=need - 1) == SKEW_ENOSPACE and backward(h, nbytes=back - 1) == SKEW_ENOSPACE
    L = loss._lib()
    assert L.skew_head_loss_bytes(None, None) == L.skew_head_loss_bytes(ctypes.byref(h), None) == SKEW_EINVAL
    assert L.skew_head_loss_backward_bytes(None, None) == L.skew_head_loss_backward_bytes(ctypes.byref(h), None) == SKEW_EINVAL
    none = head(tokens=0, x=None, targets=None)
    assert sizes(none) == ((SKEW_OK, SKEW_OK), 0, 0) and forward(none, out=None, lse=None, ws=None, nbytes=0) == SKEW_OK


@pytest.mark.parametrize("flags", [0, 2])
def test_scratch_does_not_hold_the_logits(flags):
    """65536 tokens and 50304 words: 6.6 GB of logits in bf16."""
    def of(T, d=2048, V=50304):
        rc, a, b = sizes(head(tokens=T, d=d, vocab=V, ldx=d, ldw=d if flags else V, flags=flags))
        assert rc == (SKEW_OK, SKEW_OK)
        return a, b
    a, b = of(65536)
    rows = 65536 * 2048
    assert a < 60e6 and b < (512 << 20) * 2 + 2 * rows + 4 * rows + 4 * 65536 * 16 + 1e8
    assert of(16384)[0] >= of(8192)[0]
    assert of(1 << 22)[0] == of(32768)[0]    # runs of 16384
    for T, d, V in ((1, 1, 1), (4194304, 8, 300), (1, 1048576, 3), (3, 8, 1 << 24), (16385, 7, 1000)):
        a, b = of(T, d, V)
        assert 0 < a and 0 < b < 1 << 42
