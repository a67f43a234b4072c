"""ctypes binding of ``include/skew_loss.h``: the head's softmax cross entropy and its gradients, without the logits.

The manner is that of ``moe.py``: argument checks, output allocation and marshalling only, no fallback, and inputs
that require a gradient are refused (the backward pass is a call of its own)::

    loss, lse = head_loss(x, w, targets)                 # (T), (T)
    dx, dw = head_loss_backward(x, w, targets, lse, dloss)
"""
from __future__ import annotations

import ctypes

from .moe import (MAX_COLS, TRANSPOSE, _check, _dense, _dtype_code, _ld, _no_autograd, _on, _ptr, _scratch, _tensor)
from .skewadam import lib

MAX_TOKENS, MAX_WIDTH = 4194304, 1048576

# names that include/skew_loss.h declares (checked by the CPU test suite)
EXPORTS = ("skew_head_loss_bytes", "skew_head_loss_backward_bytes", "skew_head_loss", "skew_head_loss_backward")


class HeadDesc(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w", ctypes.c_void_p), ("targets", ctypes.c_void_p), ("tokens", ctypes.c_int64),
                ("d", ctypes.c_int64), ("vocab", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("target_bytes", ctypes.c_int32), ("flags", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


_READY = None


def _lib():
    global _READY
    L = lib()
    if _READY is not L:
        p, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        for name, args in (
                ("skew_head_loss_bytes", [p, p]),
                ("skew_head_loss_backward_bytes", [p, p]),
                ("skew_head_loss", [p, p, p, p, size, p]),
                ("skew_head_loss_backward", [p, p, p, p, p, i32, i64, p, i64, p, size, p])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _READY = L
    return L


def _head(x, w, targets, tied, scale):
    """(descriptor, shape of w) after the checks of the inputs."""
    import torch
    _tensor(x, "x", (torch.bfloat16,), 2)
    _tensor(w, "w", (torch.bfloat16,), 2, x.device)
    _tensor(targets, "targets", (torch.int32, torch.int64), 1, x.device)
    T, d = x.shape
    _dense(targets, "targets", (T,))
    rows, cols = w.shape
    V = rows if tied else cols
    if (cols if tied else rows) != d:
        raise ValueError(f"w must be {('V', d) if tied else (d, 'V')}, not {(rows, cols)}")
    if T > MAX_TOKENS or not 1 <= d <= MAX_WIDTH or not 1 <= V <= MAX_COLS:
        raise ValueError(f"{T} tokens of width {d} and {V} words are not supported (at most {MAX_TOKENS}, 1 to {MAX_WIDTH} and "
                         f"1 to {MAX_COLS})")
    if not 1e-30 <= scale <= 1e30:
        raise ValueError("scale must lie between 1e-30 and 1e30")
    return HeadDesc(_ptr(x), _ptr(w), _ptr(targets), T, d, V, _ld(x, "x"), _ld(w, "w"), 8 if targets.dtype == torch.int64 else 4,
                    TRANSPOSE if tied else 0, scale, 0)


def _rows(t, what, T, device):
    import torch
    _tensor(t, what, (torch.float32,), 1, device)
    _dense(t, what, (T,))


def _apart(out, t, what):
    """Refuses an output that shares memory with an input, which is read after parts of the output are written. (Columns of the same
    rows, side by side, do not.)"""
    if out.untyped_storage().data_ptr() != t.untyped_storage().data_ptr() or not out.numel() or not t.numel():
        return
    (a, la), (b, lb) = ((v.data_ptr(), v.element_size() * _ld(v, name)) for v, name in ((out, "out"), (t, what)))
    ends = [p + (v.shape[0] - 1) * ld + v.shape[1] * v.element_size() for v, p, ld in ((out, a, la), (t, b, lb))]
    if ends[0] <= b or ends[1] <= a:
        return
    row_a, row_b = (v.shape[1] * v.element_size() for v in (out, t))
    if la == lb and row_a <= (b - a) % la <= la - row_b:
        return
    raise ValueError(f"out shares memory with {what}")


def head_loss(x, w, targets, *, tied=False, scale=1.0, stream=None):
    """Softmax cross entropy of ``targets`` (int32 or int64 (T)) under the logits ``scale`` x w: (loss, lse), float32 (T).

    ``x`` bf16 (T, d); ``w`` bf16 (d, V), or with ``tied`` the embedding's table (V, d). lse is the logits' log-sum-exp, loss = lse
    less the target's logit. A target outside [0, V) is no token: both are 0, and its row of x may hold anything. The
    logits are never held: the scratch is 1/32 to 1/16 of their bf16 bytes, of at most 16384 tokens; where rows do not begin at 16-byte
    positions, or d or V is no multiple of 8, also copies of these tokens' rows and of w (512 MiB of it at most).
    """
    import torch
    _no_autograd(x, w)
    h = _head(x, w, targets, tied, scale)
    L, dev = _lib(), x.device
    s, here = _on(dev, stream, x, w, targets)
    with here:
        out = torch.empty((2, h.tokens), dtype=torch.float32, device=dev)
        nbytes = ctypes.c_size_t()
        _check(L.skew_head_loss_bytes(ctypes.byref(h), ctypes.byref(nbytes)), "skew_head_loss_bytes")
        ws = _scratch(nbytes.value, dev)
        loss, lse = out
        _check(L.skew_head_loss(ctypes.byref(h), _ptr(loss), _ptr(lse), _ptr(ws), nbytes.value, s), "skew_head_loss")
    return loss, lse


def head_loss_backward(x, w, targets, lse, dloss, *, dlse=None, tied=False, scale=1.0, dtype=None, out=None, stream=None):
    """Gradients of `head_loss`: (dx (T, d) in bf16 or ``dtype``, dw bf16 in w's shape) from those of loss and (``dlse``) of lse,
    float32 (T), and the lse that it gave. A target outside [0, V) gives a row of zeros in dx and nothing to dw. ``out`` takes an existing
    tensor for dw, such as the gradient that an optimizer was given; it shares no memory with x or w.

    The logits are computed again, in pieces of the vocabulary whose gradient G is held, rounded: up to 512 tokens (or 2^29 of T d V) to twice
    16 bits, which leaves out 2^-16 of an entry, else to float16 (2^-11) beside powers of two of its rows and of the columns of x and w, in
    which entries below 2^-27 of a token's factor can lose bits and those below 2^-38 be 0. Words that are so rare for all tokens are
    computed again with powers of two of their own. include/skew_loss.h has the limits, and what the scratch holds: a piece of G is 512 MiB at
    most, or 256 words where that is more; with 16-bit copies of the piece's words and of x, 8192 tokens of 50304 words of width 2048 take
    647 MB, 4096 tokens 704."""
    import torch
    _no_autograd(x, w, lse, dloss, dlse, out)
    h = _head(x, w, targets, tied, scale)
    dev, T = x.device, h.tokens
    _rows(lse, "lse", T, dev)
    _rows(dloss, "dloss", T, dev)
    if dlse is not None:
        _rows(dlse, "dlse", T, dev)
    dtype = torch.bfloat16 if dtype is None else dtype
    code, L = _dtype_code(dtype, "dtype"), _lib()
    if out is not None:
        _tensor(out, "out", (torch.bfloat16,), 2, dev)
        if out.shape != w.shape:
            raise ValueError(f"out must have shape {tuple(w.shape)}, not {tuple(out.shape)}")
        for t, what in ((x, "x"), (w, "w")):
            _apart(out, t, what)
    s, here = _on(dev, stream, x, w, targets, lse, dloss, dlse, out)
    with here:
        dx = torch.empty((T, h.d), dtype=dtype, device=dev)
        if out is None:
            out = torch.empty(tuple(w.shape), dtype=torch.bfloat16, device=dev)
        ld = _ld(out, "out")
        nbytes = ctypes.c_size_t()
        _check(L.skew_head_loss_backward_bytes(ctypes.byref(h), ctypes.byref(nbytes)), "skew_head_loss_backward_bytes")
        ws = _scratch(nbytes.value, dev)
        _check(L.skew_head_loss_backward(ctypes.byref(h), _ptr(lse), _ptr(dloss), _ptr(dlse), _ptr(dx), code, h.d, _ptr(out), ld,
                                         _ptr(ws), nbytes.value, s), "skew_head_loss_backward")
    return dx, out
