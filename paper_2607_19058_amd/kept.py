"""ctypes binding of ``include/skew_kept.h``: rows kept in 8 bits for the backward pass, and the experts' activation.

The manner is that of ``moe.py``: argument checks, output allocation and marshalling only, no fallback, and inputs
that require a gradient are refused (the backward passes are calls of their own).

Gated experts that keep 8 bits of what their backward pass needs::

    g, u = (expert_matmul(x, w, plan, gather=True) for w in (w_gate, w_up))     # (T k, f)
    a, kept = expert_act(g, u, keep=True)          # a for the next product; g, u and a need not be held
    y = expert_matmul(a, w_down, plan, dtype=torch.float32)
    kept_x = keep8(x)

    a, dg, du = expert_act_backward(da, kept)
    dw_down = expert_matmul_grad(a, dy, plan)
    dw_gate, dw_up = (expert_matmul_grad(kept_x, d, plan, gather=True) for d in (dg, du))
"""
from __future__ import annotations

import ctypes

from .moe import (BF16, F32, GATHER, MAX_COLS, MAX_PLACES, Kept8, ProductDesc, _check, _dense, _dtype_code, _ld,
                  _no_autograd, _on, _plan_desc, _ptr, _rows_of, _scratch, _stack, _tensor)
from .skewadam import lib

BLOCK = 32
MAX_BLOCKS = 2**31 - 128
KINDS = {"relu": 0, "silu": 1, "gelu_tanh": 2}

# names that include/skew_kept.h declares (checked by the CPU test suite)
EXPORTS = ("skew_keep8", "skew_restore8", "skew_expert_act", "skew_expert_act_backward",
           "skew_expert_matmul_grad_kept_bytes", "skew_expert_matmul_grad_kept")


class ActDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("g", ctypes.c_void_p), ("u", ctypes.c_void_p),
                ("da", ctypes.c_void_p), ("a", ctypes.c_void_p), ("dg", ctypes.c_void_p), ("du", ctypes.c_void_p),
                ("ldg", ctypes.c_int64), ("ldu", ctypes.c_int64), ("ldda", ctypes.c_int64), ("lda", ctypes.c_int64),
                ("lddg", ctypes.c_int64), ("lddu", ctypes.c_int64), ("codes_g", ctypes.c_void_p),
                ("codes_u", ctypes.c_void_p), ("scales_g", ctypes.c_void_p), ("scales_u", ctypes.c_void_p),
                ("kind", ctypes.c_int32), ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


_READY = None


def _lib():
    global _READY
    L = lib()
    if _READY is not L:
        p, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        for name, args in (
                ("skew_keep8", [p, i32, i64, i64, i64, p, p, p]),
                ("skew_restore8", [p, p, i64, i64, p, i32, i64, p]),
                ("skew_expert_act", [p, p]),
                ("skew_expert_act_backward", [p, p]),
                ("skew_expert_matmul_grad_kept_bytes", [p, p, p]),
                ("skew_expert_matmul_grad_kept", [p, p, p, p, p, size, p])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _READY = L
    return L


def _size(rows, cols):
    """Blocks of a row."""
    blocks = -(-cols // BLOCK)
    if not 1 <= cols <= MAX_COLS or rows * blocks > MAX_BLOCKS:
        raise ValueError(f"{rows} x {cols} values are not supported (rows of 1 to {MAX_COLS}, at most 2^31 - 128 blocks of {BLOCK})")
    return blocks


def _new(rows, blocks, cols, device):
    import torch
    return Kept8(torch.empty((rows, BLOCK * blocks), dtype=torch.int8, device=device),
                 torch.empty((rows, blocks), dtype=torch.uint8, device=device), cols)


def _kept(k, what, device=None):
    """(rows, blocks) of kept rows, after their checks."""
    import torch
    if not isinstance(k, Kept8):
        raise TypeError(f"{what} must be a Kept8, not {type(k).__name__}")
    _tensor(k.codes, f"{what}.codes", (torch.int8,), 2, device)
    _tensor(k.scales, f"{what}.scales", (torch.uint8,), 2, k.codes.device)
    rows, blocks = k.codes.shape[0], _size(k.codes.shape[0], k.cols)
    _dense(k.codes, f"{what}.codes", (rows, BLOCK * blocks))
    _dense(k.scales, f"{what}.scales", (rows, blocks))
    if k.codes.data_ptr() % 16:
        raise ValueError(f"{what}.codes must be 16-byte-aligned")
    return rows, blocks


def keep8(x, *, stream=None) -> Kept8:
    """Rows ``x`` (R, C), bf16 or float32, in 8 bits. A block of 32 neighbours of a row shares the smallest power of two s,
    from 2^-126 on, with 127.5 s >= its largest finite magnitude; a value is rounded to a multiple of s (nearest, ties to
    even, at most 127 of them). An infinity or NaN is kept as NaN."""
    import torch
    _no_autograd(x)
    _tensor(x, "x", (torch.bfloat16, torch.float32), 2)
    R, C = x.shape
    blocks, ld = _size(R, C), _ld(x, "x")
    s, here = _on(x.device, stream, x)
    with here:
        k = _new(R, blocks, C, x.device)
        _check(_lib().skew_keep8(_ptr(x), _dtype_code(x.dtype, "x"), R, C, ld, _ptr(k.codes), _ptr(k.scales), s), "skew_keep8")
    return k


def restore8(kept, *, dtype=None, stream=None):
    """The values that kept rows stand for: (R, C), bf16 (which holds each exactly) or float32."""
    import torch
    R, _ = _kept(kept, "kept")
    dtype = torch.bfloat16 if dtype is None else dtype
    code, dev = _dtype_code(dtype, "dtype"), kept.codes.device
    s, here = _on(dev, stream, kept.codes, kept.scales)
    with here:
        x = torch.empty((R, kept.cols), dtype=dtype, device=dev)
        _check(_lib().skew_restore8(_ptr(kept.codes), _ptr(kept.scales), R, kept.cols, _ptr(x), code, kept.cols, s),
               "skew_restore8")
    return x


def _kind(kind):
    if kind not in KINDS:
        raise ValueError(f"kind must be one of {sorted(KINDS)}, not {kind!r}")
    return KINDS[kind]


def expert_act(g, u=None, *, kind="silu", keep=False, dtype=None, stream=None):
    """The activation between an expert's products: f(``g``) ``u``, or f(g) without u; (R, C) in g's type or ``dtype``.

    ``kind``: "relu", "silu" (g / (1 + exp(-g))) or "gelu_tanh". With ``keep`` the result is (a, kept): kept, a pair of `Kept8` (the second
    one None without u), holds g and u in 8 bits for `expert_act_backward`.
    """
    import torch
    _no_autograd(g, u)
    kind = _kind(kind)
    _tensor(g, "g", (torch.bfloat16, torch.float32), 2)
    R, C = g.shape
    blocks, ldg, ldu = _size(R, C), _ld(g, "g"), 0
    if u is not None:
        _tensor(u, "u", (g.dtype,), 2, g.device)
        ldu = _rows_of(u, "u", R, C)
    dtype = g.dtype if dtype is None else dtype
    code, dev = _dtype_code(dtype, "dtype"), g.device
    s, here = _on(dev, stream, g, u)
    with here:
        a = torch.empty((R, C), dtype=dtype, device=dev)
        kg = _new(R, blocks, C, dev) if keep else None
        ku = _new(R, blocks, C, dev) if keep and u is not None else None
        d = ActDesc(R, C, _ptr(g), _ptr(u), None, _ptr(a), None, None, ldg, ldu, 0, C, 0, 0,
                    _ptr(kg.codes) if kg else None, _ptr(ku.codes) if ku else None,
                    _ptr(kg.scales) if kg else None, _ptr(ku.scales) if ku else None,
                    kind, _dtype_code(g.dtype, "g"), code, 0)
        _check(_lib().skew_expert_act(ctypes.byref(d), s), "skew_expert_act")
    return (a, (kg, ku)) if keep else a


def expert_act_backward(da, kept, *, kind="silu", again=True, dtype=None, stream=None):
    """Gradients of `expert_act` from that of its result and what it kept: (a, dg, du) in da's type or ``dtype``. a is
    the activation of the kept values, which the next product's weights' gradient takes (None with ``again=False``); du is
    None without u. With "relu", whose slope jumps, a g below half a step is kept as 0 and takes no gradient."""
    import torch
    _no_autograd(da)
    kind = _kind(kind)
    _tensor(da, "da", (torch.bfloat16, torch.float32), 2)
    R, C = da.shape
    kg, ku = kept
    for k, what in ((kg, "kept[0]"), (ku, "kept[1]")):
        if k is not None or what == "kept[0]":
            if _kept(k, what, da.device)[0] != R or k.cols != C:
                raise ValueError(f"{what} holds {k.codes.shape[0]} x {k.cols} values, da {R} x {C}")
    _size(R, C)
    ld = _ld(da, "da")
    dtype = da.dtype if dtype is None else dtype
    code, dev = _dtype_code(dtype, "dtype"), da.device
    s, here = _on(dev, stream, da, kg.codes, kg.scales, ku.codes if ku else None, ku.scales if ku else None)
    with here:
        a = torch.empty((R, C), dtype=dtype, device=dev) if again else None
        dg = torch.empty((R, C), dtype=dtype, device=dev)
        du = torch.empty((R, C), dtype=dtype, device=dev) if ku else None
        d = ActDesc(R, C, None, None, _ptr(da), _ptr(a), _ptr(dg), _ptr(du), 0, 0, ld, C, C, C,
                    _ptr(kg.codes), _ptr(ku.codes) if ku else None, _ptr(kg.scales), _ptr(ku.scales) if ku else None,
                    kind, _dtype_code(da.dtype, "da"), code, 0)
        _check(_lib().skew_expert_act_backward(ctypes.byref(d), s), "skew_expert_act_backward")
    return a, dg, du


def _matmul_grad_kept(x, dy, plan, gather, out, stream):
    """`expert_matmul_grad` of kept rows."""
    import torch
    _no_autograd(dy, out)
    _tensor(dy, "dy", (torch.bfloat16, torch.float32), 2)
    rows, _ = _kept(x, "x", dy.device)
    r = _plan_desc(plan, dy.device)
    if dy.dtype == torch.float32 and r.tokens * r.k > MAX_PLACES // 2:
        raise ValueError("too many pairs: a float32 dy is taken as two rows a pair, which have 32-bit indices")
    if rows != (r.tokens if gather else r.tokens * r.k):
        raise ValueError(f"x must hold {r.tokens if gather else r.tokens * r.k} rows, not {rows}")
    n, m, dev = x.cols, dy.shape[1], dy.device
    ldy = _rows_of(dy, "dy", r.tokens * r.k, m)
    if out is not None:
        _tensor(out, "out", (torch.bfloat16,), 3, dev)
        if tuple(out.shape[1:]) != (n, m):
            raise ValueError(f"out must have shape {(r.experts, n, m)}, not {tuple(out.shape)}")
    s, here = _on(dev, stream, x.codes, x.scales, dy, out, *plan)
    with here:
        if out is None:
            out = torch.empty((r.experts, n, m), dtype=torch.bfloat16, device=dev)
        ldw, step = _stack(out, "out", r.experts)
        p = ProductDesc(None, _ptr(out), _ptr(dy), None, n, m, 0, ldw, step, ldy, GATHER if gather else 0,
                        F32 if dy.dtype == torch.float32 else BF16)
        L, nbytes = _lib(), ctypes.c_size_t()
        _check(L.skew_expert_matmul_grad_kept_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(nbytes)),
               "skew_expert_matmul_grad_kept_bytes")
        ws = _scratch(nbytes.value, dev)
        _check(L.skew_expert_matmul_grad_kept(ctypes.byref(r), ctypes.byref(p), _ptr(x.codes), _ptr(x.scales), _ptr(ws),
                                              nbytes.value, s), "skew_expert_matmul_grad_kept")
    return out
