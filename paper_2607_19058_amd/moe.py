"""ctypes binding of ``include/skew_moe.h``: routing, the experts' products, the token embedding.

Argument checks, output allocation and marshalling only; the work runs in the HIP library
``libskewadam.so``. Outputs (and the scratch of a call) are allocated with torch on the
stream of the call. There is no fallback: without the built library every call raises.
The backward passes are calls of their own and autograd does not follow them, so inputs that require a gradient are refused:
call under ``torch.no_grad()``, or detach them.

A layer of experts, forward and backward::

    weights, experts = route(logits, k)                          # (T, k)
    plan = expert_rows(experts, n_experts)                       # places in expert order
    h = expert_matmul(x, w_up, plan, gather=True)                # (T k, f)
    a = act(h)
    y = expert_matmul(a, w_down, plan, dtype=torch.float32)      # (T k, d)
    out = expert_combine(y, plan, weights, dtype=torch.bfloat16) # (T, d)

    dy, dweights = expert_combine_backward(dout, y, plan, weights)   # dy float32: dw_down is rounded once
    da = expert_matmul(dout, w_down, plan, gather=True, transpose=True, scale=weights)
    dw_down = expert_matmul_grad(a, dy, plan)
    ...                                                          # dh = act'(h) da
    dx = expert_combine(expert_matmul(dh, w_up, plan, transpose=True, dtype=torch.float32), plan,
                        dtype=torch.bfloat16)
    dw_up = expert_matmul_grad(x, dh, plan, gather=True)
    dlogits = route_backward(logits, experts, dweights)
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
from typing import NamedTuple

from .skewadam import SKEW_OK, SkewError, lib

BF16, F32 = 0, 1
SCORES = {"softmax": 0, "sigmoid": 1}
GATHER, TRANSPOSE = 1, 2
MAX_EXPERTS, MAX_CHOICES, MAX_GROUPS = 1024, 16, 64
MAX_PLACES, MAX_COLS = 2**31 - 1, 1 << 24

# names that include/skew_moe.h declares (checked by the CPU test suite)
EXPORTS = ("skew_route", "skew_route_backward", "skew_order_bytes", "skew_expert_rows", "skew_expert_matmul_bytes",
           "skew_expert_matmul", "skew_expert_matmul_grad", "skew_expert_matmul_grad_f32_bytes",
           "skew_expert_matmul_grad_f32", "skew_expert_combine", "skew_expert_combine_backward",
           "skew_expert_combine_backward_f32", "skew_embed", "skew_embed_grad")


class RouteDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("ld", ctypes.c_int64), ("experts", ctypes.c_int32), ("k", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("score", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("top_groups", ctypes.c_int32), ("group_sum", ctypes.c_int32), ("renormalize", ctypes.c_int32),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class RowsDesc(ctypes.Structure):
    _fields_ = [("offsets", ctypes.c_void_p), ("rows", ctypes.c_void_p), ("slots", ctypes.c_void_p),
                ("tokens", ctypes.c_int64), ("k", ctypes.c_int32), ("experts", ctypes.c_int32)]


class ProductDesc(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w", ctypes.c_void_p), ("y", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("m", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("slice", ctypes.c_int64), ("ldy", ctypes.c_int64), ("flags", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32)]


class ExpertRows(NamedTuple):
    """The (token, choice) pairs in expert order (see skew_expert_rows): what the products take.

    ``offsets`` int32 (E + 1): expert e holds places offsets[e] .. offsets[e + 1);
    ``rows`` int32 (T k): the pair t k + j at each place, -1 past the last expert's;
    ``slots`` int32 (T, k): the place of each pair, -1 where it has no expert.
    """
    offsets: "torch.Tensor"   # noqa: F821
    rows: "torch.Tensor"      # noqa: F821
    slots: "torch.Tensor"     # noqa: F821


_READY = None


def _lib():
    global _READY
    L = lib()
    if _READY is not L:
        p, i32, i64, f32, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        for name, args in (
                ("skew_route", [p, p, p, p, p, p]),
                ("skew_route_backward", [p, p, p, p, p, p]),
                ("skew_order_bytes", [i64, i64, i64, p]),
                ("skew_expert_rows", [p, i64, i32, p, p, p, p, size, p]),
                ("skew_expert_matmul_bytes", [p, p, p]),
                ("skew_expert_matmul", [p, p, p, size, p]),
                ("skew_expert_matmul_grad", [p, p, p]),
                ("skew_expert_matmul_grad_f32_bytes", [p, p, p]),
                ("skew_expert_matmul_grad_f32", [p, p, p, size, p]),
                ("skew_expert_combine", [p, p, i32, i64, p, p, i32, i64, i64, p]),
                ("skew_expert_combine_backward", [p, p, i64, p, i32, i64, p, p, i64, p, i64, p]),
                ("skew_expert_combine_backward_f32", [p, p, i64, p, i32, i64, p, p, i64, p, i64, p]),
                ("skew_embed", [p, i32, i64, p, i64, i64, i64, p, i64, i32, f32, p]),
                ("skew_embed_grad", [p, i32, i64, p, i64, p, i64, i64, i64, i32, f32, p, size, p])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _READY = L
    return L


# ---- argument checks --------------------------------------------------------------------------
def _dtype_code(t, what):
    import torch
    if t not in (torch.bfloat16, torch.float32):
        raise TypeError(f"{what} must be bfloat16 or float32, not {t}")
    return F32 if t == torch.float32 else BF16


def _no_autograd(*inputs):
    import torch
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                raise RuntimeError("autograd does not follow this call (its backward pass is a call of its own): use "
                                   "torch.no_grad(), or detach inputs that require a gradient")


def _tensor(t, what, dtypes, dims, device=None):
    """Type, device and rank of one tensor argument."""
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d).replace('torch.', '') for d in dtypes)}, not {t.dtype}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise TypeError(f"{what} must live on the HIP device of the other tensors")
    if t.dim() != dims:
        raise ValueError(f"{what} must have {dims} dimensions, not {t.dim()}")


def _ld(t, what):
    """Row stride of a row-major matrix (rows that overlap are refused)."""
    n, m = t.shape[-2:]
    if m > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what} must be row-major (unit column stride)")
    ld = t.stride(-2) if n > 1 else max(m, 1)
    if n > 1 and ld < m:
        raise ValueError(f"{what}: row stride {ld} is smaller than the row length {m} (overlapping rows)")
    return max(ld, 1)


def _dense(t, what, shape):
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")


_HERE = contextlib.nullcontext()


def _on(device, stream, *inputs):
    """(handle, context): the stream of the call, and what makes its device and it the current ones, so that outputs
    and scratch are allocated on it. The memory of inputs is not given away before another stream has used them."""
    import torch
    if stream is None:
        index = device.index
        s = torch._C._cuda_getCurrentRawStream(index)
        return s, (_HERE if index == torch.cuda.current_device() else torch.cuda.device(device))
    handle = getattr(stream, "cuda_stream", stream)
    if handle == torch._C._cuda_getCurrentRawStream(device.index) and device.index == torch.cuda.current_device():
        return handle, _HERE
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream, device=device)
    elif stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
    for t in inputs:
        if t is not None:
            t.record_stream(stream)
    return handle, torch.cuda.stream(stream)


@functools.lru_cache(maxsize=4096)
def _order_bytes(n, keys, cols):
    nbytes = ctypes.c_size_t()
    _check(_lib().skew_order_bytes(n, keys, cols, ctypes.byref(nbytes)), "skew_order_bytes")
    return nbytes.value


def _check(rc, what):
    if rc != SKEW_OK:
        raise SkewError(rc, what)


def _scratch(nbytes, device):
    import torch
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _ptr(t):
    return None if t is None else t.data_ptr() or None


# ---- routing ----------------------------------------------------------------------------------
def _route_desc(logits, k, score, renormalize, scale, groups=1, top_groups=1, group_sum=1):
    import torch
    _tensor(logits, "logits", (torch.bfloat16, torch.float32), 2)
    T, E = logits.shape
    if score not in SCORES:
        raise ValueError(f"score must be one of {sorted(SCORES)}, not {score!r}")
    if not 1 <= E <= MAX_EXPERTS:
        raise ValueError(f"{E} experts: 1 to {MAX_EXPERTS} are supported")
    if not 1 <= k <= min(MAX_CHOICES, E):
        raise ValueError(f"k = {k}: 1 to {min(MAX_CHOICES, E)} experts a token are supported")
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    if T * k > MAX_PLACES:
        raise ValueError("too many tokens: pairs have 32-bit indices")
    return RouteDesc(T, _ld(logits, "logits"), E, k, _dtype_code(logits.dtype, "logits"), SCORES[score], groups,
                     top_groups, group_sum, 1 if renormalize else 0, scale, 0)


def route(logits, k, *, score="softmax", bias=None, groups=1, top_groups=None, group_sum=1, renormalize=True,
          scale=1.0, stream=None):
    """Each token's choice of k experts: (weights float32 (T, k), experts int32 (T, k)).

    ``logits`` (T, E), bf16 or float32. ``score`` "softmax" or "sigmoid"; ``bias`` float32 (E) is added
    to the scores for the choice alone. With ``top_groups < groups`` only the best groups of
    E / groups experts are open (a group's value: the sum of its ``group_sum`` highest). The weights are
    the scores of the chosen, divided by their sum with ``renormalize``, times ``scale``. Ties go to the
    lowest index; a logit of -inf closes its expert, and places left over hold expert -1, weight 0.
    """
    import torch
    _no_autograd(logits, bias)
    top_groups = groups if top_groups is None else top_groups
    d = _route_desc(logits, k, score, renormalize, scale, groups, top_groups, group_sum)
    if not 1 <= groups <= MAX_GROUPS or d.experts % groups:
        raise ValueError(f"groups = {groups} must divide the {d.experts} experts and be at most {MAX_GROUPS}")
    if not 1 <= top_groups <= groups or k > top_groups * (d.experts // groups):
        raise ValueError(f"top_groups = {top_groups} of {groups} groups cannot hold k = {k} experts")
    if group_sum not in (1, 2) or (group_sum == 2 and bias is None):
        raise ValueError("group_sum must be 1, or 2 with a bias")
    if bias is not None:
        _tensor(bias, "bias", (torch.float32,), 1, logits.device)
        _dense(bias, "bias", (d.experts,))
    s, here = _on(logits.device, stream, logits, bias)
    with here:
        weights = torch.empty((d.tokens, k), dtype=torch.float32, device=logits.device)
        experts = torch.empty((d.tokens, k), dtype=torch.int32, device=logits.device)
        _check(_lib().skew_route(ctypes.byref(d), _ptr(logits), _ptr(bias) if bias is not None else None,
                                 _ptr(weights), _ptr(experts), s), "skew_route")
    return weights, experts


def route_backward(logits, experts, dweights, *, score="softmax", renormalize=True, scale=1.0, stream=None):
    """The logits' gradient (T, E) in their type, from that of the weights and the choice of `route`."""
    import torch
    _no_autograd(logits, dweights)
    _tensor(experts, "experts", (torch.int32,), 2, logits.device)
    d = _route_desc(logits, experts.shape[1], score, renormalize, scale)
    _dense(experts, "experts", (d.tokens, d.k))
    _tensor(dweights, "dweights", (torch.float32,), 2, logits.device)
    _dense(dweights, "dweights", (d.tokens, d.k))
    s, here = _on(logits.device, stream, logits, experts, dweights)
    with here:
        dlogits = torch.empty((d.tokens, d.experts), dtype=logits.dtype, device=logits.device)
        _check(_lib().skew_route_backward(ctypes.byref(d), _ptr(logits), _ptr(experts), _ptr(dweights),
                                          _ptr(dlogits), s), "skew_route_backward")
    return dlogits


def expert_rows(experts, n_experts, *, stream=None) -> ExpertRows:
    """The pairs of ``experts`` int32 (T, k) in the order of their experts; entries outside [0, n_experts) are none."""
    import torch
    _tensor(experts, "experts", (torch.int32,), 2)
    _dense(experts, "experts", experts.shape)
    T, k = experts.shape
    if not 1 <= n_experts <= MAX_EXPERTS:
        raise ValueError(f"{n_experts} experts: 1 to {MAX_EXPERTS} are supported")
    if not 1 <= k <= MAX_CHOICES or T * k > MAX_PLACES:
        raise ValueError(f"experts must hold 1 to {MAX_CHOICES} choices a token, of fewer than 2^31 pairs")
    L, n, dev = _lib(), T * k, experts.device
    nbytes = _order_bytes(n, n_experts, 0)
    s, here = _on(dev, stream, experts)
    with here:
        plan = ExpertRows(torch.empty(n_experts + 1, dtype=torch.int32, device=dev),
                          torch.empty(n, dtype=torch.int32, device=dev),
                          torch.empty((T, k), dtype=torch.int32, device=dev))
        ws = _scratch(nbytes, dev)
        _check(L.skew_expert_rows(_ptr(experts), n, n_experts, _ptr(plan.offsets), _ptr(plan.rows), _ptr(plan.slots),
                                  _ptr(ws), nbytes, s), "skew_expert_rows")
    return plan


# ---- the experts' products ----------------------------------------------------------------------
def _plan_desc(plan, device):
    import torch
    for t, what, dims in ((plan.offsets, "plan.offsets", 1), (plan.rows, "plan.rows", 1), (plan.slots, "plan.slots", 2)):
        _tensor(t, what, (torch.int32,), dims, device)
    T, k = plan.slots.shape
    E = plan.offsets.shape[0] - 1
    if not 1 <= k <= MAX_CHOICES or not 1 <= E <= MAX_EXPERTS or T * k > MAX_PLACES:
        raise ValueError("the plan must come from expert_rows()")
    _dense(plan.offsets, "plan.offsets", (E + 1,))
    _dense(plan.rows, "plan.rows", (T * k,))
    _dense(plan.slots, "plan.slots", (T, k))
    return RowsDesc(plan.offsets.data_ptr(), _ptr(plan.rows), _ptr(plan.slots), T, k, E)


def _stack(w, what, E):
    """Row and slice stride of a stacked (E, n, m) tensor."""
    if w.shape[0] != E:
        raise ValueError(f"{what} holds {w.shape[0]} experts, the plan {E}")
    n, m = w.shape[1:]
    if not 1 <= min(n, m) or max(n, m) > MAX_COLS:
        raise ValueError(f"{what}: {n} x {m} is not supported")
    ld = _ld(w, what)
    step = w.stride(0) if E > 1 else n * ld
    if step < n * ld:
        raise ValueError(f"{what}: slice stride {step} is smaller than a slice ({n * ld})")
    return ld, step


def _rows_of(t, what, rows, cols):
    if t.shape != (rows, cols):
        raise ValueError(f"{what} must have shape {(rows, cols)}, not {tuple(t.shape)}")
    return _ld(t, what)


def expert_matmul(x, w, plan, *, gather=False, transpose=False, scale=None, dtype=None, stream=None):
    """Each place's row times its expert's matrix: (T k, m), or (T k, n) with ``transpose``.

    ``x`` bf16: one row a place, or with ``gather`` one a token. ``w`` bf16 (E, n, m); ``transpose``
    multiplies by W[e]^T (the inputs' gradient). ``scale`` float32 (T, k) multiplies each pair's row in float32.
    The result is bf16, or float32 with ``dtype``; rows past the last expert's are zero.
    """
    import torch
    _no_autograd(x, w, scale)
    _tensor(x, "x", (torch.bfloat16,), 2)
    _tensor(w, "w", (torch.bfloat16,), 3, x.device)
    r = _plan_desc(plan, x.device)
    ldw, step = _stack(w, "w", r.experts)
    n, m = w.shape[1:]
    ldx = _rows_of(x, "x", r.tokens if gather else r.tokens * r.k, m if transpose else n)
    if scale is not None:
        _tensor(scale, "scale", (torch.float32,), 2, x.device)
        _dense(scale, "scale", (r.tokens, r.k))
    dtype = torch.bfloat16 if dtype is None else dtype
    code, cols = _dtype_code(dtype, "dtype"), n if transpose else m
    L = _lib()
    s, here = _on(x.device, stream, x, w, scale, *plan)
    with here:
        y = torch.empty((r.tokens * r.k, cols), dtype=dtype, device=x.device)
        p = ProductDesc(_ptr(x), _ptr(w), _ptr(y), _ptr(scale), n, m, ldx, ldw, step, cols,
                        (GATHER if gather else 0) | (TRANSPOSE if transpose else 0), code)
        nbytes = ctypes.c_size_t()
        _check(L.skew_expert_matmul_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(nbytes)),
               "skew_expert_matmul_bytes")
        ws = _scratch(nbytes.value, x.device)
        _check(L.skew_expert_matmul(ctypes.byref(r), ctypes.byref(p), _ptr(ws), nbytes.value, s), "skew_expert_matmul")
    return y


def expert_matmul_grad(x, dy, plan, *, gather=False, out=None, stream=None):
    """The weights' gradient bf16 (E, n, m): each expert's sum of x's rows (one a place, or with ``gather`` one a
    token) times ``dy`` (T k, m), bf16 or float32; zero for an expert without rows. A float32 ``dy`` is taken as
    two bf16 numbers (2^-16 of a value is left out), in up to twice the time. ``out`` takes an existing
    tensor, such as the gradient that an optimizer was given."""
    import torch
    _no_autograd(x, dy, out)
    _tensor(x, "x", (torch.bfloat16,), 2)
    _tensor(dy, "dy", (torch.bfloat16, torch.float32), 2, x.device)
    r = _plan_desc(plan, x.device)
    if dy.dtype == torch.float32 and r.tokens * r.k > MAX_PLACES // 2:
        raise ValueError("too many pairs: a float32 dy is taken as two rows a pair, which have 32-bit indices")
    n, m = x.shape[1], dy.shape[1]
    ldx = _rows_of(x, "x", r.tokens if gather else r.tokens * r.k, n)
    ldy = _rows_of(dy, "dy", r.tokens * r.k, m)
    if out is not None:
        _tensor(out, "out", (torch.bfloat16,), 3, x.device)
        if tuple(out.shape[1:]) != (n, m):
            raise ValueError(f"out must have shape {(r.experts, n, m)}, not {tuple(out.shape)}")
    s, here = _on(x.device, stream, x, dy, out, *plan)
    with here:
        if out is None:
            out = torch.empty((r.experts, n, m), dtype=torch.bfloat16, device=x.device)
        ldw, step = _stack(out, "out", r.experts)
        p = ProductDesc(_ptr(x), _ptr(out), _ptr(dy), None, n, m, ldx, ldw, step, ldy, GATHER if gather else 0, BF16)
        L = _lib()
        if dy.dtype == torch.bfloat16:
            _check(L.skew_expert_matmul_grad(ctypes.byref(r), ctypes.byref(p), s), "skew_expert_matmul_grad")
        else:
            nbytes = ctypes.c_size_t()
            _check(L.skew_expert_matmul_grad_f32_bytes(ctypes.byref(r), ctypes.byref(p), ctypes.byref(nbytes)),
                   "skew_expert_matmul_grad_f32_bytes")
            ws = _scratch(nbytes.value, x.device)
            _check(L.skew_expert_matmul_grad_f32(ctypes.byref(r), ctypes.byref(p), _ptr(ws), nbytes.value, s),
                   "skew_expert_matmul_grad_f32")
    return out


def expert_combine(y, plan, weights=None, *, dtype=None, stream=None):
    """Rows back to tokens: (T, m), each the sum of its pairs' rows of ``y`` times ``weights`` float32 (T, k)
    (None: 1); zero for a token without experts. The result has y's type or ``dtype``."""
    import torch
    _no_autograd(y, weights)
    _tensor(y, "y", (torch.bfloat16, torch.float32), 2)
    r = _plan_desc(plan, y.device)
    m = y.shape[1]
    ldy = _rows_of(y, "y", r.tokens * r.k, m)
    if not 1 <= m <= MAX_COLS:
        raise ValueError(f"rows of {m} columns are not supported")
    if weights is not None:
        _tensor(weights, "weights", (torch.float32,), 2, y.device)
        _dense(weights, "weights", (r.tokens, r.k))
    dtype = y.dtype if dtype is None else dtype
    code = _dtype_code(dtype, "dtype")
    s, here = _on(y.device, stream, y, weights, *plan)
    with here:
        out = torch.empty((r.tokens, m), dtype=dtype, device=y.device)
        _check(_lib().skew_expert_combine(ctypes.byref(r), _ptr(y), _dtype_code(y.dtype, "y"), ldy, _ptr(weights),
                                          _ptr(out), code, m, m, s), "skew_expert_combine")
    return out


def expert_combine_backward(dout, y, plan, weights=None, *, dtype=None, stream=None):
    """Gradients of `expert_combine`: (dy (T k, m), dweights float32 (T, k)) from ``dout`` bf16 (T, m). dy is float32, so
    that a weights' gradient made from it is rounded once; ``dtype`` bf16 gives it half the bytes, and
    `expert_matmul_grad` half the work, for a second rounding (2^-8 of each term at most)."""
    import torch
    dtype = torch.float32 if dtype is None else dtype
    code = _dtype_code(dtype, "dtype")
    _no_autograd(dout, y, weights)
    _tensor(dout, "dout", (torch.bfloat16,), 2)
    _tensor(y, "y", (torch.bfloat16, torch.float32), 2, dout.device)
    r = _plan_desc(plan, dout.device)
    m = dout.shape[1]
    if not 1 <= m <= MAX_COLS:
        raise ValueError(f"rows of {m} columns are not supported")
    ldo, ldy = _rows_of(dout, "dout", r.tokens, m), _rows_of(y, "y", r.tokens * r.k, m)
    if weights is not None:
        _tensor(weights, "weights", (torch.float32,), 2, dout.device)
        _dense(weights, "weights", (r.tokens, r.k))
    s, here = _on(dout.device, stream, dout, y, weights, *plan)
    with here:
        dy = torch.empty((r.tokens * r.k, m), dtype=dtype, device=dout.device)
        dweights = torch.empty((r.tokens, r.k), dtype=torch.float32, device=dout.device)
        name = "skew_expert_combine_backward" + ("_f32" if code == F32 else "")
        _check(getattr(_lib(), name)(ctypes.byref(r), _ptr(dout), ldo, _ptr(y), _dtype_code(y.dtype, "y"), ldy,
                                     _ptr(weights), _ptr(dy), m, _ptr(dweights), m, s), name)
    return dy, dweights


# ---- the token embedding ------------------------------------------------------------------------
def _ids(tokens, device):
    import torch
    _tensor(tokens, "tokens", (torch.int32, torch.int64), 1, device)
    _dense(tokens, "tokens", tokens.shape)
    if tokens.shape[0] > MAX_PLACES:
        raise ValueError("too many tokens: they have 32-bit indices")
    return 8 if tokens.dtype == torch.int64 else 4


def embed(tokens, table, *, scale=1.0, stream=None):
    """``scale`` times the table's rows of ``tokens`` (int32 or int64 (T)): (T, D) in the table's type (bf16,
    float32). An id outside [0, V) is no token: a row of zeros."""
    import torch
    _no_autograd(table)
    _tensor(table, "table", (torch.bfloat16, torch.float32), 2)
    size = _ids(tokens, table.device)
    (V, D), T = table.shape, tokens.shape[0]
    if not 1 <= V <= MAX_PLACES or not 1 <= D <= MAX_COLS:
        raise ValueError(f"a {V} x {D} table is not supported")
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    ld = _ld(table, "table")
    s, here = _on(table.device, stream, tokens, table)
    with here:
        out = torch.empty((T, D), dtype=table.dtype, device=table.device)
        _check(_lib().skew_embed(_ptr(tokens), size, T, _ptr(table), V, D, ld, _ptr(out), D,
                                 _dtype_code(table.dtype, "table"), scale, s), "skew_embed")
    return out


def embed_grad(tokens, dout, vocab, *, scale=1.0, out=None, stream=None):
    """The table's gradient (V, D) in dout's type: ``scale`` times the sum of ``dout``'s rows of each id, zero for
    ids without tokens. ``out`` takes an existing tensor, such as the gradient that an optimizer was given."""
    import torch
    _no_autograd(dout, out)
    _tensor(dout, "dout", (torch.bfloat16, torch.float32), 2)
    size = _ids(tokens, dout.device)
    T, D = dout.shape
    if tokens.shape[0] != T:
        raise ValueError(f"{tokens.shape[0]} tokens, {T} rows of dout")
    if not 1 <= vocab <= MAX_PLACES or not 1 <= D <= MAX_COLS:
        raise ValueError(f"a {vocab} x {D} table is not supported")
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    ldo, L, dev = _ld(dout, "dout"), _lib(), dout.device
    nbytes = _order_bytes(T, vocab, D)
    if out is not None:
        _tensor(out, "out", (dout.dtype,), 2, dev)
    s, here = _on(dev, stream, tokens, dout, out)
    with here:
        if out is None:
            out = torch.empty((vocab, D), dtype=dout.dtype, device=dev)
        ldt = _rows_of(out, "out", vocab, D)
        ws = _scratch(nbytes, dev)
        _check(L.skew_embed_grad(_ptr(tokens), size, T, _ptr(dout), ldo, out.data_ptr(), vocab, D, ldt,
                                 _dtype_code(dout.dtype, "dout"), scale, _ptr(ws), nbytes, s), "skew_embed_grad")
    return out
