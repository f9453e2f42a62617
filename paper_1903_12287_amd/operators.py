"""Python binding of include/pbg_operators.h (argument marshalling only).

The operators on a caller's own tensors: grouped matrix products, the preference loss and gradient clipping.  As in
pbg.py every function has the name of its C entry point, checks dtypes, devices, shapes and layouts, passes raw
pointers and raises pbg.PbgError when the call returns an error status.  Contexts come from pbg.pbg_bucket_init.

Nothing is recorded for autograd: gradients are had by calling the _backward functions.  Written tensors count as
modified in place, so that autograd notices where it has saved one of them for a graph of its own.
"""

from __future__ import annotations

import array
import ctypes
import math

import torch
from torch.autograd.graph import increment_version

from . import pbg

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

# every entry point the header declares
EXPORTS = ("pbg_group_linear", "pbg_group_linear_backward", "pbg_preference_loss", "pbg_preference_loss_backward",
           "pbg_clip_gradients")

_ready = None


def library() -> ctypes.CDLL:
    """The library of pbg.py, with the signatures of this header's entry points."""
    global _ready
    if _ready is not None:
        return _ready
    L = pbg.library()
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    f64, dp = ctypes.c_double, ctypes.POINTER(ctypes.c_double)
    sig = {
        "pbg_group_linear": [vp, i32, vp, i64, vp, vp, i32, i64, i32, i32, vp, i64],
        "pbg_group_linear_backward": [vp, i32, vp, i64, vp, vp, i64, vp, i32, i64, i32, i32, vp, i64, vp],
        "pbg_preference_loss": [vp, i32, vp, i64, vp, vp, i32, i64, i32, vp, f32, f32, vp, vp, vp, vp],
        "pbg_preference_loss_backward": [vp, i32, vp, i64, vp, vp, i32, i64, i32, vp, vp, vp, i64],
        "pbg_clip_gradients": [vp, i32, vp, vp, vp, vp, f64, dp],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = i32
    _ready = L
    return L


def _check(ctx, status):
    if status != 0:
        msg = library().pbg_last_error(ctx)
        raise pbg.PbgError(status, msg.decode() if msg else "")


def _type(t, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch.Tensor")
    if t.dtype not in TYPES:
        raise TypeError(f"{what} must be float32, bfloat16 or float16, got {t.dtype}")
    return t.dtype


def _rows(t, dtype, shape, what):
    """Pointer and row stride of a device matrix whose columns are consecutive."""
    n, width = shape
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and t.shape == shape
            and (width <= 1 or t.stride(1) == 1)):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{what} must be a torch.Tensor")
        if t.dtype != dtype:
            raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{what} must be a device tensor")
        if t.shape != shape:
            raise ValueError(f"{what} must be {shape}, got {tuple(t.shape)}")
        raise ValueError(f"{what} must have consecutive columns")
    return (t.data_ptr() if n and width else None), (t.stride(0) if n > 1 else max(width, 1))


def _vector(t, dtype, n, what, allow_none=False):
    if isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and t.is_contiguous() and t.numel() == n:
        return t.data_ptr() if n else None
    if t is not None and isinstance(t, torch.Tensor) and t.numel() != n:
        raise ValueError(f"{what} must hold {n} values, got {t.numel()}")
    return pbg._ptr(t, dtype, what, allow_none=allow_none)


def _here(*tensors):
    """The context's device is the current one, and so must the tensors' be."""
    d = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != d:
            raise ValueError(f"a tensor is on device {t.get_device()}, the current device is {d}")


def _values(tensors, what):
    """Types, numbers of values and pointers of contiguous device tensors of any shapes, as arrays (an attribute at a
    time over all of them: half the time of a loop over tensors; arrays, not ctypes': a quarter of theirs)."""
    T = torch.Tensor
    try:
        types = [TYPES[t.dtype] for t in tensors]
        d = set(map(T.get_device, tensors))   # -1: the host
        if (not d or d == {torch.cuda.current_device()}) and all(map(T.is_contiguous, tensors)):
            return (array.array("i", types), array.array("q", list(map(T.numel, tensors))),
                    array.array("Q", list(map(T.data_ptr, tensors))))
    except (KeyError, AttributeError, TypeError, RuntimeError):   # the last: no device at all
        pass
    for i, t in enumerate(tensors):   # which one, and why
        pbg._ptr(t, _type(t, f"{what}[{i}]"), f"{what}[{i}]")
        _here(t)
    raise TypeError(f"{what} must be tensors")


def _count(n, what):
    """A number that the library takes as 32 bits and would see the low ones alone of.  (Widths need no such check: row
    strides, which bound them, are 64 bits.)"""
    if n > 0x7FFFFFFF:
        raise ValueError(f"{what} out of range: {n}")
    return n


def _pairs(offsets):
    if not isinstance(offsets, torch.Tensor):
        raise TypeError("offsets must be a torch.Tensor")
    return _count((offsets.numel() - 1) // 2, "pairs")


def _matrices(a, dtype, what):
    if not isinstance(a, torch.Tensor) or a.dim() != 3:
        raise ValueError(f"{what} must be [groups, out_dim, in_dim]")
    return pbg._ptr(a, dtype, what)


# ------------------------------------------------------------------ entry points
def pbg_group_linear(ctx, x, a, offsets, y):
    """x [n, in_dim], a [groups, out_dim, in_dim] contiguous, offsets int64 [groups + 1], y [n, out_dim] (written)."""
    dt = _type(x, "x")
    ap = _matrices(a, dt, "a")
    if x.dim() != 2:
        raise ValueError("x must be [n, in_dim]")
    groups, m, k = a.shape
    _count(groups, "groups")
    n = x.shape[0]
    xp, ldx = _rows(x, dt, (n, k), "x")
    yp, ldy = _rows(y, dt, (n, m), "y")
    op = _vector(offsets, torch.int64, groups + 1, "offsets")
    _here(x, a, offsets, y)
    _check(ctx, library().pbg_group_linear(ctx, TYPES[dt], xp, ldx, ap, op, groups, n, k, m, yp, ldy))
    increment_version(y)   # the library writes through pointers, of which autograd sees nothing


def pbg_group_linear_backward(ctx, x, a, offsets, dy, dx=None, da=None):
    """dx [n, in_dim] and da [groups, out_dim, in_dim] are written; None: not wanted (x or a may then be None too)."""
    dt = _type(dy, "dy")
    if dy.dim() != 2:
        raise ValueError("dy must be [n, out_dim]")
    if a is None and da is None:
        raise ValueError("a is needed for dx, da for the matrices' gradients: one of them is required")
    n, m = dy.shape
    ap = None if a is None else _matrices(a, dt, "a")
    dap = None if da is None else _matrices(da, dt, "da")
    groups, rows, k = (a if a is not None else da).shape
    _count(groups, "groups")
    if rows != m or (a is not None and da is not None and a.shape != da.shape):
        raise ValueError(f"a and da must be [groups, {m}, in_dim]")
    xp, ldx = _rows(x, dt, (n, k), "x") if x is not None else (None, k)
    dxp, lddx = _rows(dx, dt, (n, k), "dx") if dx is not None else (None, k)
    dyp, lddy = _rows(dy, dt, (n, m), "dy")
    if n and ((dx is not None and a is None) or (da is not None and x is None)):
        raise ValueError("dx needs a, da needs x")
    op = _vector(offsets, torch.int64, groups + 1, "offsets")
    _here(x, a, offsets, dy, dx, da)
    _check(ctx, library().pbg_group_linear_backward(ctx, TYPES[dt], xp, ldx, ap, dyp, lddy, op, groups, n, k, m, dxp,
                                                    lddx, dap))
    increment_version([t for t in (dx, da) if t is not None])


def pbg_preference_loss(ctx, logits, labels, offsets, ref_logp, beta, smoothing, loss, logp, dlogp, row_stats):
    """logits [n, candidates], labels int32 [n], offsets int64 [2 pairs + 1]; ref_logp float32 [2 pairs] or None.
    Written: loss [pairs] (or None), logp [2 pairs], dlogp [2 pairs] (or None), row_stats [n, 2], all float32."""
    dt = _type(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [n, candidates]")
    n, cands = logits.shape
    pairs = _pairs(offsets)
    lp, ld = _rows(logits, dt, (n, cands), "logits")
    f = torch.float32
    args = (_vector(labels, torch.int32, n, "labels"), _vector(offsets, torch.int64, 2 * pairs + 1, "offsets"), pairs,
            n, cands, _vector(ref_logp, f, 2 * pairs, "ref_logp", True), float(beta), float(smoothing),
            _vector(loss, f, pairs, "loss", True), _vector(logp, f, 2 * pairs, "logp"),
            _vector(dlogp, f, 2 * pairs, "dlogp", True), _vector(row_stats, f, 2 * n, "row_stats"))
    _here(logits, labels, offsets, ref_logp, loss, logp, dlogp, row_stats)
    _check(ctx, library().pbg_preference_loss(ctx, TYPES[dt], lp, ld, *args))
    increment_version([t for t in (loss, logp, dlogp, row_stats) if t is not None])


def pbg_preference_loss_backward(ctx, logits, labels, offsets, row_stats, dlogp, dlogits):
    """dlogits [n, candidates] is written, and may be logits itself; dlogp float32 [2 pairs]."""
    dt = _type(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [n, candidates]")
    n, cands = logits.shape
    pairs = _pairs(offsets)
    lp, ld = _rows(logits, dt, (n, cands), "logits")
    dp, lddl = _rows(dlogits, dt, (n, cands), "dlogits")
    f = torch.float32
    args = (_vector(labels, torch.int32, n, "labels"), _vector(offsets, torch.int64, 2 * pairs + 1, "offsets"), pairs,
            n, cands, _vector(row_stats, f, 2 * n, "row_stats"), _vector(dlogp, f, 2 * pairs, "dlogp"))
    _here(logits, labels, offsets, row_stats, dlogp, dlogits)
    _check(ctx, library().pbg_preference_loss_backward(ctx, TYPES[dt], lp, ld, *args, dp, lddl))
    increment_version(dlogits)


def pbg_clip_gradients(ctx, grads, max_norm, outs=None) -> float:
    """grads: tensors of any shapes (contiguous; float32, bfloat16, float16 mixed); outs: as many tensors of their types
    and sizes, or None to scale in place.  Returns the joint norm before the scaling."""
    n, bound = len(grads), float(max_norm)
    if outs is not None and len(outs) != n:
        raise ValueError("one output per gradient")
    types, counts, gp = _values(grads, "grads")
    op = None
    if outs is not None:
        otypes, ocounts, op = _values(outs, "outs")
        if otypes != types or ocounts != counts:
            raise ValueError("every output must have its gradient's type and number of values")
    at = lambda v: None if v is None else v.buffer_info()[0]   # the arrays live until the call has returned
    norm = ctypes.c_double(0.0)
    _check(ctx, library().pbg_clip_gradients(ctx, n, at(types), at(counts), at(gp), at(op), bound,
                                             ctypes.byref(norm)))
    if outs is not None:
        increment_version(outs)
    elif norm.value > bound and math.isfinite(norm.value):
        increment_version(grads)
    return norm.value
