"""Dropout with the block's residual sum -- the binding of include/gdr2_dropout.h.

    y = residual + keep * x / (1 - p)          (residual None: no sum)

keep comes from a counter-based generator (Philox 4x32, ten rounds) by the element's place in
memory, the seed and the offset, each 64 bits, and is never stored: the backward forms it
again.  x is bfloat16 or float32; residual and y share a type, that of x or float32.  offset
is an int, or an int64 device tensor of one element that the kernel reads when it runs, so that a
captured call can drop other elements on every replay.  more is such a tensor too, added to an offset that
is an int (modulo 2^64): the dropouts of a captured step share one counter and have an offset each.
"""

import ctypes

from . import GDR2_BF16, GDR2_FP32, _check, _dtype_code, _on, _ptr, _require, _stream, _torch, lib

__all__ = ["gdr2_dropout_fwd", "gdr2_dropout_bwd", "Gdr2Dropout"]

_M64 = (1 << 64) - 1


class Gdr2Dropout(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("dtype", ctypes.c_int32), ("stream_dtype", ctypes.c_int32)]


def _declare(L):
    P, vp = ctypes.POINTER(Gdr2Dropout), ctypes.c_void_p
    L.gdr2_dropout_fwd.argtypes = [P] + [vp] * 5
    L.gdr2_dropout_bwd.argtypes = [P] + [vp] * 4
    for f in (L.gdr2_dropout_fwd, L.gdr2_dropout_bwd):
        f.restype = ctypes.c_int


def _problem(t, p, seed, offset, more, code, stream):
    """The problem and the device part of the offset (or None)."""
    torch = _torch()
    if not 0.0 <= p < 1.0:
        raise ValueError(f"p: {p}, expected 0 <= p < 1")
    name = "more"
    if isinstance(offset, torch.Tensor):
        if more is not None:
            raise ValueError("more: beside an offset that is a tensor itself")
        name, more, offset = "offset", offset, 0
    if more is not None:
        _require(name, more, more.shape, torch.int64, t.device)
        if more.numel() != 1:
            raise ValueError(f"{name}: expected an int64 device tensor of one element")
    return Gdr2Dropout(t.numel(), float(p), int(seed) & _M64, int(offset) & _M64, code, stream), more


def gdr2_dropout_fwd(x, p, seed, *, offset=0, more=None, residual=None, y=None):
    """Returns y, of the type of the residual (of x without one).  y may be the residual, or x of that type."""
    torch = _torch()
    code, dev = _dtype_code(x), x.device
    _require("x", x, x.shape, x.dtype)
    stream = x.dtype
    if residual is not None:
        stream = residual.dtype
        if stream != x.dtype and stream != torch.float32:
            raise TypeError(f"residual: {stream}, expected {x.dtype} or torch.float32")
        _require("residual", residual, x.shape, stream, dev)
    prob, more = _problem(x, p, seed, offset, more, code, GDR2_FP32 if stream is torch.float32 else GDR2_BF16)
    if y is None:
        y = torch.empty_like(x, dtype=stream)
    else:
        _require("y", y, x.shape, stream, dev)
    if prob.n == 0:
        return y
    with _on(x):
        st = lib().gdr2_dropout_fwd(ctypes.byref(prob), _ptr(more), _ptr(x), _ptr(residual), _ptr(y), _stream())
    _check(st, "gdr2_dropout_fwd")
    return y


def gdr2_dropout_bwd(dy, p, seed, *, offset=0, more=None, dtype=None, dx=None):
    """Returns dx, the gradient at x, in `dtype` (that of x; None: that of dy).  The residual's gradient is dy."""
    torch = _torch()
    code = _dtype_code(dy)
    _require("dy", dy, dy.shape, dy.dtype)
    if dtype is None:
        dtype = dy.dtype if dx is None else dx.dtype
    if dtype != dy.dtype and (dtype, dy.dtype) != (torch.bfloat16, torch.float32):
        raise TypeError(f"dtype: {dtype} beside a gradient in {dy.dtype}")
    prob, more = _problem(dy, p, seed, offset, more, GDR2_FP32 if dtype is torch.float32 else GDR2_BF16, code)
    if dx is None:
        dx = torch.empty_like(dy, dtype=dtype)
    else:
        _require("dx", dx, dy.shape, dtype, dy.device)
    if prob.n == 0:
        return dx
    with _on(dy):
        st = lib().gdr2_dropout_bwd(ctypes.byref(prob), _ptr(more), _ptr(dy), _ptr(dx), _stream())
    _check(st, "gdr2_dropout_bwd")
    return dx
