"""Norms before and after a block with its gate and residual scale -- the binding of
include/gdr2_blocknorm.h.

    u = y * rsqrt(mean(y^2) + eps) * w_post     (w_post None: u = y)
    a = u * silu(gate)                          (gate None: a = u)
    h = x + res_scale * a                       (res_scale None: 1; x None: no sum)
    n = h * rsqrt(mean(h^2) + eps) * w_pre      (w_pre None: no n)

over the last axis of y (any width up to 8192).  y, gate and n are bfloat16 or
float32; x and h share a type, that of y or float32; w_post, res_scale and w_pre
are float32.
"""

import ctypes

from . import _check, _dtype_code, _on, _ptr, _require, _require_ws, _stream, _torch, lib

__all__ = ["gdr2_blocknorm_workspace_bytes", "gdr2_blocknorm_fwd", "gdr2_blocknorm_bwd", "Gdr2Blocknorm"]


class Gdr2Blocknorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("stream_dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


def _declare(L):
    P, vp, sz = ctypes.POINTER(Gdr2Blocknorm), ctypes.c_void_p, ctypes.c_size_t
    L.gdr2_blocknorm_fwd.argtypes = [P] + [vp] * 9
    L.gdr2_blocknorm_workspace_bytes.argtypes = [P, ctypes.POINTER(sz)]
    L.gdr2_blocknorm_bwd.argtypes = [P] + [vp] * 15 + [sz, vp]
    for f in (L.gdr2_blocknorm_fwd, L.gdr2_blocknorm_workspace_bytes, L.gdr2_blocknorm_bwd):
        f.restype = ctypes.c_int


def _inputs(y, w_post, gate, x, res_scale, w_pre, eps):
    """Checks the inputs; returns the problem and the type of h."""
    torch = _torch()
    if y.dim() == 0:
        raise ValueError("y: expected rows along the last axis")
    D, dev = y.shape[-1], y.device
    code = _dtype_code(y)
    shape, dt = y.shape, y.dtype
    _require("y", y, shape, dt)
    _require("gate", gate, shape, dt, dev)
    if x is not None and x.dtype != dt and x.dtype != torch.float32:
        raise TypeError(f"x: {x.dtype}, expected {dt} or torch.float32")
    stream = dt if x is None else x.dtype
    _require("x", x, shape, stream, dev)
    _require("w_post", w_post, (D,), torch.float32, dev)
    _require("res_scale", res_scale, (D,), torch.float32, dev)
    _require("w_pre", w_pre, (D,), torch.float32, dev)
    rows = y.numel() // D if D else 0
    return Gdr2Blocknorm(rows, D, code, 1 if stream is torch.float32 else 0, float(eps)), stream


def gdr2_blocknorm_workspace_bytes(problem):
    """Bytes of workspace of the backward of a Gdr2Blocknorm."""
    n = ctypes.c_size_t(0)
    _check(lib().gdr2_blocknorm_workspace_bytes(ctypes.byref(problem), ctypes.byref(n)), "gdr2_blocknorm_workspace_bytes")
    return n.value


def gdr2_blocknorm_fwd(y, *, w_post=None, gate=None, x=None, res_scale=None, w_pre=None, eps=1e-6, h=None, n=None,
                       want_h=True):
    """Returns (h, n); n is None without w_pre, h is None with want_h=False."""
    torch = _torch()
    p, stream = _inputs(y, w_post, gate, x, res_scale, w_pre, eps)
    if h is None and want_h:
        h = torch.empty_like(y, dtype=stream)
    else:
        _require("h", h, y.shape, stream, y.device)
    if n is None and w_pre is not None:
        n = torch.empty_like(y)
    elif n is not None and w_pre is None:
        raise ValueError("n: given, but the call has no w_pre")
    else:
        _require("n", n, y.shape, y.dtype, y.device)
    if p.rows == 0:
        return h, n
    with _on(y):
        st = lib().gdr2_blocknorm_fwd(ctypes.byref(p), _ptr(y), _ptr(w_post), _ptr(gate), _ptr(x), _ptr(res_scale),
                                      _ptr(w_pre), _ptr(h), _ptr(n), _stream())
    _check(st, "gdr2_blocknorm_fwd")
    return h, n


def gdr2_blocknorm_bwd(y, dh, dn=None, *, w_post=None, gate=None, x=None, res_scale=None, w_pre=None, eps=1e-6,
                       grads=None, ws=None):
    """Gradients of sum <h, dh> + <n, dn> (dh None: zero).  Returns dict dy, dw_post, dgate,
    dx, dres_scale, dw_pre, None for what the call did not have."""
    torch = _torch()
    p, stream = _inputs(y, w_post, gate, x, res_scale, w_pre, eps)
    dev = y.device
    _require("dh", dh, y.shape, stream, dev)
    _require("dn", dn, y.shape, y.dtype, dev)
    if (dn is None) != (w_pre is None):
        raise ValueError("dn is given exactly where w_pre is")
    if dh is None and dn is None:
        raise ValueError("neither dh nor dn is given")
    g = dict(grads or {})
    for name, like in (("dy", y), ("dw_post", w_post), ("dgate", gate), ("dx", x), ("dres_scale", res_scale),
                       ("dw_pre", w_pre)):
        if like is None:
            if g.get(name) is not None:
                raise ValueError(f"{name}: given, but the call has no such input")
            g[name] = None
        elif g.get(name) is None:
            g[name] = torch.empty_like(like)
        else:
            _require(name, g[name], like.shape, like.dtype, dev)
    if p.rows == 0:
        for name in ("dw_post", "dres_scale", "dw_pre"):
            if g[name] is not None:
                g[name].zero_()
        return g
    need = gdr2_blocknorm_workspace_bytes(p)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _require_ws(ws, need, dev)
    with _on(y):
        st = lib().gdr2_blocknorm_bwd(ctypes.byref(p), _ptr(y), _ptr(w_post), _ptr(gate), _ptr(x), _ptr(res_scale),
                                      _ptr(w_pre), _ptr(dh), _ptr(dn), _ptr(g["dy"]), _ptr(g["dw_post"]), _ptr(g["dgate"]),
                                      _ptr(g["dx"]), _ptr(g["dres_scale"]), _ptr(g["dw_pre"]), _ptr(ws), ws.numel(),
                                      _stream())
    _check(st, "gdr2_blocknorm_bwd")
    return g
