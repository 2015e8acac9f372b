"""Gated feed-forward block -- the binding of include/gdr2_gatedff.h.

    y = (act(x w_gate^T) * (x w_up^T)) w_down^T

x (..., D), w_gate and w_up (F, D), w_down (D, F), all bfloat16 or all float32; D and F multiples
of 8; act "silu" or "gelu" (with erf).
"""

import ctypes

from . import _check, _dtype_code, _on, _ptr, _require, _require_ws, _stream, _torch, lib

__all__ = ["gdr2_gatedff_workspace_bytes", "gdr2_gatedff_fwd", "gdr2_gatedff_bwd", "Gdr2Gatedff", "GDR2_ACT_SILU",
           "GDR2_ACT_GELU"]

GDR2_ACT_SILU, GDR2_ACT_GELU = 0, 1
_ACTS = {"silu": GDR2_ACT_SILU, "gelu": GDR2_ACT_GELU}


class Gdr2Gatedff(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("D", ctypes.c_int32), ("F", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("act", ctypes.c_int32)]


def _declare(L):
    P, vp, sz = ctypes.POINTER(Gdr2Gatedff), ctypes.c_void_p, ctypes.c_size_t
    L.gdr2_gatedff_workspace_bytes.argtypes = [P, ctypes.c_int, ctypes.POINTER(sz)]
    L.gdr2_gatedff_fwd.argtypes = [P] + [vp] * 6 + [sz, ctypes.c_int, vp]
    L.gdr2_gatedff_bwd.argtypes = [P] + [vp] * 10 + [sz, ctypes.c_int, vp]
    for f in (L.gdr2_gatedff_workspace_bytes, L.gdr2_gatedff_fwd, L.gdr2_gatedff_bwd):
        f.restype = ctypes.c_int


def _inputs(x, w_gate, w_up, w_down, act):
    if x.dim() == 0 or w_gate.dim() != 2:
        raise ValueError("x: expected rows along the last axis, w_gate: (F, D)")
    D, F = x.shape[-1], w_gate.shape[0]
    if act not in _ACTS:
        raise ValueError(f"act: {act!r}, expected 'silu' or 'gelu'")
    code, dt, dev = _dtype_code(x), x.dtype, x.device
    _require("x", x, x.shape, dt)
    _require("w_gate", w_gate, (F, D), dt, dev)
    _require("w_up", w_up, (F, D), dt, dev)
    _require("w_down", w_down, (D, F), dt, dev)
    return Gdr2Gatedff(x.numel() // D if D else 0, D, F, code, _ACTS[act])


def gdr2_gatedff_workspace_bytes(problem, for_backward):
    """Bytes of workspace of a Gdr2Gatedff (for_backward: 1 also for save=True)."""
    n = ctypes.c_size_t(0)
    _check(lib().gdr2_gatedff_workspace_bytes(ctypes.byref(problem), int(for_backward), ctypes.byref(n)),
           "gdr2_gatedff_workspace_bytes")
    return n.value


def gdr2_gatedff_fwd(x, w_gate, w_up, w_down, *, act="silu", y=None, ws=None, save=False):
    """Forward.  Returns y, shaped as x.

    save=True (ws required, sized for the backward) leaves the hidden values that
    gdr2_gatedff_bwd(..., ws=ws, saved=True) starts from in ws."""
    torch = _torch()
    p = _inputs(x, w_gate, w_up, w_down, act)
    if y is None:
        y = torch.empty_like(x)
    else:
        _require("y", y, x.shape, x.dtype, x.device)
    need = gdr2_gatedff_workspace_bytes(p, 1 if save else 0)
    if ws is None:
        if save:
            raise ValueError("save=True needs the workspace that the backward will read")
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    _require_ws(ws, need, x.device)
    if p.rows == 0:
        return y
    with _on(x):
        st = lib().gdr2_gatedff_fwd(ctypes.byref(p), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(y), _ptr(ws),
                                    ws.numel(), 1 if save else 0, _stream())
    _check(st, "gdr2_gatedff_fwd")
    return y


def gdr2_gatedff_bwd(x, w_gate, w_up, w_down, dy, *, act="silu", grads=None, want_dx=True, want_dw=True, ws=None,
                     saved=False):
    """Gradients of sum <y, dy>.  Returns dict dx, dw_gate, dw_up, dw_down (None where not wanted).

    saved=True reads the hidden values that a save=True forward left in ws."""
    torch = _torch()
    p = _inputs(x, w_gate, w_up, w_down, act)
    dev, dt = x.device, x.dtype
    if dy is None:
        raise ValueError("dy: the gradient of y is required")
    _require("dy", dy, x.shape, dt, dev)
    if not want_dx and not want_dw:
        raise ValueError("neither want_dx nor want_dw: the call has nothing to do")
    g = dict(grads or {})
    for n, like, want in (("dx", x, want_dx), ("dw_gate", w_gate, want_dw), ("dw_up", w_up, want_dw),
                          ("dw_down", w_down, want_dw)):
        if not want:
            if g.get(n) is not None:
                raise ValueError(f"{n}: given, but not wanted")
            g[n] = None
        elif g.get(n) is None:
            g[n] = torch.empty_like(like)
        else:
            _require(n, g[n], like.shape, dt, dev)
    need = gdr2_gatedff_workspace_bytes(p, 1)
    if ws is None:
        if saved:
            raise ValueError("saved=True needs the workspace of the saving forward")
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _require_ws(ws, need, dev)
    if p.rows == 0:
        for n in ("dw_gate", "dw_up", "dw_down"):
            if g[n] is not None:
                g[n].zero_()
        return g
    with _on(x):
        st = lib().gdr2_gatedff_bwd(ctypes.byref(p), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy),
                                    _ptr(g["dx"]), _ptr(g["dw_gate"]), _ptr(g["dw_up"]), _ptr(g["dw_down"]), _ptr(ws),
                                    ws.numel(), 1 if saved else 0, _stream())
    _check(st, "gdr2_gatedff_bwd")
    return g
