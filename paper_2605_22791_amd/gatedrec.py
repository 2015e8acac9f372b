"""Gated linear recurrence -- the binding of include/gdr2_gatedrec.h.

    h_t = exp(g_t) h_{t-1} + m_t i_t x_t,    o_t = h_t

for each channel; m = 1, or sqrt(1 - exp(2 g)) with normalize=True.  x and the input gate i (None:
1) are (B, T, D) in bfloat16 or float32, log_decay g (B, T, D) float32, g <= 0, states (B, D)
float32.  With cu_seqlens (int32 device tensor of n_seqs + 1 offsets; B = 1) the sequences of a
packed batch, and states (n_seqs, D); rows outside every sequence keep what the outputs held.
"""

import ctypes

from . import (_check, _cu, _dtype_code, _on, _ptr, _require, _require_grads, _require_ws, _stream, _torch, lib)

__all__ = ["gdr2_gatedrec_workspace_bytes", "gdr2_gatedrec_fwd", "gdr2_gatedrec_bwd", "gdr2_gatedrec_step",
           "Gdr2Gatedrec"]


class Gdr2Gatedrec(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("normalize", ctypes.c_int32)]


def _declare(L):
    P, vp, i32, sz = ctypes.POINTER(Gdr2Gatedrec), ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    L.gdr2_gatedrec_workspace_bytes.argtypes = [P, i32, ctypes.c_int, ctypes.POINTER(sz)]
    L.gdr2_gatedrec_fwd.argtypes = [P, vp, i32] + [vp] * 7 + [sz, ctypes.c_int, vp]
    L.gdr2_gatedrec_bwd.argtypes = [P, vp, i32] + [vp] * 11 + [sz, ctypes.c_int, vp]
    L.gdr2_gatedrec_step.argtypes = [P, vp, i32] + [vp] * 6
    for f in (L.gdr2_gatedrec_workspace_bytes, L.gdr2_gatedrec_fwd, L.gdr2_gatedrec_bwd, L.gdr2_gatedrec_step):
        f.restype = ctypes.c_int


def _inputs(x, log_decay, gate, cu_seqlens, normalize):
    """Checks the inputs; returns (problem, sequences of a packed batch or 0, shape of the states)."""
    torch = _torch()
    if x.dim() != 3:
        raise ValueError("x: expected (B, T, D)")
    B, T, D = shape = x.shape
    code = _dtype_code(x)
    _require("x", x, shape, x.dtype)
    _require("log_decay", log_decay, shape, torch.float32, x.device)
    _require("gate", gate, shape, x.dtype, x.device)
    N = 0 if cu_seqlens is None else _cu(cu_seqlens, T, x.device)
    return Gdr2Gatedrec(B, T, D, code, 1 if normalize else 0), N, (N or B, D)


def gdr2_gatedrec_workspace_bytes(problem, n_seqs, for_backward):
    """Bytes of workspace of a Gdr2Gatedrec (n_seqs = 0: fixed length; for_backward: 1 also for save=True)."""
    n = ctypes.c_size_t(0)
    _check(lib().gdr2_gatedrec_workspace_bytes(ctypes.byref(problem), int(n_seqs), int(for_backward), ctypes.byref(n)),
           "gdr2_gatedrec_workspace_bytes")
    return n.value


def gdr2_gatedrec_fwd(x, log_decay, gate=None, h0=None, *, cu_seqlens=None, normalize=False, o=None, h_T=None,
                      want_state=True, ws=None, save=False):
    """Forward.  Returns (o, h_T) (h_T None unless wanted).

    save=True (ws required, sized for the backward) leaves the states that
    gdr2_gatedrec_bwd(..., ws=ws, saved=True) starts from in ws."""
    torch = _torch()
    p, N, state = _inputs(x, log_decay, gate, cu_seqlens, normalize)
    dev = x.device
    _require("h0", h0, state, torch.float32, dev)
    if o is None:
        o = torch.empty_like(x)
    else:
        _require("o", o, x.shape, x.dtype, dev)
    if h_T is None and want_state:
        h_T = torch.empty(state, dtype=torch.float32, device=dev)
    else:
        _require("h_T", h_T, state, torch.float32, dev)
    need = gdr2_gatedrec_workspace_bytes(p, N, 1 if save else 0)
    if ws is None:
        if save:
            raise ValueError("save=True needs the workspace that the backward will read")
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _require_ws(ws, need, dev)
    with _on(x):
        st = lib().gdr2_gatedrec_fwd(ctypes.byref(p), _ptr(cu_seqlens), N, _ptr(x), _ptr(log_decay), _ptr(gate), _ptr(h0),
                                     _ptr(o), _ptr(h_T), _ptr(ws), ws.numel(), 1 if save else 0, _stream())
    _check(st, "gdr2_gatedrec_fwd")
    return o, h_T


def gdr2_gatedrec_bwd(x, log_decay, gate, h0, dout, dh_T=None, *, cu_seqlens=None, normalize=False, grads=None,
                      want_dh0=True, ws=None, saved=False):
    """Gradients of sum <o, dout> + <h_T, dh_T>.  Returns dict dx, dlog_decay, dgate (None without a gate), dh0.

    saved=True reads the states that a save=True forward left in ws."""
    torch = _torch()
    p, N, state = _inputs(x, log_decay, gate, cu_seqlens, normalize)
    dev = x.device
    _require("h0", h0, state, torch.float32, dev)
    if dout is None:
        raise ValueError("dout: the gradient of o is required")
    _require("dout", dout, x.shape, x.dtype, dev)
    _require("dh_T", dh_T, state, torch.float32, dev)
    g = dict(grads or {})
    if gate is None and g.get("dgate") is not None:
        raise ValueError("dgate: given, but the call has no gate")
    for n, like in (("dx", x), ("dlog_decay", log_decay), ("dgate", gate)):
        if g.get(n) is None:
            g[n] = None if like is None else torch.empty_like(like)
    if want_dh0 and g.get("dh0") is None:
        g["dh0"] = torch.empty(state, dtype=torch.float32, device=dev)
    g.setdefault("dh0", None)
    _require_grads(g, {"dx": (x.shape, x.dtype), "dlog_decay": (x.shape, torch.float32), "dgate": (x.shape, x.dtype),
                       "dh0": (state, torch.float32)}, dev)
    need = gdr2_gatedrec_workspace_bytes(p, N, 1)
    if ws is None:
        if saved:
            raise ValueError("saved=True needs the workspace of the saving forward")
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _require_ws(ws, need, dev)
    with _on(x):
        st = lib().gdr2_gatedrec_bwd(ctypes.byref(p), _ptr(cu_seqlens), N, _ptr(x), _ptr(log_decay), _ptr(gate), _ptr(h0),
                                     _ptr(dout), _ptr(dh_T), _ptr(g["dx"]), _ptr(g["dlog_decay"]), _ptr(g["dgate"]),
                                     _ptr(g["dh0"]), _ptr(ws), ws.numel(), 1 if saved else 0, _stream())
    _check(st, "gdr2_gatedrec_bwd")
    return g


def gdr2_gatedrec_step(x, log_decay, gate, h, *, cu_seqlens=None, normalize=False, o=None):
    """Token by token over x.shape[1] tokens (decoding); h is updated in place.  Returns o."""
    torch = _torch()
    p, N, state = _inputs(x, log_decay, gate, cu_seqlens, normalize)
    if h is None:
        raise ValueError("h: the state that the tokens are added to is required")
    _require("h", h, state, torch.float32, x.device)
    if o is None:
        o = torch.empty_like(x)
    else:
        _require("o", o, x.shape, x.dtype, x.device)
    with _on(x):
        st = lib().gdr2_gatedrec_step(ctypes.byref(p), _ptr(cu_seqlens), N, _ptr(x), _ptr(log_decay), _ptr(gate), _ptr(h),
                                      _ptr(o), _stream())
    _check(st, "gdr2_gatedrec_step")
    return o
