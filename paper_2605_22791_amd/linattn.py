"""Linear attention with a decay for each head -- the binding of include/gdr2_linattn.h.

    S_t = exp(g_t) S_{t-1} + k_t v_t^T,    o_t = scale * S_t^T q_t

q, k (B, T, H, Dk) and v (B, T, Hv, Dv) in bfloat16 or float32, Hv a multiple of H;
log_decay float32, (B, T, Hv) for a decay of each token and value head or (Hv,) for
one of each value head; states float32, (B, Hv, Dk, Dv).  With cu_seqlens (int32
device tensor of n_seqs + 1 offsets; B = 1) the sequences of a packed batch, and
states (n_seqs, Hv, Dk, Dv).
"""

import ctypes

from . import (_check, _cu, _on, _problem, _ptr, _require, _require_grads, _require_ws, _stream, _torch, lib, Gdr2Problem)

__all__ = ["gdr2_linattn_workspace_bytes", "gdr2_linattn_fwd", "gdr2_linattn_bwd", "gdr2_linattn_step",
           "GDR2_DECAY_TOKEN", "GDR2_DECAY_HEAD"]

GDR2_DECAY_TOKEN, GDR2_DECAY_HEAD = 0, 1


def _declare(L):
    P, vp, i32, sz = ctypes.POINTER(Gdr2Problem), ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    L.gdr2_linattn_workspace_bytes.argtypes = [P, i32, ctypes.c_int, ctypes.POINTER(sz)]
    L.gdr2_linattn_fwd.argtypes = [P, i32, vp, i32] + [vp] * 8 + [sz, ctypes.c_int, vp]
    L.gdr2_linattn_bwd.argtypes = [P, i32, vp, i32] + [vp] * 13 + [sz, ctypes.c_int, vp]
    L.gdr2_linattn_step.argtypes = [P, i32, vp, i32] + [vp] * 6 + [vp]
    for f in (L.gdr2_linattn_workspace_bytes, L.gdr2_linattn_fwd, L.gdr2_linattn_bwd, L.gdr2_linattn_step):
        f.restype = ctypes.c_int


def _shapes(q, k, v, log_decay, cu_seqlens):
    """Checks the inputs; returns (B, T, Hv, Dk, Dv, sequences of a packed batch or 0, decay kind)."""
    torch = _torch()
    qs, vs = q.shape, v.shape
    if len(qs) != 4 or len(vs) != 4:
        raise ValueError("q, k: expected (B, T, H, Dk), v: (B, T, Hv, Dv)")
    B, T, H, Dk = qs
    _, _, Hv, Dv = vs
    if H == 0 or Hv % H != 0:
        raise ValueError(f"value heads ({Hv}) must be a multiple of key heads ({H})")
    dev, dt = q.device, q.dtype
    _require("q", q, qs, dt)
    _require("k", k, qs, dt, dev)
    _require("v", v, (B, T, Hv, Dv), dt, dev)
    head = log_decay.dim() == 1
    _require("log_decay", log_decay, (Hv,) if head else (B, T, Hv), torch.float32, dev)
    N = 0 if cu_seqlens is None else _cu(cu_seqlens, T, dev)
    return B, T, Hv, Dk, Dv, N, GDR2_DECAY_HEAD if head else GDR2_DECAY_TOKEN


def gdr2_linattn_workspace_bytes(problem, n_seqs, for_backward):
    """Bytes of workspace of a chunk call (n_seqs = 0: fixed length; for_backward: 1 also for save=True)."""
    n = ctypes.c_size_t(0)
    _check(lib().gdr2_linattn_workspace_bytes(ctypes.byref(problem), int(n_seqs), int(for_backward), ctypes.byref(n)),
           "gdr2_linattn_workspace_bytes")
    return n.value


def gdr2_linattn_fwd(q, k, v, log_decay, S0=None, *, cu_seqlens=None, scale=None, o=None, S_T=None, want_state=True,
                     ws=None, save=False):
    """Chunk forward.  Returns (o, S_T) (S_T None unless wanted); scale defaults to Dk ** -0.5.

    save=True (ws required, sized for the backward) leaves the states that
    gdr2_linattn_bwd(..., ws=ws, saved=True) starts from in ws."""
    torch = _torch()
    B, T, Hv, Dk, Dv, N, decay = _shapes(q, k, v, log_decay, cu_seqlens)
    state = (N or B, Hv, Dk, Dv)
    _require("S0", S0, state, torch.float32, q.device)
    prob = _problem(q, v, scale)
    if o is None:
        o = torch.empty_like(v)   # v is contiguous: 0.7 us less than by shape and type
    else:
        _require("o", o, (B, T, Hv, Dv), q.dtype, q.device)
    if S_T is None and want_state:
        S_T = torch.empty(state, dtype=torch.float32, device=q.device)
    else:
        _require("S_T", S_T, state, torch.float32, q.device)
    need = gdr2_linattn_workspace_bytes(prob, N, 1 if save else 0)
    if ws is None:
        if save:
            raise ValueError("save=True needs the workspace that the backward will read")
        ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _require_ws(ws, need, q.device)
    with _on(q):
        st = lib().gdr2_linattn_fwd(ctypes.byref(prob), decay, _ptr(cu_seqlens), N, _ptr(q), _ptr(k), _ptr(v),
                                    _ptr(log_decay), _ptr(S0), _ptr(o), _ptr(S_T), _ptr(ws), ws.numel(),
                                    1 if save else 0, _stream())
    _check(st, "gdr2_linattn_fwd")
    return o, S_T


def gdr2_linattn_bwd(q, k, v, log_decay, S0, dout, dS_T=None, *, cu_seqlens=None, scale=None, grads=None, want_dS0=True,
                     ws=None, saved=False):
    """Gradients of sum <o, dout> + <S_T, dS_T>.  Returns dict dq, dk, dv, dlog_decay, dS0.

    saved=True reads the states that a save=True forward left in ws."""
    torch = _torch()
    B, T, Hv, Dk, Dv, N, decay = _shapes(q, k, v, log_decay, cu_seqlens)
    state, dev = (N or B, Hv, Dk, Dv), q.device
    _require("S0", S0, state, torch.float32, dev)
    _require("dout", dout, (B, T, Hv, Dv), q.dtype, dev)
    _require("dS_T", dS_T, state, torch.float32, dev)
    prob = _problem(q, v, scale)
    g = dict(grads or {})
    for n, like in (("dq", q), ("dk", k), ("dv", v), ("dlog_decay", log_decay)):
        if g.get(n) is None:
            g[n] = torch.empty_like(like)
    if want_dS0 and g.get("dS0") is None:
        g["dS0"] = torch.empty(state, dtype=torch.float32, device=dev)
    g.setdefault("dS0", None)
    need = gdr2_linattn_workspace_bytes(prob, N, 1)
    if ws is None:
        if saved:
            raise ValueError("saved=True needs the workspace of the saving forward")
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _require_ws(ws, need, dev)
    _require_grads(g, {"dq": (q.shape, q.dtype), "dk": (k.shape, q.dtype), "dv": (v.shape, q.dtype),
                       "dlog_decay": (log_decay.shape, torch.float32), "dS0": (state, torch.float32)}, dev)
    with _on(q):
        st = lib().gdr2_linattn_bwd(ctypes.byref(prob), decay, _ptr(cu_seqlens), N, _ptr(q), _ptr(k), _ptr(v),
                                    _ptr(log_decay), _ptr(S0), _ptr(dout), _ptr(dS_T), _ptr(g["dq"]), _ptr(g["dk"]),
                                    _ptr(g["dv"]), _ptr(g["dlog_decay"]), _ptr(g["dS0"]), _ptr(ws), ws.numel(),
                                    1 if saved else 0, _stream())
    _check(st, "gdr2_linattn_bwd")
    return g


def gdr2_linattn_step(q, k, v, log_decay, S, *, cu_seqlens=None, scale=None, o=None):
    """Token by token over q.shape[1] tokens (decoding); S is updated in place.  Returns o."""
    torch = _torch()
    B, T, Hv, Dk, Dv, N, decay = _shapes(q, k, v, log_decay, cu_seqlens)
    if S is None:
        raise ValueError("S: the state that the tokens are added to is required")
    _require("S", S, (N or B, Hv, Dk, Dv), torch.float32, q.device)
    prob = _problem(q, v, scale)
    if o is None:
        o = torch.empty_like(v)
    else:
        _require("o", o, (B, T, Hv, Dv), q.dtype, q.device)
    with _on(q):
        st = lib().gdr2_linattn_step(ctypes.byref(prob), decay, _ptr(cu_seqlens), N, _ptr(q), _ptr(k), _ptr(v),
                                     _ptr(log_decay), _ptr(S), _ptr(o), _stream())
    _check(st, "gdr2_linattn_step")
    return o
