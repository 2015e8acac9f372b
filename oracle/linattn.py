"""Linear attention with a decay for each head, token by token (fp64 numpy).

TEST INFRASTRUCTURE ONLY -- see oracle/__init__.py.

    S_t = exp(g_t) S_{t-1} + k_t v_t^T,   o_t = scale * S_t^T q_t

q, k (B, T, H, Dk), v (B, T, Hv, Dv), g (B, T, Hv) or (Hv,), states (B, Hv, Dk, Dv);
value head j reads key head j // (Hv / H).  The backward is the adjoint of that loop
for L = sum_t <o_t, do_t> + <S_T, dS_T>, one line reversed at a time.
"""

import numpy as np

__all__ = ["linattn_fwd", "linattn_bwd", "linattn_packed_fwd", "linattn_packed_bwd"]


def _spread(q, k, v, g):
    """Everything in fp64 on the value heads, one decay a token."""
    q, k, v, g = (np.asarray(x, dtype=np.float64) for x in (q, k, v, g))
    G = v.shape[2] // k.shape[2]
    g = np.broadcast_to(g, v.shape[:3])
    return np.repeat(q, G, axis=2), np.repeat(k, G, axis=2), v, g


def _start(S0, v, Dk):
    B, _, H, Dv = v.shape
    return np.zeros((B, H, Dk, Dv)) if S0 is None else np.array(S0, dtype=np.float64)


def linattn_fwd(q, k, v, g, S0=None, scale=1.0):
    q, k, v, g = _spread(q, k, v, g)
    S = _start(S0, v, k.shape[-1])
    o = np.empty(v.shape)
    for t in range(v.shape[1]):
        S = np.exp(g[:, t])[..., None, None] * S + k[:, t][..., :, None] * v[:, t][..., None, :]
        o[:, t] = scale * np.einsum("bhkv,bhk->bhv", S, q[:, t])
    return o, S


def linattn_bwd(q, k, v, g, S0, do, dST=None, scale=1.0):
    """dict dq, dk, dv, dg, dS0 (dq, dk summed over a key head's value heads; dg shaped as g)."""
    Hk, per_head = k.shape[2], np.ndim(g) == 1
    q, k, v, g = _spread(q, k, v, g)
    do = np.asarray(do, dtype=np.float64)
    B, T, H, Dk = k.shape
    S = _start(S0, v, Dk)
    before = []
    for t in range(T):
        before.append(S)
        S = np.exp(g[:, t])[..., None, None] * S + k[:, t][..., :, None] * v[:, t][..., None, :]
    dS = np.zeros_like(S) if dST is None else np.array(dST, dtype=np.float64)
    dq, dk, dv, dg = np.empty(q.shape), np.empty(k.shape), np.empty(v.shape), np.empty(g.shape)
    for t in reversed(range(T)):
        a = np.exp(g[:, t])[..., None, None]
        now = a * before[t] + k[:, t][..., :, None] * v[:, t][..., None, :]
        dq[:, t] = scale * np.einsum("bhkv,bhv->bhk", now, do[:, t])
        dS = dS + scale * q[:, t][..., :, None] * do[:, t][..., None, :]
        dk[:, t] = np.einsum("bhkv,bhv->bhk", dS, v[:, t])
        dv[:, t] = np.einsum("bhkv,bhk->bhv", dS, k[:, t])
        dg[:, t] = np.sum(dS * a * before[t], axis=(-1, -2))
        dS = a * dS
    group = lambda x: x.reshape(B, T, Hk, H // Hk, Dk).sum(axis=3)  # noqa: E731
    return {"dq": group(dq), "dk": group(dk), "dv": dv, "dg": dg.sum(axis=(0, 1)) if per_head else dg, "dS0": dS}


def _cuts(cu, g, n):
    for i in range(len(cu) - 1):
        s = slice(int(cu[i]), int(cu[i + 1]))
        yield i, s, (g if np.ndim(g) == 1 else g[:, s])


def linattn_packed_fwd(q, k, v, g, cu, S0=None, scale=1.0):
    """The sequences of a packed batch (B = 1) run one by one; states (n_seqs, Hv, Dk, Dv)."""
    os, Ss = [], []
    for i, s, gi in _cuts(cu, g, len(cu) - 1):
        o, S = linattn_fwd(q[:, s], k[:, s], v[:, s], gi, None if S0 is None else S0[i:i + 1], scale)
        os.append(o)
        Ss.append(S)
    return np.concatenate(os, axis=1), np.concatenate(Ss)


def linattn_packed_bwd(q, k, v, g, cu, S0, do, dST=None, scale=1.0):
    parts = []
    for i, s, gi in _cuts(cu, g, len(cu) - 1):
        parts.append(linattn_bwd(q[:, s], k[:, s], v[:, s], gi, None if S0 is None else S0[i:i + 1], do[:, s],
                                 None if dST is None else dST[i:i + 1], scale))
    out = {n: np.concatenate([p[n] for p in parts], axis=1) for n in ("dq", "dk", "dv")}
    out["dg"] = sum(p["dg"] for p in parts) if np.ndim(g) == 1 else np.concatenate([p["dg"] for p in parts], axis=1)
    out["dS0"] = np.concatenate([p["dS0"] for p in parts])
    return out
