"""Gated linear recurrence, token by token (fp64 numpy).

TEST INFRASTRUCTURE ONLY -- see oracle/__init__.py.

    h_t = a_t h_{t-1} + m_t i_t x_t,  a_t = exp(g_t),  m_t = 1 or sqrt(1 - a_t^2)

x, g and i (None: 1) are (B, T, D), states (B, D).  A packed batch is its sequences one by one;
rows outside every sequence are NaN in the results.
"""

import numpy as np

__all__ = ["gatedrec_fwd", "gatedrec_bwd", "gatedrec_packed_fwd", "gatedrec_packed_bwd"]


def _f64(*xs):
    return [None if x is None else np.asarray(x, dtype=np.float64) for x in xs]


def _factors(x, g, i, normalize):
    m = np.sqrt(-np.expm1(2.0 * g)) if normalize else np.ones_like(g)
    return np.exp(g), m, np.ones_like(x) if i is None else i


def gatedrec_fwd(x, g, i=None, h0=None, normalize=False):
    """Returns (h of every token, the last state)."""
    x, g, i, h0 = _f64(x, g, i, h0)
    a, m, i = _factors(x, g, i, normalize)
    h = np.zeros(x[:, 0].shape if x.shape[1] else (x.shape[0], x.shape[2])) if h0 is None else h0
    o = np.empty_like(x)
    for t in range(x.shape[1]):
        h = a[:, t] * h + m[:, t] * i[:, t] * x[:, t]
        o[:, t] = h
    return o, h.copy()


def gatedrec_bwd(x, g, i, h0, do, dhT=None, normalize=False):
    """Gradients of sum <o, do> + <h_T, dh_T>: dict dx, dg, di (None without i), dh0."""
    o, _ = gatedrec_fwd(x, g, i, h0, normalize)
    gated = i is not None
    x, g, i, h0, do, dhT = _f64(x, g, i, h0, do, dhT)
    a, m, i = _factors(x, g, i, normalize)
    c = np.zeros((x.shape[0], x.shape[2])) if dhT is None else dhT.copy()
    d = {n: np.empty_like(x) for n in ("dx", "dg", "di")}
    for t in reversed(range(x.shape[1])):
        dh = do[:, t] + c
        before = o[:, t - 1] if t else (0.0 if h0 is None else h0)
        c = a[:, t] * dh
        d["dx"][:, t] = m[:, t] * i[:, t] * dh
        d["di"][:, t] = m[:, t] * x[:, t] * dh
        d["dg"][:, t] = c * before
        if normalize:  # dm/dg = -a^2 / m; at m = 0 the term is left out
            some = m[:, t] > 0
            slope = np.where(some, a[:, t] ** 2 / np.where(some, m[:, t], 1.0), 0.0)
            d["dg"][:, t] -= slope * i[:, t] * x[:, t] * dh
    d["dh0"] = c
    if not gated:
        d["di"] = None
    return d


def _part(x, a, b):
    return None if x is None else x[:, a:b]


def gatedrec_packed_fwd(x, g, i, h0, cu, normalize=False):
    o, hT = np.full(np.shape(x), np.nan), []
    for s, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
        o[:, a:b], h = gatedrec_fwd(x[:, a:b], g[:, a:b], _part(i, a, b), None if h0 is None else h0[s:s + 1], normalize)
        hT.append(h[0])
    return o, np.stack(hT)


def gatedrec_packed_bwd(x, g, i, h0, do, dhT, cu, normalize=False):
    d = {n: np.full(np.shape(x), np.nan) for n in ("dx", "dg", "di")}
    d["dh0"] = []
    for s, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
        one = gatedrec_bwd(x[:, a:b], g[:, a:b], _part(i, a, b), None if h0 is None else h0[s:s + 1], do[:, a:b],
                           None if dhT is None else dhT[s:s + 1], normalize)
        for n in ("dx", "dg", "di"):
            if one[n] is not None:
                d[n][:, a:b] = one[n]
        d["dh0"].append(one["dh0"][0])
    d["dh0"] = np.stack(d["dh0"])
    if i is None:
        d["di"] = None
    return d
