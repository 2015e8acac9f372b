"""Gated feed-forward block (fp64 numpy).

TEST INFRASTRUCTURE ONLY -- see oracle/__init__.py.

    y = (act(x Wg^T) * (x Wu^T)) Wd^T,   act: SiLU or GELU (with erf)
"""

import math

import numpy as np

__all__ = ["gatedff_fwd", "gatedff_bwd"]

_erf = np.vectorize(math.erf, otypes=[float])


def _act(g, act):
    """act(g) and its slope."""
    if act == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * g))
        return g * s, s + g * s * (1.0 - s)
    s = 0.5 * (1.0 + _erf(g / math.sqrt(2.0)))
    return g * s, s + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def _f64(*xs):
    return [np.asarray(x, dtype=np.float64) for x in xs]


def gatedff_fwd(x, wg, wu, wd, act="silu"):
    x, wg, wu, wd = _f64(x, wg, wu, wd)
    return (_act(x @ wg.T, act)[0] * (x @ wu.T)) @ wd.T


def gatedff_bwd(x, wg, wu, wd, dy, act="silu"):
    """Gradients of sum <y, dy> for rows x (n, D): dict dx, dw_gate, dw_up, dw_down."""
    x, wg, wu, wd, dy = _f64(x, wg, wu, wd, dy)
    g, u = x @ wg.T, x @ wu.T
    a, slope = _act(g, act)
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    return dict(dx=dg @ wg + du @ wu, dw_gate=dg.T @ x, dw_up=du.T @ x, dw_down=dy.T @ (a * u))
