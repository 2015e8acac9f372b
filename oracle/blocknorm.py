"""Norms before and after a block with its gate and residual scale (fp64 numpy).

TEST INFRASTRUCTURE ONLY -- see oracle/__init__.py.

    u = y (mean(y^2) + eps)^(-1/2) w_post,  a = u silu(z),  h = x + c a,
    n = h (mean(h^2) + eps)^(-1/2) w_pre

Each of w_post, z, x, c and w_pre may be None (that step is left out).
"""

import numpy as np

__all__ = ["blocknorm_fwd", "blocknorm_bwd"]


def _norm(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def _norm_vjp(x, r, dy):
    """Gradient at x of y = x r(x), given that of y."""
    return r * (dy - x * r * r * np.mean(dy * x, axis=-1, keepdims=True))


def _f64(*xs):
    return [None if x is None else np.asarray(x, dtype=np.float64) for x in xs]


def _parts(y, w_post, z, x, c, eps):
    ry = None if w_post is None else _norm(y, eps)
    u = y if w_post is None else y * ry * w_post
    sg = None if z is None else 0.5 * (1.0 + np.tanh(0.5 * z))
    a = u if z is None else u * z * sg
    h = a if c is None else c * a
    return ry, u, sg, a, (h if x is None else x + h)


def blocknorm_fwd(y, w_post=None, z=None, x=None, c=None, w_pre=None, eps=1e-6):
    y, w_post, z, x, c, w_pre = _f64(y, w_post, z, x, c, w_pre)
    h = _parts(y, w_post, z, x, c, eps)[-1]
    return h, (None if w_pre is None else h * _norm(h, eps) * w_pre)


def blocknorm_bwd(y, dh, dn=None, w_post=None, z=None, x=None, c=None, w_pre=None, eps=1e-6):
    """Gradients of sum <h, dh> + <n, dn>: dict dy, dw_post, dgate, dx, dres_scale, dw_pre."""
    y, dh, dn, w_post, z, x, c, w_pre = _f64(y, dh, dn, w_post, z, x, c, w_pre)
    ry, u, sg, a, h = _parts(y, w_post, z, x, c, eps)
    rows = tuple(range(y.ndim - 1))
    out = dict.fromkeys(("dy", "dw_post", "dgate", "dx", "dres_scale", "dw_pre"))
    dh = np.zeros_like(h) if dh is None else dh
    if w_pre is not None:
        rh = _norm(h, eps)
        out["dw_pre"] = np.sum(dn * h * rh, axis=rows)
        dh = dh + _norm_vjp(h, rh, dn * w_pre)
    if x is not None:
        out["dx"] = dh
    if c is not None:
        out["dres_scale"] = np.sum(dh * a, axis=rows)
    da = dh if c is None else dh * c
    if z is not None:
        out["dgate"] = da * u * (sg + z * sg * (1.0 - sg))
        da = da * z * sg
    if w_post is not None:
        out["dw_post"] = np.sum(da * y * ry, axis=rows)
        da = _norm_vjp(y, ry, da * w_post)
    out["dy"] = da
    return out
