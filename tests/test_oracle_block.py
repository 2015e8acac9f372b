"""Pins of the oracle's linear attention and block norms (CPU): the forward against other
definitions and closed forms, the gradients against finite differences."""

import numpy as np
import pytest

from oracle import gdr2_recurrent_fwd
from oracle.blocknorm import blocknorm_bwd, blocknorm_fwd
from oracle.linattn import linattn_bwd, linattn_fwd, linattn_packed_bwd, linattn_packed_fwd
from tests.helpers import rel_l2


def _problem(seed, B=2, T=7, H=2, Hv=4, Dk=3, Dv=5, per_head=False):
    r = np.random.default_rng(seed)
    g = -np.abs(r.standard_normal((Hv,) if per_head else (B, T, Hv)))
    return dict(q=r.standard_normal((B, T, H, Dk)), k=r.standard_normal((B, T, H, Dk)), v=r.standard_normal((B, T, Hv, Dv)),
                g=g, S0=r.standard_normal((B, Hv, Dk, Dv)), do=r.standard_normal((B, T, Hv, Dv)),
                dST=r.standard_normal((B, Hv, Dk, Dv)))


def test_linattn_is_gdr2_without_erasing():
    p = _problem(0, H=4)
    one = np.ones(p["v"].shape)
    g = np.broadcast_to(p["g"][..., None], p["q"].shape)
    o, S = gdr2_recurrent_fwd(p["q"], p["k"], p["v"], g, np.zeros(p["q"].shape), one, p["S0"], 0.3)
    o2, S2 = linattn_fwd(p["q"], p["k"], p["v"], p["g"], p["S0"], 0.3)
    assert rel_l2(o2, o) < 1e-14 and rel_l2(S2, S) < 1e-14


def test_linattn_closed_form():
    p = _problem(1, B=1, H=1, Hv=1)
    G = np.cumsum(p["g"][0, :, 0])
    A = np.tril(np.exp(G[:, None] - G[None, :])) * (p["q"][0, :, 0] @ p["k"][0, :, 0].T)
    o = 0.5 * (A @ p["v"][0, :, 0] + np.exp(G)[:, None] * (p["q"][0, :, 0] @ p["S0"][0, 0]))
    assert rel_l2(linattn_fwd(p["q"], p["k"], p["v"], p["g"], p["S0"], 0.5)[0][0, :, 0], o) < 1e-13


@pytest.mark.parametrize("per_head", [False, True])
def test_linattn_gradients_by_differences(per_head):
    p = _problem(2, T=5, per_head=per_head)
    d = linattn_bwd(p["q"], p["k"], p["v"], p["g"], p["S0"], p["do"], p["dST"], 0.7)

    def loss(**kw):
        x = {n: kw.get(n, p[n]) for n in ("q", "k", "v", "g", "S0")}
        o, S = linattn_fwd(*x.values(), 0.7)
        return np.sum(o * p["do"]) + np.sum(S * p["dST"])

    r = np.random.default_rng(3)
    for n in ("q", "k", "v", "g", "S0"):
        for _ in range(3):
            e = r.standard_normal(p[n].shape)
            fd = (loss(**{n: p[n] + 1e-6 * e}) - loss(**{n: p[n] - 1e-6 * e})) / 2e-6
            assert abs(fd - np.sum(d["d" + n] * e)) < 1e-7 * (1 + abs(fd)), n


def test_linattn_packed_is_its_sequences():
    r = np.random.default_rng(4)
    cu, p = [0, 3, 3, 8], _problem(5, B=1, T=8)
    S0, dST = r.standard_normal((3, 4, 3, 5)), r.standard_normal((3, 4, 3, 5))
    o, S = linattn_packed_fwd(p["q"], p["k"], p["v"], p["g"], cu, S0, 0.3)
    d = linattn_packed_bwd(p["q"], p["k"], p["v"], p["g"], cu, S0, p["do"], dST, 0.3)
    assert np.array_equal(S[1], S0[1]) and np.array_equal(d["dS0"][1], dST[1])
    o2, S2 = linattn_fwd(p["q"][:, 3:], p["k"][:, 3:], p["v"][:, 3:], p["g"][:, 3:], S0[2:], 0.3)
    assert np.allclose(o[:, 3:], o2) and np.allclose(S[2], S2[0])


@pytest.mark.parametrize("parts", ["", "p", "g", "pg", "xn", "pxcn", "pgxcn", "n"])
def test_blocknorm_gradients_by_differences(parts):
    r = np.random.default_rng(len(parts))
    sh, D = (2, 3, 6), 6
    p = dict(y=r.standard_normal(sh))
    for key, name, shape in (("p", "w_post", D), ("g", "z", sh), ("x", "x", sh), ("c", "c", D), ("n", "w_pre", D)):
        if key in parts:
            p[name] = r.standard_normal(shape)
    dh, dn = r.standard_normal(sh), r.standard_normal(sh) if "n" in parts else None
    d = blocknorm_bwd(dh=dh, dn=dn, eps=1e-3, **p)

    def loss(q):
        h, n = blocknorm_fwd(eps=1e-3, **q)
        return np.sum(h * dh) + (0.0 if n is None else np.sum(n * dn))

    names = dict(y="dy", w_post="dw_post", z="dgate", x="dx", c="dres_scale", w_pre="dw_pre")
    for n in p:
        e = r.standard_normal(p[n].shape)
        fd = (loss({**p, n: p[n] + 1e-6 * e}) - loss({**p, n: p[n] - 1e-6 * e})) / 2e-6
        assert abs(fd - np.sum(d[names[n]] * e)) < 1e-7 * (1 + abs(fd)), n
    assert all(d[names[n]] is None for n in names if n not in p)


def test_blocknorm_worked_values():
    # mean square of (3, 4) is 12.5; with eps = 12.5 the divisor is 5
    h, n = blocknorm_fwd(np.array([[3.0, 4.0]]), w_post=np.array([1.0, 2.0]), eps=12.5)
    assert np.allclose(h, [[0.6, 1.6]]) and n is None
    h, n = blocknorm_fwd(np.array([[1.0, -1.0]]), x=np.array([[2.0, 5.0]]), c=np.ones(2), w_pre=np.ones(2), eps=0.0)
    assert np.allclose(h, [[3.0, 4.0]]) and np.allclose(n, np.array([[3.0, 4.0]]) / np.sqrt(12.5))
