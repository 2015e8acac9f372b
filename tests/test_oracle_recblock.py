"""Pins of the oracle's gated linear recurrence, gated feed-forward block and dropout (CPU): closed
forms, other definitions, published values, finite differences."""

import math

import numpy as np
import pytest

from oracle.dropout import dropout_fwd, dropout_keep, philox, words
from oracle.gatedff import gatedff_bwd, gatedff_fwd
from oracle.gatedrec import gatedrec_bwd, gatedrec_fwd, gatedrec_packed_bwd, gatedrec_packed_fwd
from oracle.linattn import linattn_fwd
from tests.helpers import rel_l2


def _problem(seed, B=2, T=6, D=5, gate=True):
    r = np.random.default_rng(seed)
    f = lambda *s: r.standard_normal(s)  # noqa: E731
    return dict(x=f(B, T, D), g=-np.abs(f(B, T, D)), i=1 / (1 + np.exp(-f(B, T, D))) if gate else None, h0=f(B, D)), f(B, T, D), f(B, D)


def test_recurrence_closed_form():
    p, _, _ = _problem(0)
    G = np.cumsum(p["g"], axis=1)
    o, h = gatedrec_fwd(**p)
    for t in range(6):
        want = np.exp(G[:, t]) * p["h0"] + sum(np.exp(G[:, t] - G[:, s]) * p["i"][:, s] * p["x"][:, s] for s in range(t + 1))
        assert rel_l2(o[:, t], want) < 1e-14
    assert np.array_equal(h, o[:, -1])


def test_recurrence_is_linear_attention_of_one_channel():
    p, _, _ = _problem(1, D=1, gate=False)
    one = np.ones((2, 6, 1, 1))
    o, S = linattn_fwd(one, one, p["x"][..., None], p["g"], p["h0"][..., None, None], 1.0)
    o2, h = gatedrec_fwd(**p)
    assert rel_l2(o2[..., 0], o[..., 0, 0]) < 1e-14 and rel_l2(h[:, 0], S[:, 0, 0, 0]) < 1e-14


def test_normalized_input_keeps_the_variance():
    """Of independent inputs of variance 1: the sum of the squared weights of h_t is 1 - a^(2t), its limit 1."""
    g = np.full((1, 300, 1), -0.05)
    squares = 0.0
    for s in range(300):
        x = np.zeros((1, 300, 1))
        x[0, s] = 1.0
        squares += gatedrec_fwd(x, g, normalize=True)[1][0, 0] ** 2
    assert abs(squares - (1.0 - math.exp(-0.1 * 300))) < 1e-12


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("gate", [False, True])
def test_recurrence_gradients_by_differences(normalize, gate):
    p, do, dhT = _problem(2, gate=gate)
    d = gatedrec_bwd(**p, do=do, dhT=dhT, normalize=normalize)

    def loss(**kw):
        o, h = gatedrec_fwd(**{**p, **kw}, normalize=normalize)
        return np.sum(o * do) + np.sum(h * dhT)

    r = np.random.default_rng(3)
    for n in ("x", "g", "h0") + (("i",) if gate else ()):
        e = r.standard_normal(p[n].shape)
        if n == "g":
            e *= p["g"]  # g stays negative, and its differences small beside it
        fd = (loss(**{n: p[n] + 1e-6 * e}) - loss(**{n: p[n] - 1e-6 * e})) / 2e-6
        assert abs(fd - np.sum(d["d" + n] * e)) < 1e-7 * (1 + abs(fd)), n
    assert gate or d["di"] is None


def test_recurrence_packed_is_its_sequences():
    p, do, _ = _problem(4, B=1, T=9)
    r = np.random.default_rng(5)
    h0, dhT, cu = r.standard_normal((3, 5)), r.standard_normal((3, 5)), [1, 4, 4, 8]
    o, h = gatedrec_packed_fwd(p["x"], p["g"], p["i"], h0, cu)
    d = gatedrec_packed_bwd(p["x"], p["g"], p["i"], h0, do, dhT, cu)
    assert np.array_equal(h[1], h0[1]) and np.array_equal(d["dh0"][1], dhT[1])
    assert np.isnan(o[0, [0, 8]]).all() and np.isnan(d["dx"][0, [0, 8]]).all()
    o2, h2 = gatedrec_fwd(p["x"][:, 4:8], p["g"][:, 4:8], p["i"][:, 4:8], h0[2:])
    assert np.array_equal(o[:, 4:8], o2) and np.array_equal(h[2], h2[0])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_feed_forward_gradients_by_differences(act):
    r = np.random.default_rng(6)
    p = dict(x=r.standard_normal((3, 4)), wg=r.standard_normal((7, 4)), wu=r.standard_normal((7, 4)), wd=r.standard_normal((4, 7)))
    dy = r.standard_normal((3, 4))
    d = gatedff_bwd(**p, dy=dy, act=act)
    for n, m in (("x", "dx"), ("wg", "dw_gate"), ("wu", "dw_up"), ("wd", "dw_down")):
        e = r.standard_normal(p[n].shape)
        up, down = (np.sum(gatedff_fwd(**{**p, n: p[n] + s * e}, act=act) * dy) for s in (1e-6, -1e-6))
        assert abs((up - down) / 2e-6 - np.sum(d[m] * e)) < 1e-7 * (1 + abs(up - down) / 2e-6), n


def test_feed_forward_worked_values():
    one = np.ones((1, 1))
    # silu(2) = 2 / (1 + e^-2); gelu(1) = Phi(1)
    assert abs(gatedff_fwd(one, 2 * one, 3 * one, 5 * one)[0, 0] - 15 * 2 / (1 + math.exp(-2))) < 1e-13
    assert abs(gatedff_fwd(one, one, one, one, "gelu")[0, 0] - 0.8413447460685429) < 1e-13


def test_generator_known_values():
    """The method's published known-answer values, and a standard library's 10000th word of its default engine."""
    assert philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    # C++26's philox4x32: key 20111115, counter from 0
    assert words(9999, 1, 20111115, 0)[0] == 1955073260


def test_words_do_not_depend_on_where_a_call_starts():
    whole = words(0, 40, 7 << 40, 5 << 33)
    assert np.array_equal(words(13, 11, 7 << 40, 5 << 33), whole[13:24])
    assert not np.array_equal(words(0, 40, 7 << 40, 6 << 33), whole)


def test_dropout_values():
    x = np.arange(1.0, 2001.0)
    y = dropout_fwd(x, 0.25, 3)
    keep = dropout_keep(2000, 0.25, 3, 0)
    assert np.array_equal(y, np.where(keep, x / 0.75, 0.0))
    assert abs(keep.mean() - 0.75) < 4 * math.sqrt(0.25 * 0.75 / 2000)
    assert np.array_equal(dropout_fwd(x, 0.0, 3), x)
