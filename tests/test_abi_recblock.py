"""C-ABI and binding checks of the gated linear recurrence, the gated feed-forward block and dropout
that need no GPU.

Every C call here is rejected before any HIP call, so the made-up pointers are never used.
"""

import ctypes
import os
import re

import pytest

import paper_2605_22791_amd as g2

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(not os.path.exists(g2.lib_path()),
                                reason="libgdr2.so not built (python -m paper_2605_22791_amd.build)")

FAKE = 0x10000
BIG = 1 << 62
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = g2.GDR2_OK, g2.GDR2_EINVAL, g2.GDR2_EUNSUPPORTED, g2.GDR2_EWORKSPACE


@pytest.mark.parametrize("header,names", [
    ("gdr2_gatedrec.h", ["gdr2_gatedrec_bwd", "gdr2_gatedrec_fwd", "gdr2_gatedrec_step", "gdr2_gatedrec_workspace_bytes"]),
    ("gdr2_gatedff.h", ["gdr2_gatedff_bwd", "gdr2_gatedff_fwd", "gdr2_gatedff_workspace_bytes"]),
    ("gdr2_dropout.h", ["gdr2_dropout_bwd", "gdr2_dropout_fwd"])])
def test_headers_declare_what_the_library_exports(header, names):
    text = open(os.path.join(ROOT, "include", header)).read()
    assert sorted(set(re.findall(r"^gdr2_status\s+(gdr2_\w+)\s*\(", text, re.M))) == names
    assert all(hasattr(g2.lib(), n) and hasattr(g2, n) for n in names)


# ------------------------------------------------------------------ gated linear recurrence
def _rec(**kw):
    return g2.Gdr2Gatedrec(**{**dict(B=2, T=128, D=96, dtype=g2.GDR2_BF16, normalize=1), **kw})


def _rc(which, prob, cu=None, n=0, ptrs=None, ws_bytes=BIG):
    """fwd: x g i h0 o hT ws; bwd: x g i h0 dout dhT dx dg di dh0 ws; step: x g i h o"""
    p = [FAKE] * {"fwd": 7, "bwd": 11, "step": 5}[which]
    for i, x in (ptrs or {}).items():
        p[i] = x
    tail = [] if which == "step" else [ws_bytes, 0]
    return getattr(g2.lib(), "gdr2_gatedrec_" + which)(ctypes.byref(prob), cu, n, *p, *tail, None)


@pytest.mark.parametrize("which", ["fwd", "bwd", "step"])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), EINVAL), (dict(T=0), EINVAL), (dict(D=-3), EINVAL), (dict(dtype=2), EINVAL), (dict(normalize=2), EINVAL),
    (dict(D=65537), EUNSUPPORTED), (dict(B=1 << 16, T=1 << 15), EUNSUPPORTED), (dict(B=1 << 15, T=1 << 15, D=1), EUNSUPPORTED),
    (dict(B=1 << 10, T=1 << 17, D=1024), EUNSUPPORTED)])
def test_recurrence_problem_checks(which, kw, code):
    assert _rc(which, _rec(**kw)) == code
    n = ctypes.c_size_t(0)
    assert g2.lib().gdr2_gatedrec_workspace_bytes(ctypes.byref(_rec(**kw)), 0, 0, ctypes.byref(n)) == code


def test_recurrence_argument_checks():
    for which in ("fwd", "bwd", "step"):
        assert _rc(which, _rec(), n=-1) == EINVAL
        assert _rc(which, _rec(), n=3, cu=FAKE) == EINVAL            # B != 1
        assert _rc(which, _rec(B=1), n=3, cu=None) == EINVAL
        assert _rc(which, _rec(B=1), n=3, cu=FAKE + 2) == EINVAL
        assert _rc(which, _rec(B=1), n=(1 << 24) + 1, cu=FAKE) == EUNSUPPORTED
    optional = {"fwd": (2, 3, 5), "bwd": (3, 5, 9), "step": (2,)}    # (bwd: i and di go together)
    for which, n in (("fwd", 7), ("bwd", 11), ("step", 5)):
        for i in range(n):
            assert _rc(which, _rec(), ptrs={i: FAKE + 8}) == EINVAL, (which, i)
            if i not in optional[which]:
                assert _rc(which, _rec(), ptrs={i: None}) == EINVAL, (which, i)
    for which in ("fwd", "bwd"):
        assert _rc(which, _rec(), ws_bytes=64) == EWORKSPACE
    assert g2.lib().gdr2_gatedrec_workspace_bytes(ctypes.byref(_rec()), 0, 0, None) == EINVAL


def test_recurrence_workspace_grows_with_the_call():
    fwd, bwd = (g2.gdr2_gatedrec_workspace_bytes(_rec(), 0, b) for b in (0, 1))
    assert 0 < fwd <= bwd
    assert g2.gdr2_gatedrec_workspace_bytes(_rec(T=65536), 0, 1) > bwd
    assert g2.gdr2_gatedrec_workspace_bytes(_rec(B=1), 7, 1) > 0
    with pytest.raises(g2.Gdr2Error):
        g2.gdr2_gatedrec_workspace_bytes(_rec(D=0), 0, 0)


# ------------------------------------------------------------------ gated feed-forward block
def _ff(**kw):
    return g2.Gdr2Gatedff(**{**dict(rows=100, D=64, F=176, dtype=g2.GDR2_BF16, act=g2.GDR2_ACT_SILU), **kw})


def _fc(which, prob, ptrs=None, ws_bytes=BIG):
    """fwd: x Wg Wu Wd y ws; bwd: x Wg Wu Wd dy dx dWg dWu dWd ws"""
    p = [FAKE] * {"fwd": 6, "bwd": 10}[which]
    for i, x in (ptrs or {}).items():
        p[i] = x
    return getattr(g2.lib(), "gdr2_gatedff_" + which)(ctypes.byref(prob), *p, ws_bytes, 0, None)


@pytest.mark.parametrize("which", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), EINVAL), (dict(D=0), EINVAL), (dict(F=-8), EINVAL), (dict(dtype=5), EINVAL), (dict(act=2), EINVAL),
    (dict(D=68), EUNSUPPORTED), (dict(F=4), EUNSUPPORTED), (dict(D=65544), EUNSUPPORTED),
    (dict(rows=(1 << 24) + 1), EUNSUPPORTED), (dict(rows=1 << 24, F=4096), EUNSUPPORTED)])
def test_feed_forward_problem_checks(which, kw, code):
    assert _fc(which, _ff(**kw)) == code
    n = ctypes.c_size_t(0)
    assert g2.lib().gdr2_gatedff_workspace_bytes(ctypes.byref(_ff(**kw)), 1, ctypes.byref(n)) == code


def test_feed_forward_argument_checks():
    for which, n in (("fwd", 6), ("bwd", 10)):
        for i in range(n):
            assert _fc(which, _ff(), ptrs={i: FAKE + 8}) == EINVAL, (which, i)
            if (which, i) != ("bwd", 5):  # dx alone may be left out
                assert _fc(which, _ff(), ptrs={i: None}) == EINVAL, (which, i)
        assert _fc(which, _ff(), ws_bytes=64) == EWORKSPACE
    assert _fc("bwd", _ff(), ptrs={5: None, 6: None, 7: None, 8: None}) == EINVAL
    assert _fc("fwd", _ff(rows=0), ptrs={0: None, 4: None}) == OK    # nothing to do, nothing launched
    assert g2.lib().gdr2_gatedff_workspace_bytes(ctypes.byref(_ff()), 0, None) == EINVAL
    fwd, bwd = (g2.gdr2_gatedff_workspace_bytes(_ff(), b) for b in (0, 1))
    assert 0 < fwd <= bwd < g2.gdr2_gatedff_workspace_bytes(_ff(rows=1000), 1)


# ------------------------------------------------------------------ dropout
def _drop(**kw):
    return g2.Gdr2Dropout(**{**dict(n=1000, p=0.1, seed=1, offset=2, dtype=g2.GDR2_BF16, stream_dtype=g2.GDR2_FP32), **kw})


def _dc(prob, fwd=None, bwd=None):
    f = dict(more=None, x=FAKE, r=FAKE, y=FAKE, **{}) | (fwd or {})
    b = dict(more=None, dy=FAKE, dx=FAKE) | (bwd or {})
    return (g2.lib().gdr2_dropout_fwd(ctypes.byref(prob), *f.values(), None),
            g2.lib().gdr2_dropout_bwd(ctypes.byref(prob), *b.values(), None))


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), EINVAL), (dict(p=-0.1), EINVAL), (dict(p=1.0), EINVAL), (dict(p=float("nan")), EINVAL),
    (dict(dtype=2), EINVAL), (dict(dtype=g2.GDR2_FP32, stream_dtype=g2.GDR2_BF16), EINVAL), (dict(stream_dtype=9), EINVAL),
    (dict(n=(1 << 40) + 1), EUNSUPPORTED), (dict(n=0), OK)])
def test_dropout_problem_checks(kw, code):
    assert _dc(_drop(**kw)) == (code, code)


def test_dropout_argument_checks():
    for n in ("x", "y"):
        assert _dc(_drop(), fwd={n: None})[0] == EINVAL, n
    for n in ("x", "r", "y", "more"):
        assert _dc(_drop(), fwd={n: FAKE + 4})[0] == EINVAL, n
    for n in ("dy", "dx"):
        assert _dc(_drop(), bwd={n: None})[1] == EINVAL, n
    for n in ("dy", "dx", "more"):
        assert _dc(_drop(), bwd={n: FAKE + 4})[1] == EINVAL, n


# ------------------------------------------------------------------ the binding
def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    x, w, wd = torch.zeros((1, 4, 8)), torch.zeros((16, 8)), torch.zeros((8, 16))
    for call in (lambda: g2.gdr2_gatedrec_fwd(x, x), lambda: g2.gdr2_gatedrec_bwd(x, x, None, None, x),
                 lambda: g2.gdr2_gatedrec_step(x, x, None, torch.zeros((1, 8))), lambda: g2.gdr2_gatedrec_fwd(x[0], x[0]),
                 lambda: g2.gdr2_gatedff_fwd(x, w, w, wd), lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x),
                 lambda: g2.gdr2_gatedff_fwd(x, w[0], w, wd), lambda: g2.gdr2_gatedff_fwd(x, w, w, wd, act="relu"),
                 lambda: g2.gdr2_dropout_fwd(x, 0.1, 1), lambda: g2.gdr2_dropout_bwd(x, 0.1, 1)):
        with pytest.raises(ValueError):
            call()
    h = x.to(torch.float16)
    for call in (lambda: g2.gdr2_gatedrec_fwd(h, x), lambda: g2.gdr2_gatedff_fwd(h, w, w, wd),
                 lambda: g2.gdr2_dropout_fwd(h, 0.1, 1), lambda: g2.gdr2_dropout_bwd(h, 0.1, 1)):
        with pytest.raises(TypeError):
            call()
