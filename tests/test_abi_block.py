"""C-ABI and binding checks of linear attention and the block norms that need no GPU.

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
BIG = 1 << 45


@pytest.mark.parametrize("header,names", [
    ("gdr2_linattn.h", ["gdr2_linattn_bwd", "gdr2_linattn_fwd", "gdr2_linattn_step", "gdr2_linattn_workspace_bytes"]),
    ("gdr2_blocknorm.h", ["gdr2_blocknorm_bwd", "gdr2_blocknorm_fwd", "gdr2_blocknorm_workspace_bytes"])])
def test_headers_declare_what_the_library_exports(header, names):
    text = open(os.path.join(ROOT, "include", header)).read()
    assert sorted(set(re.findall(r"^gdr2_status\s+(gdr2_\w+)\s*\(", text, re.M))) == names
    assert all(hasattr(g2.lib(), n) and hasattr(g2, n) for n in names)


def _prob(**kw):
    d = dict(B=2, T=128, H=4, Dk=128, Dv=128, chunk=64, scale=0.1, dtype=g2.GDR2_BF16, Hv=0)
    d.update(kw)
    return g2.Gdr2Problem(**d)


def _la(which, prob, decay=0, cu=None, n=0, ptrs=None, ws_bytes=BIG):
    """fwd: q k v g S0 o ST ws; bwd: q k v g S0 dout dST dq dk dv dg dS0 ws; step: q k v g S o"""
    p = {"fwd": [FAKE] * 4 + [None, FAKE, None, FAKE], "bwd": [FAKE] * 4 + [None, FAKE, None] + [FAKE] * 4 + [None, FAKE],
         "step": [FAKE] * 6}[which]
    for i, x in (ptrs or {}).items():
        p[i] = x
    tail = [] if which == "step" else [ws_bytes, 0]
    return getattr(g2.lib(), "gdr2_linattn_" + which)(ctypes.byref(prob), decay, cu, n, *p, *tail, None)


@pytest.mark.parametrize("which", ["fwd", "bwd", "step"])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), g2.GDR2_EINVAL), (dict(T=-1), g2.GDR2_EINVAL), (dict(H=0), g2.GDR2_EINVAL), (dict(Dk=0), g2.GDR2_EINVAL),
    (dict(scale=float("nan")), g2.GDR2_EINVAL), (dict(dtype=7), g2.GDR2_EINVAL), (dict(Hv=6), g2.GDR2_EINVAL),
    (dict(Dk=96), g2.GDR2_EUNSUPPORTED), (dict(Dv=256), g2.GDR2_EUNSUPPORTED),
    (dict(B=1 << 20, T=1 << 16), g2.GDR2_EUNSUPPORTED)])
def test_linattn_problem_checks(which, kw, code):
    assert _la(which, _prob(**kw)) == code
    n = ctypes.c_size_t(0)
    assert g2.lib().gdr2_linattn_workspace_bytes(ctypes.byref(_prob(**kw)), 0, 0, ctypes.byref(n)) == code


def test_linattn_argument_checks():
    for which in ("fwd", "bwd"):
        assert _la(which, _prob(chunk=32)) == g2.GDR2_EUNSUPPORTED
        assert _la(which, _prob(), ws_bytes=64) == g2.GDR2_EWORKSPACE
    for which in ("fwd", "bwd", "step"):
        assert _la(which, _prob(), decay=2) == g2.GDR2_EINVAL
        assert _la(which, _prob(), n=-1) == g2.GDR2_EINVAL
        assert _la(which, _prob(), n=3, cu=FAKE) == g2.GDR2_EINVAL                # B != 1
        assert _la(which, _prob(B=1), n=3, cu=None) == g2.GDR2_EINVAL
        assert _la(which, _prob(B=1), n=3, cu=FAKE + 2) == g2.GDR2_EINVAL
        assert _la(which, _prob(B=1), n=(1 << 24) + 1, cu=FAKE) == g2.GDR2_EUNSUPPORTED
    optional = {"fwd": (4, 6), "bwd": (4, 6, 11), "step": ()}
    for which, n in (("fwd", 8), ("bwd", 13), ("step", 6)):
        for i in range(n):
            assert _la(which, _prob(), ptrs={i: FAKE + 8}) == g2.GDR2_EINVAL, (which, i)
            if i not in optional[which]:
                assert _la(which, _prob(), ptrs={i: None}) == g2.GDR2_EINVAL, (which, i)
    assert g2.lib().gdr2_linattn_workspace_bytes(ctypes.byref(_prob()), 0, 0, None) == g2.GDR2_EINVAL


def test_linattn_workspace_grows_with_the_call():
    p = _prob()
    fwd, bwd = (g2.gdr2_linattn_workspace_bytes(p, 0, b) for b in (0, 1))
    assert 0 < fwd <= bwd
    assert g2.gdr2_linattn_workspace_bytes(_prob(T=4096), 0, 1) > bwd
    assert g2.gdr2_linattn_workspace_bytes(_prob(B=1), 7, 1) > 0
    with pytest.raises(g2.Gdr2Error):
        g2.gdr2_linattn_workspace_bytes(_prob(Dk=32), 0, 0)


def _norm(**kw):
    d = dict(rows=8, D=128, dtype=g2.GDR2_BF16, stream_dtype=g2.GDR2_FP32, eps=1e-6)
    d.update(kw)
    return g2.Gdr2Blocknorm(**d)


def _nf(p, **kw):
    a = dict(y=FAKE, w_post=FAKE, z=FAKE, x=FAKE, c=FAKE, w_pre=FAKE, h=FAKE, n=FAKE)
    a.update(kw)
    return g2.lib().gdr2_blocknorm_fwd(ctypes.byref(p) if p is not None else None, *a.values(), None)


def _nb(p, ws_bytes=BIG, **kw):
    a = dict(y=FAKE, w_post=FAKE, z=FAKE, x=FAKE, c=FAKE, w_pre=FAKE, dh=FAKE, dn=FAKE, dy=FAKE, dw_post=FAKE, dz=FAKE,
             dx=FAKE, dc=FAKE, dw_pre=FAKE, ws=FAKE)
    a.update(kw)
    return g2.lib().gdr2_blocknorm_bwd(ctypes.byref(p), *a.values(), ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), g2.GDR2_EINVAL), (dict(D=0), g2.GDR2_EINVAL), (dict(D=8193), g2.GDR2_EUNSUPPORTED),
    (dict(eps=-1.0), g2.GDR2_EINVAL), (dict(eps=float("inf")), g2.GDR2_EINVAL), (dict(dtype=3), g2.GDR2_EINVAL),
    (dict(dtype=g2.GDR2_FP32, stream_dtype=g2.GDR2_BF16), g2.GDR2_EINVAL), (dict(rows=1 << 40), g2.GDR2_EUNSUPPORTED)])
def test_blocknorm_problem_checks(kw, code):
    assert _nf(_norm(**kw)) == code and _nb(_norm(**kw)) == code
    n = ctypes.c_size_t(0)
    assert g2.lib().gdr2_blocknorm_workspace_bytes(ctypes.byref(_norm(**kw)), ctypes.byref(n)) == code


def test_blocknorm_argument_checks():
    p = _norm()
    assert _nf(None) == g2.GDR2_EINVAL and _nf(p, y=None) == g2.GDR2_EINVAL
    assert _nf(p, n=None) == g2.GDR2_EINVAL and _nf(p, w_pre=None) == g2.GDR2_EINVAL
    assert _nf(p, h=None, n=None, w_pre=None) == g2.GDR2_EINVAL
    for name in ("y", "w_post", "z", "x", "c", "w_pre", "h", "n"):
        assert _nf(p, **{name: FAKE + 4}) == g2.GDR2_EINVAL, name
    for name in ("y", "dy", "dn", "w_post", "z", "c", "w_pre", "dw_post", "dz", "dc", "dw_pre", "ws", "x"):
        assert _nb(p, **{name: None}) == g2.GDR2_EINVAL, name
    for name in ("y", "dh", "dx", "ws", "dw_pre"):
        assert _nb(p, **{name: FAKE + 4}) == g2.GDR2_EINVAL, name
    assert _nb(p, dh=None, dn=None, w_pre=None, dw_pre=None) == g2.GDR2_EINVAL
    assert _nb(p, ws_bytes=64) == g2.GDR2_EWORKSPACE
    assert _nf(_norm(rows=0)) == g2.GDR2_OK                                       # nothing to do, nothing launched


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    q = torch.zeros((1, 4, 2, 64))
    v, g = torch.zeros((1, 4, 2, 64)), torch.zeros((1, 4, 2))
    for call in (lambda: g2.gdr2_linattn_fwd(q, q, v, g), lambda: g2.gdr2_linattn_bwd(q, q, v, g, None, v),
                 lambda: g2.gdr2_linattn_step(q, q, v, g, torch.zeros((1, 2, 64, 64))),
                 lambda: g2.gdr2_linattn_fwd(q, q, torch.zeros((1, 4, 3, 64)), g),
                 lambda: g2.gdr2_linattn_fwd(q[0], q[0], v, g),
                 lambda: g2.gdr2_blocknorm_fwd(torch.zeros((4, 8))), lambda: g2.gdr2_blocknorm_bwd(torch.zeros((4, 8)), None)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        g2.gdr2_blocknorm_fwd(torch.zeros((4, 8), dtype=torch.float16))


def test_a_token_of_a_chunk_call_has_at_most_two_to_the_22_values():
    wide = dict(H=1 << 15, Hv=(1 << 15) + (1 << 15), T=64, B=1)  # 2^16 value heads of 128: 2^23 values
    for which in ("fwd", "bwd"):
        assert _la(which, _prob(**wide)) == g2.GDR2_EUNSUPPORTED
    n = ctypes.c_size_t(0)
    assert g2.lib().gdr2_linattn_workspace_bytes(ctypes.byref(_prob(**wide)), 0, 1, ctypes.byref(n)) == g2.GDR2_EUNSUPPORTED
    # at the bound itself the call is counted
    assert g2.lib().gdr2_linattn_workspace_bytes(ctypes.byref(_prob(H=1 << 15, T=64, B=1)), 0, 1, ctypes.byref(n)) == g2.GDR2_OK
    assert n.value > 0
