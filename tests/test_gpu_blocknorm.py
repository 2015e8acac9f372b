"""GPU parity of the block norms against the fp64 oracle.

Tolerances (rel-L2): a bf16 output is the rounding of an fp32 result, 2e-3 or 1.1 times what
rounding the oracle's values costs where the tensor is small; an fp32 output is a few
operations and sums over a row, 2e-6; the weights' gradients sum the rows' products, 5e-6."""

import numpy as np
import pytest

from oracle.blocknorm import blocknorm_bwd, blocknorm_fwd
from paper_2605_22791_amd.inputs import bf16_round
from tests.helpers import rel_l2

pytestmark = pytest.mark.gpu

NAMES = dict(y="dy", w_post="dw_post", z="dgate", x="dx", c="dres_scale", w_pre="dw_pre")


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _problem(shape, parts, dtype, stream, seed):
    r = np.random.default_rng(seed)
    rnd = {"bf16": bf16_round, "fp32": lambda x: x}
    f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    D = shape[-1]
    p = dict.fromkeys(NAMES)
    p["y"] = rnd[dtype](f(*shape))
    if "p" in parts:
        p["w_post"] = 1 + np.float32(0.2) * f(D)
    if "g" in parts:
        p["z"] = rnd[dtype](2 * f(*shape))
    if "x" in parts:
        p["x"] = rnd[stream](2 * f(*shape))
    if "c" in parts:
        p["c"] = np.float32(0.5) * f(D)
    if "n" in parts:
        p["w_pre"] = 1 + np.float32(0.2) * f(D)
    dh = rnd[stream if "x" in parts else dtype](f(*shape))
    return p, dh, rnd[dtype](f(*shape)) if "n" in parts else None


def _dev(x, dtype):
    import torch
    if x is None:
        return None
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _close(name, got, want, tol):
    import torch
    assert tuple(got.shape) == want.shape, name
    if got.dtype == torch.bfloat16:
        tol = max(2e-3, 1.1 * rel_l2(bf16_round(want.astype(np.float32)), want))
    e = rel_l2(got.detach().float().cpu().numpy(), want)
    print(f"{name} {e:.1e}", end="  ", flush=True)
    assert e < tol, (name, e, tol)


def _check(shape, parts, dtype, stream, seed=0, eps=1e-6, want_dh=True, edit=None):
    import paper_2605_22791_amd as g2
    p, dh, dn = _problem(shape, parts, dtype, stream, seed)
    if edit:
        edit(p)
    if not want_dh:
        dh = None
    hs = stream if "x" in parts else dtype
    t = dict(w_post=_dev(p["w_post"], "fp32"), gate=_dev(p["z"], dtype), x=_dev(p["x"], stream), res_scale=_dev(p["c"], "fp32"),
             w_pre=_dev(p["w_pre"], "fp32"))
    y = _dev(p["y"], dtype)
    h, n = g2.gdr2_blocknorm_fwd(y, **t, eps=eps)
    d = g2.gdr2_blocknorm_bwd(y, _dev(dh, hs), _dev(dn, dtype), **t, eps=eps)
    hh, nn = blocknorm_fwd(**p, eps=eps)
    dd = blocknorm_bwd(dh=dh, dn=dn, **p, eps=eps)
    _close("h", h, hh, 2e-6)
    assert (n is None) == (nn is None)
    if nn is not None:
        _close("n", n, nn, 2e-6)
    for m, v in dd.items():
        assert (d[m] is None) == (v is None), m
        if v is not None:
            _close(m, d[m], v, 5e-6 if m[:2] == "dw" or m == "dres_scale" else 2e-6)


TYPES = [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")]


@pytest.mark.parametrize("D", [1, 3, 8, 63, 64, 65, 128, 200, 256, 511, 512, 520, 1000, 1024, 1155, 2048, 2056, 4096, 4100,
                               5000, 8191, 8192])
def test_widths(D):
    _case(f"width {D}")
    for dtype, stream in TYPES:
        _check((37, D), "pgxcn", dtype, stream, seed=D)


@pytest.mark.parametrize("parts", ["", "p", "g", "c", "x", "n", "pg", "pgc", "xn", "pxn", "xcn", "pgx", "pgxn", "gxcn", "pgn"])
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_parts(parts, dtype, stream):
    _case(f"parts '{parts}' {dtype} {stream}")
    _check((3, 17, 128), parts, dtype, stream, seed=len(parts))
    _check((2, 9, 1030), parts, dtype, stream, seed=len(parts) + 1)


@pytest.mark.parametrize("rows", [1, 2, 16, 31, 255, 257, 5000, 40000])
@pytest.mark.parametrize("D", [128, 320])
def test_rows(rows, D):
    _case(f"rows {rows} width {D}")
    _check((rows, D), "pgxcn", "bf16", "fp32", seed=rows)


def test_no_gradient_into_h():
    _case("dh None")
    _check((19, 256), "pgxcn", "bf16", "fp32", want_dh=False)
    _check((19, 256), "xn", "fp32", "fp32", want_dh=False)


def test_rows_of_zeros_and_large_values():
    """A row of zeros has the norm eps^(1/2); gates far out have a logistic of zero or one."""
    _case("zeros, large values, far gates")

    def edit(p):
        p["y"][3] = 0.0
        p["y"][5] *= 1e15
        p["x"][3] = 0.0
        p["z"][:, :4] = [200.0, -200.0, 0.0, -80.0]

    import paper_2605_22791_amd as g2
    p, dh, dn = _problem((9, 128), "pgxcn", "fp32", "fp32", 3)
    edit(p)
    t = dict(w_post=_dev(p["w_post"], "fp32"), gate=_dev(p["z"], "fp32"), x=_dev(p["x"], "fp32"),
             res_scale=_dev(p["c"], "fp32"), w_pre=_dev(p["w_pre"], "fp32"))
    y = _dev(p["y"], "fp32")
    h, n = g2.gdr2_blocknorm_fwd(y, **t, eps=1e-3)
    d = g2.gdr2_blocknorm_bwd(y, _dev(dh, "fp32"), _dev(dn, "fp32"), **t, eps=1e-3)
    hh, nn = blocknorm_fwd(**p, eps=1e-3)
    dd = blocknorm_bwd(dh=dh, dn=dn, **p, eps=1e-3)
    for name, got, want in [("h", h, hh), ("n", n, nn)] + [(m, d[m], dd[m]) for m in dd]:
        if want.ndim == 2:  # row by row: their sizes differ by 1e15
            for r in range(9):
                assert rel_l2(got[r].cpu().numpy(), want[r]) < 1e-5, (name, r)
        else:
            assert rel_l2(got.cpu().numpy(), want) < 1e-5, name


def test_no_rows():
    import torch
    import paper_2605_22791_amd as g2
    _case("no rows")
    y, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    h, n = g2.gdr2_blocknorm_fwd(y, w_pre=w)
    assert h.shape == n.shape == (0, 64)
    d = g2.gdr2_blocknorm_bwd(y, h, n, w_pre=w, grads={"dw_pre": torch.full((64,), 7.0, device="cuda")})
    assert d["dy"].shape == (0, 64) and bool((d["dw_pre"] == 0).all())


def test_gradient_by_differences():
    """Along random directions, from the fp32 forward (2 h = 2e-2; good to h^2 and 1e-7 / h): 1e-3."""
    import torch
    import paper_2605_22791_amd as g2
    _case("differences of the fp32 forward")
    p, dh, dn = _problem((23, 150), "pgxcn", "fp32", "fp32", 5)
    t = {a: _dev(p[b], "fp32") for a, b in (("y", "y"), ("w_post", "w_post"), ("gate", "z"), ("x", "x"), ("res_scale", "c"),
                                            ("w_pre", "w_pre"))}
    dh, dn = _dev(dh, "fp32"), _dev(dn, "fp32")
    rest = lambda a: {n: v for n, v in a.items() if n != "y"}  # noqa: E731
    d = g2.gdr2_blocknorm_bwd(t["y"], dh, dn, **rest(t), eps=1e-2)

    def loss(a):
        h, n = g2.gdr2_blocknorm_fwd(a["y"], **rest(a), eps=1e-2)
        return float((h.double() * dh.double()).sum() + (n.double() * dn.double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(2)
    for n in t:
        g = d["d" + n]
        e = g / g.norm() + 0.1 * torch.randn(g.shape, generator=gen, device="cuda") / g.numel() ** 0.5
        fd = (loss({**t, n: t[n] + 1e-2 * e}) - loss({**t, n: t[n] - 1e-2 * e})) / 2e-2
        want = float((g.double() * e.double()).sum())
        assert abs(fd - want) < 1e-3 * abs(want), n


def test_guards_bits_and_graph():
    import torch
    import paper_2605_22791_amd as g2
    _case("guards, bits, graph")
    p, dh, dn = _problem((33, 77), "pgxcn", "bf16", "fp32", 6)
    t = dict(w_post=_dev(p["w_post"], "fp32"), gate=_dev(p["z"], "bf16"), x=_dev(p["x"], "fp32"),
             res_scale=_dev(p["c"], "fp32"), w_pre=_dev(p["w_pre"], "fp32"))
    y, dh, dn = _dev(p["y"], "bf16"), _dev(dh, "fp32"), _dev(dn, "bf16")
    h, n = g2.gdr2_blocknorm_fwd(y, **t)
    d = g2.gdr2_blocknorm_bwd(y, dh, dn, **t)

    def guarded(like):
        big = torch.full((like.numel() + 1024,), float("nan"), dtype=like.dtype, device="cuda")
        return big, big[512:512 + like.numel()].view(like.shape)

    hb, nb = guarded(h), guarded(n)
    db = {m: guarded(v) for m, v in d.items()}
    graph = torch.cuda.CUDAGraph()
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(graph):
        g2.gdr2_blocknorm_fwd(y, **t, h=hb[1], n=nb[1])
        g2.gdr2_blocknorm_bwd(y, dh, dn, **t, grads={m: v[1] for m, v in db.items()}, ws=ws)
    for _ in range(3):
        hb[1].zero_()
        db["dw_pre"][1].zero_()
        graph.replay()
        g2.gdr2_blocknorm_fwd(y, **t)
        torch.cuda.synchronize()
        assert torch.equal(hb[1], h) and torch.equal(nb[1], n)
        assert all(torch.equal(db[m][1], d[m]) for m in d)
    for big, _ in [hb, nb, *db.values()]:
        assert torch.isnan(big[:512]).all() and torch.isnan(big[-512:]).all()


def test_refusals():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    y = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    bad = [lambda: g2.gdr2_blocknorm_fwd(y, gate=y[:2]), lambda: g2.gdr2_blocknorm_fwd(y, w_post=w[:32].contiguous()),
           lambda: g2.gdr2_blocknorm_fwd(y.t()), lambda: g2.gdr2_blocknorm_fwd(y, w_pre=w.to(torch.bfloat16)),
           lambda: g2.gdr2_blocknorm_fwd(y, n=y), lambda: g2.gdr2_blocknorm_fwd(y, h=y.float()),
           lambda: g2.gdr2_blocknorm_bwd(y, None), lambda: g2.gdr2_blocknorm_bwd(y, y, w_pre=w),
           lambda: g2.gdr2_blocknorm_bwd(y, y, y), lambda: g2.gdr2_blocknorm_bwd(y, y.float()),
           lambda: g2.gdr2_blocknorm_bwd(y, y, grads={"dx": y}),
           lambda: g2.gdr2_blocknorm_bwd(y, y, w_post=w, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        g2.gdr2_blocknorm_fwd(y.float(), x=y)
    with pytest.raises(g2.Gdr2Error):
        g2.gdr2_blocknorm_fwd(torch.zeros((2, 8200), device="cuda"))
