"""The gated feed-forward block on the GPU against 64-bit references.

Tolerances (rel-L2).  bf16: every output is rounded once, and so is one factor of its last product (h,
or the gradients at g and u); a rounding is off by 2^-8 at most, evenly spread 2^-8 / sqrt 3 = 2.3e-3
in the mean square, two of them that fall differently 3.2e-3; 4e-3 allows for the sums of small
tensors.  fp32: sums of up to 4096 products and two such sums behind one another, each step good to
2^-24: 64 * 2^-24 = 3.8e-6 if the steps' roundings fall differently; 8e-6."""

import numpy as np
import pytest

from oracle.gatedff import gatedff_bwd, gatedff_fwd
from paper_2605_22791_amd.inputs import bf16_round
from tests.helpers import rel_l2

pytestmark = pytest.mark.gpu

TOL = {"bf16": 4e-3, "fp32": 8e-6}
WEIGHTS = ("w_gate", "w_up", "w_down")


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _inputs(rows, D, F, dtype, seed):
    r = np.random.default_rng(seed)
    rnd = bf16_round if dtype == "bf16" else (lambda x: x)
    f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    return dict(x=rnd(f(rows, D)), w_gate=rnd(f(F, D) * np.float32(D ** -0.5)), w_up=rnd(f(F, D) * np.float32(D ** -0.5)),
                w_down=rnd(f(D, F) * np.float32(F ** -0.5))), rnd(f(rows, D))


def _t(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _ws(rows, D, F, dtype, act, bwd=1):
    import torch
    import paper_2605_22791_amd as g2
    p = g2.Gdr2Gatedff(rows, D, F, g2.GDR2_BF16 if dtype == "bf16" else g2.GDR2_FP32,
                       g2.GDR2_ACT_SILU if act == "silu" else g2.GDR2_ACT_GELU)
    return torch.full((g2.gdr2_gatedff_workspace_bytes(p, bwd),), 0xFF, dtype=torch.uint8, device="cuda")


def _run(t, dy, dtype, act, saved):
    import paper_2605_22791_amd as g2
    rows, D = t["x"].shape
    ws = _ws(rows, D, t["w_gate"].shape[0], dtype, act)
    y = g2.gdr2_gatedff_fwd(*t.values(), act=act, ws=ws, save=saved)
    if not saved:
        ws.fill_(0xFF)
    return {"y": y, **g2.gdr2_gatedff_bwd(*t.values(), dy, act=act, ws=ws, saved=saved)}


def _close(name, got, want, dtype):
    assert tuple(got.shape) == want.shape, name
    e = rel_l2(got.float().cpu().numpy(), want)
    print(f"{name} {e:.1e}", end="  ", flush=True)
    assert e < TOL[dtype], (name, e)


def _check(rows, D, F, dtype, act="silu", seed=0, saved=False, edit=None):
    p, dy = _inputs(rows, D, F, dtype, seed)
    if edit:
        edit(p)
    got = _run({n: _t(x, dtype) for n, x in p.items()}, _t(dy, dtype), dtype, act, saved)
    q = (p["x"], p["w_gate"], p["w_up"], p["w_down"])
    want = {"y": gatedff_fwd(*q, act=act), **gatedff_bwd(*q, dy, act=act)}
    for n in want:
        _close(n, got[n], want[n], dtype)


@pytest.mark.parametrize("rows", [1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows(rows, dtype):
    _case(f"rows {rows} {dtype}")
    _check(rows, 128, 352, dtype, seed=rows)
    _check(rows, 72, 200, dtype, seed=rows + 1, saved=True)


@pytest.mark.parametrize("D,F", [(8, 8), (8, 136), (16, 24), (40, 8), (56, 64), (64, 64), (120, 264), (128, 128), (136, 392),
                                 (248, 504), (256, 256), (264, 520), (320, 1000), (512, 1376), (1032, 2056)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_widths(D, F, dtype):
    _case(f"D {D} F {F} {dtype}")
    for rows in (1, 7, 40, 150):
        _check(rows, D, F, dtype, act="gelu", seed=D + rows, saved=rows % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("saved", [False, True])
def test_options(dtype, act, saved):
    _case(f"{act} {dtype} saved {saved}")
    _check(333, 192, 512, dtype, act=act, seed=5, saved=saved)

    def far(p):  # g of up to some 40: the activation's ends
        p["w_gate"] *= 16
    _check(333, 192, 512, dtype, act=act, seed=6, saved=saved, edit=far)


def test_larger_against_torch_in_64_bits():
    """Enough tiles for every CU, partial ones at the ends; few rows of wide weights; the reference on the GPU in
    64 bits."""
    import torch
    for rows, D, F, act in ((2100, 1048, 2840, "silu"), (4096, 1024, 2816, "gelu"), (700, 2048, 5504, "silu"),
                              (4100, 2048, 5504, "gelu"), (32, 2048, 6000, "silu"), (33, 2048, 6000, "silu"), (64, 2048, 6000, "gelu")):
        _case(f"rows {rows} D {D} F {F}")
        gen = torch.Generator(device="cuda").manual_seed(rows)
        f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        t = {"x": f(rows, D), "w_gate": f(F, D) * D ** -0.5, "w_up": f(F, D) * D ** -0.5, "w_down": f(D, F) * F ** -0.5}
        t = {n: x.to(torch.bfloat16) for n, x in t.items()}
        dy = f(rows, D).to(torch.bfloat16)
        p = {n: x.double().requires_grad_(True) for n, x in t.items()}
        a = getattr(torch.nn.functional, act)(p["x"] @ p["w_gate"].T)
        y = (a * (p["x"] @ p["w_up"].T)) @ p["w_down"].T
        y.backward(dy.double())
        for saved in (False, True):
            got = _run(t, dy, "bf16", act, saved)
            for n, want in {"y": y.detach(), **{"d" + m: v.grad for m, v in p.items()}}.items():
                e = float((got[n].double() - want).norm() / want.norm())
                print(f"{n} {e:.1e}", end="  ", flush=True)
                assert e < TOL["bf16"], (n, e)


def test_no_rows():
    import torch
    import paper_2605_22791_amd as g2
    _case("no rows")
    x, w, wd = (torch.zeros(s, device="cuda") for s in ((0, 16), (24, 16), (16, 24)))
    assert g2.gdr2_gatedff_fwd(x, w, w, wd).shape == (0, 16)
    d = g2.gdr2_gatedff_bwd(x, w, w, wd, x, grads={"dw_up": torch.full((24, 16), 7.0, device="cuda")})
    assert d["dx"].shape == (0, 16) and all(bool((d["d" + n] == 0).all()) for n in WEIGHTS)


def test_only_some_gradients():
    import torch
    import paper_2605_22791_amd as g2
    _case("only some gradients")
    p, dy = _inputs(77, 64, 136, "bf16", 3)
    t, dy = {n: _t(x, "bf16") for n, x in p.items()}, _t(dy, "bf16")
    whole = g2.gdr2_gatedff_bwd(*t.values(), dy)
    a, b = g2.gdr2_gatedff_bwd(*t.values(), dy, want_dw=False), g2.gdr2_gatedff_bwd(*t.values(), dy, want_dx=False)
    assert torch.equal(a["dx"], whole["dx"]) and a["dw_up"] is None and b["dx"] is None
    assert all(torch.equal(b["d" + n], whole["d" + n]) for n in WEIGHTS)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_of_one_row_do_not_reach_another(dtype):
    import torch
    import paper_2605_22791_amd as g2
    _case(f"NaN in one row {dtype}")
    for rows, at in ((5, 4), (200, 130), (200, 0)):
        p, dy = _inputs(rows, 72, 136, dtype, 4)
        t, dy = {n: _t(x, dtype) for n, x in p.items()}, _t(dy, dtype)
        y, dx = g2.gdr2_gatedff_fwd(*t.values()), g2.gdr2_gatedff_bwd(*t.values(), dy)["dx"]
        t["x"][at] = float("nan")
        y2, dx2 = g2.gdr2_gatedff_fwd(*t.values()), g2.gdr2_gatedff_bwd(*t.values(), dy)["dx"]
        rest = torch.arange(rows, device="cuda") != at
        assert torch.equal(y2[rest], y[rest]) and torch.equal(dx2[rest], dx[rest])
        assert bool(torch.isnan(y2[at]).all()) and bool(torch.isnan(dx2[at]).all())


def test_gradient_by_differences():
    """Along the gradient and a random direction, from the fp32 forward (2 h = 2e-2; good to h^2 and 1e-7 / h): 2e-3."""
    import torch
    import paper_2605_22791_amd as g2
    _case("differences of the fp32 forward")
    p, dy = _inputs(23, 40, 72, "fp32", 5)
    t, dy = {n: _t(x, "fp32") for n, x in p.items()}, _t(dy, "fp32")
    d = g2.gdr2_gatedff_bwd(*t.values(), dy)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for n in t:
        g = d["d" + n]
        e = g / g.norm() + 0.1 * torch.randn(g.shape, generator=gen, device="cuda") / g.numel() ** 0.5
        up, down = (float((g2.gdr2_gatedff_fwd(**{**t, n: t[n] + s * e}).double() * dy.double()).sum()) for s in (1e-2, -1e-2))
        want = float((g.double() * e.double()).sum())
        assert abs((up - down) / 2e-2 - want) < 2e-3 * abs(want), n


@pytest.mark.parametrize("rows", [1, 150, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bits_guards_graph_and_streams(rows, dtype):
    import torch
    import paper_2605_22791_amd as g2
    _case(f"bits, guards, graph, streams rows {rows} {dtype}")
    p, dy = _inputs(rows, 136, 264, dtype, 6)
    t, dy = {n: _t(x, dtype) for n, x in p.items()}, _t(dy, dtype)
    want = _run(t, dy, dtype, "silu", False)
    again, kept = _run(t, dy, dtype, "silu", False), _run(t, dy, dtype, "silu", True)
    assert all(torch.equal(want[m], again[m]) for m in want)
    assert all(torch.equal(want[m], kept[m]) for m in want if m != "y")  # (few rows: a forward that keeps nothing sums otherwise)
    _close("y", kept["y"], want["y"].double().cpu().numpy(), dtype)

    def guarded(like):
        big = torch.full((like.numel() + 1024,), float("nan"), dtype=like.dtype, device="cuda")
        return big, big[512:512 + like.numel()].view(like.shape)

    out, ws = {m: guarded(v) for m, v in want.items()}, _ws(rows, 136, 264, dtype, "silu")

    def both():
        g2.gdr2_gatedff_fwd(*t.values(), y=out["y"][1], ws=ws)
        g2.gdr2_gatedff_fwd(*t.values(), ws=ws, save=True)
        g2.gdr2_gatedff_bwd(*t.values(), dy, ws=ws, saved=True, grads={m: v[1] for m, v in out.items() if m != "y"})

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for _, v in out.values():
            v.zero_()
        ws.fill_(0xFF)
        graph.replay()
        g2.gdr2_gatedff_fwd(*t.values())
        torch.cuda.synchronize()
        assert all(torch.equal(out[m][1], want[m]) for m in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, v in out.values():
            v.zero_()
        both()
    side.synchronize()
    assert all(torch.equal(out[m][1], want[m]) for m in want)
    for big, _ in out.values():
        assert torch.isnan(big[:512]).all() and torch.isnan(big[-512:]).all()


def test_refusals():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    x, w, wd = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 16), (24, 16), (16, 24)))
    for f in (lambda: g2.gdr2_gatedff_fwd(x, w, w[:8], wd), lambda: g2.gdr2_gatedff_fwd(x, w, w, w),
              lambda: g2.gdr2_gatedff_fwd(x, w, w.float(), wd), lambda: g2.gdr2_gatedff_fwd(x, w, w, wd, act="tanh"),
              lambda: g2.gdr2_gatedff_fwd(x, w, w, w.t()), lambda: g2.gdr2_gatedff_fwd(x, w, w, wd, y=x.float()),
              lambda: g2.gdr2_gatedff_fwd(x, w, w, wd, save=True), lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, None),
              lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x, saved=True), lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x[:2]),
              lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x, want_dx=False, want_dw=False),
              lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x, want_dx=False, grads={"dx": x}),
              lambda: g2.gdr2_gatedff_bwd(x, w, w, wd, x, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(g2.Gdr2Error):  # widths that 8 does not divide
        g2.gdr2_gatedff_fwd(x[:, :12].contiguous(), w[:, :12].contiguous(), w[:, :12].contiguous(), wd[:12].contiguous())
