"""The gated feed-forward block on the GPU at sizes that tests/test_gpu_gatedff.py does not have: every tile that a
product may take, whole and cut, the widest rows, the largest launches.  References in 64 bits on the GPU.

Tolerances are those of that file: bf16 for its reasons; fp32 sums have up to 11056 products here (dx, 2 F), 105 * 2^-24 =
6.3e-6 if the steps' roundings fall differently, beside 29 * 2^-24 = 1.8e-6 of the sums of 864 before them: 6.6e-6 together,
below 8e-6."""

import ctypes

import pytest

from tests.test_gpu_gatedff import TOL, _run

pytestmark = pytest.mark.gpu

# rows, D, F, type, activation: between them each of the five products in each of its tiles, whole and cut along the
# sum (tests/test_gatedff_plan.py holds them against the plan), most with partial tiles at every end
SHAPES = [(8200, 2048, 5504, "bf16", "silu"), (1000, 2048, 5504, "bf16", "silu"), (2507, 1656, 1816, "bf16", "gelu"),
          (3244, 1352, 984, "bf16", "silu"), (5095, 808, 3288, "bf16", "gelu"), (259, 6600, 6000, "bf16", "silu"),
          (70, 616, 72, "bf16", "silu"), (50, 136, 65528, "bf16", "gelu"), (70, 65528, 72, "bf16", "silu"),
          (777, 520, 1368, "fp32", "gelu"), (4000, 1024, 2816, "fp32", "silu"), (3517, 3000, 736, "fp32", "gelu"),
          (1096, 72, 5528, "fp32", "silu"), (72, 864, 5496, "fp32", "gelu")]


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("rows,D,F,dtype,act", SHAPES)
def test_every_tile(rows, D, F, dtype, act):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(rows + D)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    t = {"x": f(rows, D), "w_gate": f(F, D) * D ** -0.5, "w_up": f(F, D) * D ** -0.5, "w_down": f(D, F) * F ** -0.5}
    t = {n: x.to(dt) for n, x in t.items()}
    dy = f(rows, D).to(dt)
    p = {n: x.double().requires_grad_(True) for n, x in t.items()}
    a = getattr(torch.nn.functional, act)(p["x"] @ p["w_gate"].T)
    y = (a * (p["x"] @ p["w_up"].T)) @ p["w_down"].T
    y.backward(dy.double())
    for saved in (False, True):
        _case(f"rows {rows} D {D} F {F} {dtype} {act} saved {saved}")
        got = _run(t, dy, dtype, act, saved)
        for n, want in {"y": y.detach(), **{"d" + m: v.grad for m, v in p.items()}}.items():
            e = _rel(got[n], want)
            print(f"{n} {e:.1e}", end="  ", flush=True)
            assert e < TOL[dtype], (n, e)


@pytest.mark.parametrize("rows,D,F,dtype,act", [SHAPES[k] for k in (1, 2, 3, 4, 5, 9, 11, 13)])
def test_bits_guards_and_a_row_of_nan(rows, D, F, dtype, act):
    """The same bits again; nothing beside the outputs is written; one row's values stay out of the others'."""
    import torch
    import paper_2605_22791_amd as g2
    _case(f"bits, guards, NaN: rows {rows} D {D} F {F} {dtype}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(rows)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)  # noqa: E731
    t = {"x": f(rows, D), "w_gate": f(F, D) * D ** -0.5, "w_up": f(F, D) * D ** -0.5, "w_down": f(D, F) * F ** -0.5}
    dy = f(rows, D)
    want = _run(t, dy, dtype, act, True)

    def guarded(like):
        big = torch.full((like.numel() + 1024,), float("nan"), dtype=dt, device="cuda")
        return big, big[512:512 + like.numel()].view(like.shape)

    out = {m: guarded(v) for m, v in want.items()}
    p = g2.Gdr2Gatedff(rows, D, F, g2.GDR2_BF16 if dtype == "bf16" else g2.GDR2_FP32,
                       g2.GDR2_ACT_SILU if act == "silu" else g2.GDR2_ACT_GELU)
    need = g2.gdr2_gatedff_workspace_bytes(p, 1)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    ws = room[2048:2048 + need]
    g2.gdr2_gatedff_fwd(*t.values(), act=act, y=out["y"][1], ws=ws, save=True)
    g2.gdr2_gatedff_bwd(*t.values(), dy, act=act, ws=ws, saved=True, grads={m: v[1] for m, v in out.items() if m != "y"})
    for m, (big, v) in out.items():
        assert torch.equal(v, want[m]), m
        assert torch.isnan(big[:512]).all() and torch.isnan(big[-512:]).all(), m
    assert bool((room[:2048] == 0xA5).all()) and bool((room[-2048:] == 0xA5).all())
    at = rows - 1 - rows // 3
    t["x"][at] = float("nan")
    got = _run(t, dy, dtype, act, True)
    rest = torch.arange(rows, device="cuda") != at
    for m in ("y", "dx"):
        assert torch.equal(got[m][rest], want[m][rest]) and bool(torch.isnan(got[m][at]).all()), m


def test_no_rows_through_the_c_abi():
    """The binding clears the gradients of an empty batch itself; the library does too."""
    import torch
    import paper_2605_22791_amd as g2
    for code, dt in ((g2.GDR2_BF16, torch.bfloat16), (g2.GDR2_FP32, torch.float32)):
        _case(f"no rows, {dt}")
        p = g2.Gdr2Gatedff(0, 72, 200, code, g2.GDR2_ACT_SILU)
        w = [torch.ones(s, dtype=dt, device="cuda") for s in ((200, 72), (200, 72), (72, 200))]
        g = [torch.full_like(x, 7.0) for x in w]
        ws = torch.empty(g2.gdr2_gatedff_workspace_bytes(p, 1), dtype=torch.uint8, device="cuda")
        at = lambda ts: [x.data_ptr() for x in ts]  # noqa: E731
        st = g2.lib().gdr2_gatedff_bwd(ctypes.byref(p), None, *at(w), None, None, *at(g), ws.data_ptr(), ws.numel(), 0,
                                       torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == g2.GDR2_OK and all(bool((x == 0).all()) for x in g)


def test_a_launch_of_2_35_values():
    """fp32, 2^24 rows of 8, 2056 hidden channels (h: 138 GB): in 64 x 64 tiles, 32 columns of g and u each, more
    threads than a launch has."""
    import torch
    import paper_2605_22791_amd as g2
    rows, D, F = 1 << 24, 8, 2056
    _case(f"feed-forward of {rows} x {D} x {F} fp32")
    gen = torch.Generator(device="cuda").manual_seed(3)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, wg, wu, wd = f(rows, D), f(F, D) * D ** -0.5, f(F, D) * D ** -0.5, f(D, F) * F ** -0.5
    y = g2.gdr2_gatedff_fwd(x, wg, wu, wd)
    for a in (0, rows // 2 - 700, rows - 1000):
        part = x[a:a + 1000].double()
        want = (torch.nn.functional.silu(part @ wg.double().T) * (part @ wu.double().T)) @ wd.double().T
        e = _rel(y[a:a + 1000], want)
        print(f"rows from {a} {e:.1e}", end="  ", flush=True)
        assert e < TOL["fp32"], a
    del x, y
    torch.cuda.empty_cache()
