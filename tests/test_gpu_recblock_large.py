"""The recurrence, the feed-forward block and dropout past 32-bit offsets: what lies behind them agrees with
calls on that part alone."""

import numpy as np
import pytest

from oracle.dropout import dropout_keep

pytestmark = pytest.mark.gpu


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def test_recurrence():
    """2.2e9 elements: a long packed batch whose last sequence is compared with a call of its own.  The same tokens
    fall into other tiles there: bf16 outputs are off by the rounding of a few, fp32 ones by 1e-6."""
    import torch
    import paper_2605_22791_amd as g2
    T, D, last = (1 << 20) + 333, 2048, 1500
    _case(f"recurrence of {T} x {D}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, T, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    do = torch.randn((1, T, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    g = -torch.rand((1, T, D), generator=gen, device="cuda")
    h0 = torch.randn((2, D), generator=gen, device="cuda")
    cu = torch.tensor([0, T - last, T], dtype=torch.int32, device="cuda")
    o, h = g2.gdr2_gatedrec_fwd(x, g, None, h0, cu_seqlens=cu, normalize=True)
    d = g2.gdr2_gatedrec_bwd(x, g, None, h0, do, cu_seqlens=cu, normalize=True)
    part = lambda t: t[:, T - last:].contiguous()  # noqa: E731
    o2, h2 = g2.gdr2_gatedrec_fwd(part(x), part(g), None, h0[1:], normalize=True)
    d2 = g2.gdr2_gatedrec_bwd(part(x), part(g), None, h0[1:], part(do), normalize=True)
    assert _rel(part(o), o2) < 2e-4 and _rel(h[1:], h2) < 1e-6
    assert _rel(part(d["dx"]), d2["dx"]) < 2e-4 and _rel(part(d["dlog_decay"]), d2["dlog_decay"]) < 1e-6
    assert _rel(d["dh0"][1:], d2["dh0"]) < 1e-6


def test_feed_forward():
    """2.2e9 hidden values: the last rows' outputs against a call on them, and weights' gradients where only they
    have one.  Both calls round the same values, in other tiles: far below the bf16 bound of 4e-3."""
    import torch
    import paper_2605_22791_amd as g2
    rows, D, F, last = (1 << 20) + 77, 64, 2056, 300
    _case(f"feed-forward of {rows} x {D} x {F}")
    gen = torch.Generator(device="cuda").manual_seed(2)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    x, wg, wu, wd, dy = f(rows, D), f(F, D) * D ** -0.5, f(F, D) * D ** -0.5, f(D, F) * F ** -0.5, f(rows, D)
    dy[:-last] = 0
    y = g2.gdr2_gatedff_fwd(x, wg, wu, wd)
    d = g2.gdr2_gatedff_bwd(x, wg, wu, wd, dy)
    y2 = g2.gdr2_gatedff_fwd(x[-last:], wg, wu, wd)
    d2 = g2.gdr2_gatedff_bwd(x[-last:], wg, wu, wd, dy[-last:])
    assert _rel(y[-last:], y2) < 1e-3 and _rel(d["dx"][-last:], d2["dx"]) < 1e-3
    assert bool((d["dx"][:-last] == 0).all())
    for n in ("dw_gate", "dw_up", "dw_down"):
        assert _rel(d[n], d2[n]) < 1e-3, n


def test_dropout():
    """More elements than a launch has threads for at eight each."""
    import torch
    import paper_2605_22791_amd as g2
    n, p, seed = (1 << 32) + (1 << 23) + 5, 0.3, 77
    _case(f"dropout of {n}")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = g2.gdr2_dropout_fwd(x, p, seed)
    for first in (0, (1 << 32) - 64, (1 << 32) + (1 << 22), n - 101):
        keep = dropout_keep(101, p, seed, 0, first=first)
        assert np.array_equal(y[first:first + 101].float().cpu().numpy() != 0, keep), first
    kept = float(torch.count_nonzero(y[:1 << 31]) + torch.count_nonzero(y[1 << 31:])) / n
    assert abs(kept - 0.7) < 5 * (0.21 / n) ** 0.5
