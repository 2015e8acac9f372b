"""The gated feed-forward block on the GPU at sizes that tests/test_gpu_gatedff.py does not have: its largest launches, the
widest rows.  References in 64 bits on the GPU; the tolerances are those of that file, for its reasons."""

import pytest

from tests.test_gpu_gatedff import TOL

pytestmark = pytest.mark.gpu


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


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
