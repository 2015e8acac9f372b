"""Dropout with the residual sum on the GPU against the oracle's generator.

Which elements are dropped has to be the oracle's exactly.  Values: an fp32 output is a product by
a rounded 1 / (1 - p) and a sum, three roundings of 2^-24 each: 2e-7 of the largest; a bf16 output is
the rounding of that, 2^-8 and the same."""

import numpy as np
import pytest

from oracle.dropout import dropout_fwd, dropout_keep, words
from paper_2605_22791_amd.inputs import bf16_round

pytestmark = pytest.mark.gpu

TYPES = [("bf16", None), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", None), ("fp32", "fp32")]


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _t(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _draw(n, dtype, seed):
    x = np.random.default_rng(seed).standard_normal(n).astype(np.float32)
    x[x == 0] = 1.0
    return bf16_round(x) if dtype == "bf16" else x


def _close(got, want, size):
    """Element by element, of `size`: the magnitudes that were added."""
    import torch
    tol = 2.0 ** -8 + 2e-7 if got.dtype == torch.bfloat16 else 2e-7
    d = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    assert (d <= tol * size).all(), (d / size).max()


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 31, 257, 2047, 2048, 2049, 5003])
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_sizes_and_types(n, dtype, stream):
    import torch
    import paper_2605_22791_amd as g2
    _case(f"n {n} {dtype} residual {stream}")
    x, r = _draw(n, dtype, n), None if stream is None else _draw(n, stream, n + 1)
    seed, offset = 0xFEDCBA9876543210 + n, (3 << 32) + 5
    y = g2.gdr2_dropout_fwd(_t(x, dtype), 0.3, seed, offset=offset, residual=None if r is None else _t(r, stream))
    assert y.dtype == (torch.bfloat16 if (stream or dtype) == "bf16" else torch.float32)
    _close(y, dropout_fwd(x, 0.3, seed, offset, r), np.abs(x) / 0.7 + (0 if r is None else np.abs(r)))
    dy = _draw(n, stream or dtype, n + 2)
    dx = g2.gdr2_dropout_bwd(_t(dy, stream or dtype), 0.3, seed, offset=offset, dtype=_t(x, dtype).dtype)
    keep = dropout_keep(n, 0.3, seed, offset)
    assert np.array_equal(dx.float().cpu().numpy() != 0, keep)
    _close(dx, np.where(keep, dy.astype(np.float64) / 0.7, 0.0), np.abs(dy) / 0.7)


@pytest.mark.parametrize("p", [0.0, 1e-9, 0.5, 0.999, 1.0 - 2.0 ** -53])
def test_rates(p):
    import torch
    import paper_2605_22791_amd as g2
    _case(f"p {p}")
    n = 4000
    y = g2.gdr2_dropout_fwd(torch.ones(n, device="cuda"), p, 9)
    keep = words(0, n, 9, 0) >= min(round(p * 2 ** 32), 2 ** 32 - 1)
    assert np.array_equal(y.cpu().numpy() != 0, keep)
    if p == 0.0:
        assert bool((y == 1).all())


def test_seeds_offsets_and_a_device_offset():
    import torch
    import paper_2605_22791_amd as g2
    _case("seeds and offsets")
    x = torch.ones(3001, device="cuda")
    mask = lambda s, o: (g2.gdr2_dropout_fwd(x, 0.5, s, offset=o) != 0).cpu().numpy()  # noqa: E731
    for s, o in ((0, 0), (1, 0), (0, 1), (1 << 32, 0), (0, 1 << 32), ((1 << 64) - 1, (1 << 64) - 1), (-1, -1)):
        assert np.array_equal(mask(s, o), dropout_keep(3001, 0.5, s, o)), (s, o)
    for o in (7, (1 << 40) + 3, -2):
        assert np.array_equal(mask(5, torch.tensor([o], device="cuda")), dropout_keep(3001, 0.5, 5, o))


def test_dropped_elements_may_hold_anything():
    import torch
    import paper_2605_22791_amd as g2
    _case("infinities and NaN in dropped places")
    x, r = torch.randn(2000, device="cuda"), torch.randn(2000, device="cuda")
    keep = torch.from_numpy(dropout_keep(2000, 0.4, 2, 0)).cuda()
    want = g2.gdr2_dropout_fwd(x, 0.4, 2, residual=r)
    for v in (float("inf"), float("nan"), -float("inf")):
        assert torch.equal(g2.gdr2_dropout_fwd(torch.where(keep, x, v), 0.4, 2, residual=r), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place(dtype):
    import paper_2605_22791_amd as g2
    _case(f"in place {dtype}")
    x, r = _t(_draw(999, dtype, 0), dtype), _t(_draw(999, dtype, 1), dtype)
    want, dx = g2.gdr2_dropout_fwd(x, 0.2, 3, residual=r), g2.gdr2_dropout_bwd(x, 0.2, 3)
    for into in ("x", "r"):
        a, b = x.clone(), r.clone()
        y = g2.gdr2_dropout_fwd(a, 0.2, 3, residual=b, y=a if into == "x" else b)
        assert bool((y == want).all())
    assert bool((g2.gdr2_dropout_bwd(x, 0.2, 3, dx=x) == dx).all())


def test_guards_and_a_replayed_graph_that_drops_others():
    import torch
    import paper_2605_22791_amd as g2
    _case("guards, graph, another stream")
    n = 4099
    x, r = torch.randn(n, device="cuda").to(torch.bfloat16), torch.randn(n, device="cuda")
    big = torch.full((n + 1024,), float("nan"), device="cuda")
    y, step = big[512:512 + n], torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g2.gdr2_dropout_fwd(x, 0.3, 4, offset=step, residual=r, y=y)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        g2.gdr2_dropout_fwd(x, 0.3, 4, offset=step, residual=r, y=y)
        step += 1
    for k in range(4):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, g2.gdr2_dropout_fwd(x, 0.3, 4, offset=k, residual=r)), k
    assert torch.isnan(big[:512]).all() and torch.isnan(big[-512:]).all()


def test_refusals():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    x = torch.zeros((4, 6), dtype=torch.bfloat16, device="cuda")
    for f in (lambda: g2.gdr2_dropout_fwd(x, 1.0, 0), lambda: g2.gdr2_dropout_fwd(x, float("nan"), 0),
              lambda: g2.gdr2_dropout_fwd(x.t(), 0.1, 0), lambda: g2.gdr2_dropout_fwd(x, 0.1, 0, residual=x[:2]),
              lambda: g2.gdr2_dropout_fwd(x, 0.1, 0, y=x.float()),
              lambda: g2.gdr2_dropout_fwd(x, 0.1, 0, offset=torch.zeros(2, dtype=torch.int64, device="cuda")),
              lambda: g2.gdr2_dropout_fwd(x, 0.1, 0, offset=torch.zeros(1, dtype=torch.int64)),
              lambda: g2.gdr2_dropout_bwd(x, -0.1, 0), lambda: g2.gdr2_dropout_bwd(x, 0.1, 0, dx=x[:1])):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: g2.gdr2_dropout_fwd(x.float(), 0.1, 0, residual=x), lambda: g2.gdr2_dropout_bwd(x, 0.1, 0, dtype=torch.float32)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(g2.Gdr2Error):  # a view that starts off 16 bytes
        g2.gdr2_dropout_fwd(torch.zeros(9, device="cuda")[1:], 0.1, 0)
    assert g2.gdr2_dropout_fwd(x[:0], 0.1, 0).shape == (0, 6)
