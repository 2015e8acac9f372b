"""The gated linear recurrence on the GPU against the fp64 oracle.

Tolerances (rel-L2).  A bf16 output is the rounding of a result that is good to fp32: 2e-3, or
1.1 times what rounding the oracle's values costs where the tensor is small.  fp32 outputs: a
value's weight falls by a factor a step, each factor and each sum good to 2^-23, over memories of up to
some 60 tokens here (decays of softplus(N - 4), about 0.02 a token): 60 * 2^-23 = 7e-6 if every rounding
fell the same way, their square root of it if they fall differently; 5e-6."""

import numpy as np
import pytest

from oracle.gatedrec import gatedrec_bwd, gatedrec_fwd, gatedrec_packed_bwd, gatedrec_packed_fwd
from paper_2605_22791_amd.inputs import bf16_round
from tests.helpers import rel_l2

pytestmark = pytest.mark.gpu

TOL32 = 5e-6
NAMES = {"dx": "dx", "dlog_decay": "dg", "dgate": "di", "dh0": "dh0"}


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _inputs(B, T, D, dtype, seed, n_seqs=0, gate=True, state=True, shift=-2.0):
    r = np.random.default_rng(seed)
    rnd = bf16_round if dtype == "bf16" else (lambda x: x)
    f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    ns = n_seqs or B
    d = dict(x=rnd(f(B, T, D)), g=-np.logaddexp(np.float32(0), f(B, T, D) + np.float32(shift)).astype(np.float32),
             i=rnd((1 / (1 + np.exp(-f(B, T, D)))).astype(np.float32)) if gate else None, do=rnd(f(B, T, D)))
    d["h0"], d["dhT"] = (f(ns, D), f(ns, D)) if state else (None, None)
    return d


def _dev(d, dtype):
    import torch
    io = torch.bfloat16 if dtype == "bf16" else torch.float32
    return {n: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda().to(io if n in ("x", "i", "do") else torch.float32)
            for n, x in d.items()}


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _close(name, got, want, where=None):
    import torch
    assert tuple(got.shape) == want.shape, name
    got32 = _host(got)
    if where is not None:
        got32, want = got32[where], want[where]
    tol = TOL32
    if got.dtype == torch.bfloat16:
        tol = max(2e-3, 1.1 * rel_l2(bf16_round(want.astype(np.float32)), want))
    e = rel_l2(got32, want)
    print(f"{name} {e:.1e}", end="  ", flush=True)
    assert e < tol, (name, e, tol)


def _ws(t, cu, normalize, fill=0xFF):
    import torch
    import paper_2605_22791_amd as g2
    B, T, D = t["x"].shape
    p = g2.Gdr2Gatedrec(B, T, D, g2.GDR2_BF16 if t["x"].dtype == torch.bfloat16 else g2.GDR2_FP32, int(normalize))
    n = g2.gdr2_gatedrec_workspace_bytes(p, 0 if cu is None else cu.numel() - 1, 1)
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda")


def _run(t, cu=None, normalize=False, saved=False, fill=0xFF):
    """What the workspace holds before a call (NaN, or zeros, or values) means nothing."""
    import paper_2605_22791_amd as g2
    how = dict(cu_seqlens=cu, normalize=normalize)
    ws = _ws(t, cu, normalize, fill)
    o, h = g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], save=saved, ws=ws, **how)
    if not saved:
        ws.fill_(fill)
    d = g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], ws=ws, saved=saved, **how)
    return {"o": o, "h_T": h, **d}


def _check(B, T, D, dtype, seed=0, normalize=False, saved=False, **kw):
    d = _inputs(B, T, D, dtype, seed, **kw)
    got = _run(_dev(d, dtype), normalize=normalize, saved=saved)
    o, h = gatedrec_fwd(d["x"], d["g"], d["i"], d["h0"], normalize)
    want = gatedrec_bwd(d["x"], d["g"], d["i"], d["h0"], d["do"], d["dhT"], normalize)
    _close("o", got["o"], o)
    _close("h_T", got["h_T"], h)
    for n, m in NAMES.items():
        assert (got[n] is None) == (want[m] is None), n
        if want[m] is not None:
            _close(n, got[n], want[m])


@pytest.mark.parametrize("B,T,D", [(1, 1, 1), (2, 1, 64), (3, 5, 7), (4, 2, 300), (1, 63, 65), (2, 64, 130), (1, 65, 127),
                                   (3, 129, 512), (1, 511, 96), (2, 512, 128), (1, 513, 129), (2, 1000, 257), (7, 300, 66),
                                   (1, 4099, 33), (5, 100, 1155), (1, 2048, 1024), (40, 33, 200),
                                   (1, 20000, 33), (1, 30000, 200)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shapes(B, T, D, dtype):
    _case(f"B {B} T {T} D {D} {dtype}")
    _check(B, T, D, dtype, seed=T, normalize=True)
    _check(B, T, D, dtype, seed=T + 1, saved=True)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_options(gate, state, normalize, dtype):
    _case(f"gate {gate} state {state} normalize {normalize} {dtype}")
    for saved in (False, True):
        _check(2, 700, 160, dtype, seed=3, gate=gate, state=state, normalize=normalize, saved=saved)


@pytest.mark.parametrize("shift", [3.0, 0.0, -4.0])
@pytest.mark.parametrize("T", [3000, 9000])
def test_decays(shift, T):
    _case(f"decays of softplus(N + {shift}), T {T}")
    _check(1, T, 128, "fp32", seed=int(shift) + 9, shift=shift, normalize=True)
    _check(1, T, 128, "bf16", seed=int(shift) + 10, shift=shift, saved=True)


PACKED = [[1], [5, 1, 2], [0, 3, 0, 0, 4, 0], [64, 64, 64], [1] * 130, [300, 0, 17, 1, 1025, 63, 64, 65, 2, 511],
          [2000, 1, 1, 1, 3000], [9000, 12000, 0, 700], [0, 0, 0], [7] * 200, [512, 512, 512, 512], [513, 511, 1, 1535]]


@pytest.mark.parametrize("lengths", PACKED, ids=lambda x: f"{len(x)}x{sum(x)}")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed(lengths, dtype):
    import torch
    import paper_2605_22791_amd as g2
    for D, before, behind, normalize in ((96, 0, 0, True), (129, 3, 5, False)):
        _case(f"packed {lengths[:12]} D {D} before {before} behind {behind} {dtype}")
        cu = np.cumsum([before] + lengths)
        T = int(cu[-1]) + behind
        if T == 0:
            T = 2
        n = len(lengths)
        d = _inputs(1, T, D, dtype, seed=T, n_seqs=n)
        d["x"][:, :before], d["x"][:, cu[-1]:] = np.nan, np.inf  # rows of no sequence
        t, cut = _dev(d, dtype), torch.from_numpy(cu.astype(np.int32)).cuda()
        o, h = gatedrec_packed_fwd(d["x"], d["g"], d["i"], d["h0"], cu, normalize)
        want = gatedrec_packed_bwd(d["x"], d["g"], d["i"], d["h0"], d["do"], d["dhT"], cu, normalize)
        inside = ~np.isnan(o)
        for saved in (False, True):
            how = dict(cu_seqlens=cut, normalize=normalize)
            ws = _ws(t, cut, normalize)
            to = torch.full_like(t["x"], 77.0)
            _, hT = g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], o=to, ws=ws, save=saved, **how)
            grads = {"dx": torch.full_like(t["x"], 77.0), "dgate": torch.full_like(t["x"], 77.0),
                     "dlog_decay": torch.full_like(t["g"], 77.0)}
            g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], grads=grads, ws=ws, saved=saved,
                                 want_dh0=False, **how)
            dh0 = g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], ws=ws, saved=saved, **how)["dh0"]
            _close("h_T", hT, h)
            _close("dh0", dh0, want["dh0"])
            for name, a, b in [("o", to, o)] + [(m, grads[m], want[NAMES[m]]) for m in grads]:
                if inside.any():
                    _close(name, a, b, inside)
                assert (_host(a)[~inside] == 77.0).all(), name  # left as they were
    empty = np.array(lengths) == 0
    assert np.array_equal(_host(hT)[empty], d["h0"][empty].astype(np.float64))


@pytest.mark.parametrize("T", [1, 2, 9, 40])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_step(T, dtype):
    import paper_2605_22791_amd as g2
    _case(f"step T {T} {dtype}")
    for B, D, gate, normalize in ((1, 2048, True, True), (33, 130, False, False), (5, 7, True, False)):
        d = _inputs(B, T, D, dtype, seed=T, gate=gate)
        t = _dev(d, dtype)
        h = t["h0"].clone()
        o = g2.gdr2_gatedrec_step(t["x"], t["g"], t["i"], h, normalize=normalize)
        wo, wh = gatedrec_fwd(d["x"], d["g"], d["i"], d["h0"], normalize)
        _close("o", o, wo)
        _close("h", h, wh)


def test_step_packed_and_behind_a_forward():
    import torch
    import paper_2605_22791_amd as g2
    _case("step packed")
    lengths = [1, 4, 0, 1, 16, 2]
    cu = np.cumsum([0] + lengths)
    d = _inputs(1, 26, 100, "bf16", seed=8, n_seqs=6)
    t = _dev(d, "bf16")
    h, o = t["h0"].clone(), torch.full_like(t["x"], 77.0)
    g2.gdr2_gatedrec_step(t["x"], t["g"], t["i"], h, cu_seqlens=torch.from_numpy(cu.astype(np.int32)).cuda(), o=o)
    wo, wh = gatedrec_packed_fwd(d["x"], d["g"], d["i"], d["h0"], cu)
    _close("o", o[:, :24].contiguous(), wo[:, :24])
    _close("h", h, wh)
    assert bool((o[:, 24:] == 77.0).all())
    _case("a prompt, then tokens")
    d = _inputs(3, 600, 65, "fp32", seed=9)
    t = _dev(d, "fp32")
    cut = lambda n, a, b: t[n][:, a:b].contiguous()  # noqa: E731
    o1, h = g2.gdr2_gatedrec_fwd(cut("x", 0, 590), cut("g", 0, 590), cut("i", 0, 590), t["h0"], normalize=True)
    o2 = g2.gdr2_gatedrec_step(cut("x", 590, 600), cut("g", 590, 600), cut("i", 590, 600), h, normalize=True)
    wo, wh = gatedrec_fwd(d["x"], d["g"], d["i"], d["h0"], True)
    _close("o", torch.cat([o1, o2], 1), wo)
    _close("h", h, wh)


def test_far_decays():
    """-inf and very negative decays forget the state; a decay of 0 keeps it, and its normalized input is nothing."""
    _case("far decays")
    for normalize in (False, True):
        d = _inputs(2, 300, 64, "fp32", seed=11)
        d["g"][:, 5] = -np.inf
        d["g"][:, 17] = -300.0
        d["g"][:, 100:103] = 0.0
        d["g"][:, 200, ::2] = -1e-30
        got = _run(_dev(d, "fp32"), normalize=normalize)
        o, h = gatedrec_fwd(d["x"], d["g"], d["i"], d["h0"], normalize)
        want = gatedrec_bwd(d["x"], d["g"], d["i"], d["h0"], d["do"], d["dhT"], normalize)
        _close("o", got["o"], o)
        _close("h_T", got["h_T"], h)
        rest = np.ones(300, bool)
        rest[200] = False  # normalized, the slope there is 1e15: looked at by itself
        for n, m in NAMES.items():
            if n == "dlog_decay":
                _close(n, got[n][:, rest.tolist()], want[m][:, rest])
                _close(n, got[n][:, 200], want[m][:, 200])
            else:
                _close(n, got[n], want[m])


def test_values_of_one_sequence_do_not_reach_another():
    import torch
    import paper_2605_22791_amd as g2
    lengths = [70, 3, 600, 1, 0, 400, 513]
    cu = np.cumsum([0] + lengths)
    cut = torch.from_numpy(cu.astype(np.int32)).cuda()
    d = _inputs(1, int(cu[-1]), 80, "bf16", seed=12, n_seqs=7)
    t = _dev(d, "bf16")
    clean = _run(t, cut, True)
    for s in (0, 2, 3, 6):
        for v in (float("nan"), float("inf")):
            _case(f"{v} in sequence {s}")
            u = {n: None if x is None else x.clone() for n, x in t.items()}
            at = int(cu[s]) + lengths[s] // 2
            u["x"][:, at] = v
            u["do"][:, at] = v
            got = _run(u, cut, True)
            for n, x in got.items():
                other = torch.ones(x.shape[0 if n in ("h_T", "dh0") else 1], dtype=torch.bool, device="cuda")
                other[s if n in ("h_T", "dh0") else slice(int(cu[s]), int(cu[s + 1]))] = False
                a, b = (x[other], clean[n][other]) if n in ("h_T", "dh0") else (x[:, other], clean[n][:, other])
                assert torch.equal(a, b), (s, n)


def test_gradient_by_differences():
    """Along random directions, from the fp32 forward (2 h = 2e-2; good to h^2 and 1e-7 / h): 1e-3."""
    import torch
    import paper_2605_22791_amd as g2
    _case("differences of the fp32 forward")
    d = _inputs(2, 90, 33, "fp32", seed=13, shift=0.0)
    t = _dev(d, "fp32")
    grads = _run(t, normalize=True)

    def loss(a):
        o, h = g2.gdr2_gatedrec_fwd(a["x"], a["g"], a["i"], a["h0"], normalize=True)
        return float((o.double() * t["do"].double()).sum() + (h.double() * t["dhT"].double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(2)
    for n, m in (("x", "dx"), ("g", "dlog_decay"), ("i", "dgate"), ("h0", "dh0")):
        g = grads[m]
        e = g / g.norm() + 0.1 * torch.randn(g.shape, generator=gen, device="cuda") / g.numel() ** 0.5
        fd = (loss({**t, n: t[n] + 1e-2 * e}) - loss({**t, n: t[n] - 1e-2 * e})) / 2e-2
        want = float((g.double() * e.double()).sum())
        assert abs(fd - want) < 1e-3 * abs(want), n


@pytest.mark.parametrize("lengths", [None, [700, 0, 1, 1300, 99]])
def test_bits_guards_graphs_and_streams(lengths):
    """The same bits every time: again, saved, in two captured graphs that share a workspace, replayed among eager calls, on
    another stream; and nothing written beside the outputs."""
    import torch
    import paper_2605_22791_amd as g2
    _case(f"bits, guards, graphs, streams {lengths}")
    n = 0 if lengths is None else len(lengths)
    d = _inputs(1 if n else 2, 2100, 133, "bf16", seed=14, n_seqs=n)
    t = _dev(d, "bf16")
    cu = torch.from_numpy(np.cumsum([0] + lengths).astype(np.int32)).cuda() if n else None
    how = dict(cu_seqlens=cu, normalize=True)
    want = _run(t, cu, True)
    for other in [_run(t, cu, True, saved=s, fill=f) for s in (False, True) for f in (0xFF, 0x00, 0x3E)]:
        assert all(torch.equal(want[m], other[m]) for m in want)

    def guarded(like):
        big = torch.full((like.numel() + 1024,), float("nan"), dtype=like.dtype, device="cuda")
        return big, big[512:512 + like.numel()].view(like.shape)

    out = {m: guarded(v) for m, v in want.items()}
    ws = _ws(t, cu, True)

    def forward():
        g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], o=out["o"][1], h_T=out["h_T"][1], ws=ws, **how)

    def backward():
        g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], ws=ws,
                             grads={m: out[m][1] for m in NAMES}, **how)

    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        forward()
    with torch.cuda.graph(two):
        backward()
    for fill in (0xFF, 0x00, 0x3E):
        for _, v in out.values():
            v.zero_()
        ws.fill_(fill)
        one.replay()
        two.replay()
        g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], **how)
        torch.cuda.synchronize()
        assert all(torch.equal(out[m][1], want[m]) for m in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, v in out.values():
            v.zero_()
        forward()
        backward()
    side.synchronize()
    assert all(torch.equal(out[m][1], want[m]) for m in want)
    for big, _ in out.values():
        assert torch.isnan(big[:512]).all() and torch.isnan(big[-512:]).all()


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    import torch
    import paper_2605_22791_amd as g2
    _case("two streams")
    ts = [_dev(_inputs(1, 6000, 256, "bf16", seed=s), "bf16") for s in (20, 21)]
    want = [_run(t, None, True) for t in ts]
    streams = [torch.cuda.Stream() for _ in ts]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, (t, st) in enumerate(zip(ts, streams)):
            with torch.cuda.stream(st):
                got[k].append(_run(t, None, True))
    torch.cuda.synchronize()
    for k in (0, 1):
        for g in got[k]:
            assert all(torch.equal(g[m], want[k][m]) for m in g)


def test_offsets_that_are_out_of_order_stay_in_range():
    """Such offsets describe no sequences; the call's results are unspecified, but nothing outside its buffers is touched:
    the guards around every output hold."""
    import torch
    import paper_2605_22791_amd as g2
    _case("offsets out of order")
    d = _inputs(1, 300, 64, "fp32", seed=15, n_seqs=4)
    t = _dev(d, "fp32")
    for cu in ([0, 200, 100, 400, 300], [-50, 20, 10 ** 9, -10 ** 9, 5], [300, 200, 100, 50, 0]):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        big = torch.full((4, 300 * 64 + 1024), 5.0, device="cuda")
        out = [b[512:512 + 300 * 64].view(1, 300, 64) for b in big]
        st = torch.full((2, 4 * 64 + 1024), 5.0, device="cuda")
        hT, dh0 = (b[512:512 + 256].view(4, 64) for b in st)
        g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], cu_seqlens=c, o=out[0], h_T=hT)
        g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], cu_seqlens=c,
                             grads={"dx": out[1], "dlog_decay": out[2], "dgate": out[3], "dh0": dh0})
        torch.cuda.synchronize()
        for b in (big, st):
            assert bool((b[:, :512] == 5).all()) and bool((b[:, -512:] == 5).all())


def test_refusals():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    x = torch.zeros((1, 4, 16), dtype=torch.bfloat16, device="cuda")
    g, h = torch.zeros((1, 4, 16), device="cuda"), torch.zeros((1, 16), device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    ws = torch.empty(8, dtype=torch.uint8, device="cuda")
    for f in (lambda: g2.gdr2_gatedrec_fwd(x, x), lambda: g2.gdr2_gatedrec_fwd(x, g, g), lambda: g2.gdr2_gatedrec_fwd(x, g, h0=h[:, :8]),
              lambda: g2.gdr2_gatedrec_fwd(x, g, cu_seqlens=cu.long()), lambda: g2.gdr2_gatedrec_fwd(x, g, cu_seqlens=cu[:1]),
              lambda: g2.gdr2_gatedrec_fwd(x, g, ws=ws), lambda: g2.gdr2_gatedrec_fwd(x, g, save=True),
              lambda: g2.gdr2_gatedrec_fwd(x, g, o=g), lambda: g2.gdr2_gatedrec_fwd(x, g, h_T=h.half()),
              lambda: g2.gdr2_gatedrec_fwd(x.transpose(1, 2), g), lambda: g2.gdr2_gatedrec_bwd(x, g, None, None, None),
              lambda: g2.gdr2_gatedrec_bwd(x, g, None, None, g), lambda: g2.gdr2_gatedrec_bwd(x, g, None, None, x, saved=True),
              lambda: g2.gdr2_gatedrec_bwd(x, g, None, None, x, grads={"dgate": x}),
              lambda: g2.gdr2_gatedrec_bwd(x, g, None, None, x, grads={"dx": g}),
              lambda: g2.gdr2_gatedrec_step(x, g, None, None), lambda: g2.gdr2_gatedrec_step(x, g, None, h[:, :3])):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(g2.Gdr2Error):  # a packed batch has one row
        g2.gdr2_gatedrec_fwd(x.repeat(2, 1, 1), g.repeat(2, 1, 1), cu_seqlens=cu)
