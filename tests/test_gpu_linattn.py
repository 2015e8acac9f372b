"""GPU parity of linear attention with a decay for each head against the fp64 oracle.

Tolerances (rel-L2).  A bf16 output is the rounding of a result that is good to fp32: the
operator's bound 2e-3, or 1.1 times what rounding the oracle's values costs where the tensor
is small.  fp32 outputs, of either type of problem: sums of products over 64 to 128 channels,
64 rows and a state carried over the chunks, each step good to some 2^-23, so 5e-6 for
outputs, states and gradients; the decays' gradient sums up to a chunk's values of either
sign once more: 2e-5."""

import numpy as np
import pytest

from oracle.linattn import linattn_packed_bwd, linattn_packed_fwd, linattn_bwd, linattn_fwd
from paper_2605_22791_amd.inputs import bf16_round
from tests.helpers import rel_l2

pytestmark = pytest.mark.gpu

TOL32, TOL_DECAY = 5e-6, 2e-5


def _case(msg):
    print(f"\n[gpu case] {msg}", flush=True)


def _inputs(B, T, H, Hv, Dk, Dv, dtype, decay, seed, n_seqs=0, shift=-2.0, state=True):
    r = np.random.default_rng(seed)
    rnd = bf16_round if dtype == "bf16" else (lambda x: x)
    f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    ns = n_seqs or B
    d = dict(q=rnd(unit(f(B, T, H, Dk))), k=rnd(unit(f(B, T, H, Dk))), v=rnd(f(B, T, Hv, Dv)), do=rnd(f(B, T, Hv, Dv)))
    g = f(Hv) if decay == "head" else f(B, T, Hv)
    d["g"] = -np.logaddexp(np.float32(0), g + np.float32(shift)).astype(np.float32)
    d["S0"] = np.float32(0.3) * f(ns, Hv, Dk, Dv) if state else None
    d["dST"] = np.float32(0.3) * f(ns, Hv, Dk, Dv) if state else None
    return d


def _dev(d, dtype):
    import torch
    io = torch.bfloat16 if dtype == "bf16" else torch.float32
    out = {}
    for n, x in d.items():
        out[n] = None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        if n in ("q", "k", "v", "do"):
            out[n] = out[n].to(io)
    return out


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _close(name, got, want, dtype, tol=TOL32):
    import torch
    assert tuple(got.shape) == want.shape, name
    if got.dtype == torch.bfloat16:
        tol = max(2e-3, 1.1 * rel_l2(bf16_round(want.astype(np.float32)), want))
    e = rel_l2(_host(got), want)
    print(f"{name} {e:.2e}", end="  ", flush=True)
    assert e < tol, (name, e, tol)


def _check(d, dtype, cu=None, saved=False, dST=True):
    import torch
    import paper_2605_22791_amd as g2
    x = _dev(d, dtype)
    Dk = d["q"].shape[-1]
    scale = Dk ** -0.5
    kw = {} if cu is None else {"cu_seqlens": torch.tensor(cu, dtype=torch.int32, device="cuda")}
    args = x["q"], x["k"], x["v"], x["g"]
    ws = None
    if saved:
        prob = g2._problem(x["q"], x["v"], None)
        ws = torch.empty(g2.gdr2_linattn_workspace_bytes(prob, 0 if cu is None else len(cu) - 1, 1), dtype=torch.uint8,
                         device="cuda")
    o, ST = g2.gdr2_linattn_fwd(*args, x["S0"], ws=ws, save=saved, **kw)
    grads = g2.gdr2_linattn_bwd(*args, x["S0"], x["do"], x["dST"], ws=ws, saved=saved, **kw)
    torch.cuda.synchronize()
    if cu is None:
        oo, SS = linattn_fwd(d["q"], d["k"], d["v"], d["g"], d["S0"], scale)
        gg = linattn_bwd(d["q"], d["k"], d["v"], d["g"], d["S0"], d["do"], d["dST"], scale)
    else:
        oo, SS = linattn_packed_fwd(d["q"], d["k"], d["v"], d["g"], cu, d["S0"], scale)
        gg = linattn_packed_bwd(d["q"], d["k"], d["v"], d["g"], cu, d["S0"], d["do"], d["dST"], scale)
    _close("o", o, oo, dtype)
    _close("S_T", ST, SS, dtype)
    for n in ("dq", "dk", "dv", "dS0"):
        _close(n, grads[n], gg[n], dtype)
    _close("dlog_decay", grads["dlog_decay"], gg["dg"], dtype, TOL_DECAY)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths(T, dtype):
    _case(f"lengths T{T} {dtype}")
    _check(_inputs(2, T, 2, 2, 128, 128, dtype, "token", seed=T), dtype, saved=T % 2 == 1)


@pytest.mark.parametrize("Dk,Dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hv", [(2, 2), (2, 6)])
def test_widths_and_groups(Dk, Dv, dtype, H, Hv):
    _case(f"widths Dk{Dk} Dv{Dv} H{H} Hv{Hv} {dtype}")
    _check(_inputs(1, 150, H, Hv, Dk, Dv, dtype, "token", seed=Dk + Dv + Hv), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("saved", [False, True])
def test_per_head_decay(dtype, saved):
    _case(f"per-head decay {dtype} saved {saved}")
    _check(_inputs(3, 130, 2, 4, 128, 64, dtype, "head", seed=11), dtype, saved=saved)


def test_no_state():
    _case("no initial state")
    _check(_inputs(2, 100, 3, 3, 64, 128, "bf16", "token", seed=12, state=False), "bf16")


@pytest.mark.parametrize("shift", [-8.0, 0.0, 3.0])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slow_and_fast_decays(shift, dtype):
    _case(f"decays shift {shift} {dtype}")
    _check(_inputs(1, 300, 2, 2, 128, 128, dtype, "token", seed=13, shift=shift), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [-np.inf, -3.4e38, -500.0])
def test_forgetting_tokens(dtype, value):
    """Decays of zero here and there (first token, block and chunk edges, neighbours)."""
    _case(f"forgetting tokens {value} {dtype}")
    d = _inputs(2, 200, 2, 2, 128, 64, dtype, "token", seed=14)
    for t in (0, 5, 6, 15, 16, 63, 64, 100, 127, 128, 199):
        d["g"][:, t, :] = value
    d["g"][0, 100:140, 1] = value
    _check(d, dtype)


def test_forgetting_heads():
    _case("per-head decays of zero and one")
    d = _inputs(2, 100, 4, 4, 64, 64, "bf16", "head", seed=15)
    d["g"][:] = [0.0, -np.inf, -0.1, -1e30]
    _check(d, "bf16")


@pytest.mark.parametrize("lengths", [[1], [64, 64], [0, 37, 0, 200, 1, 64, 65, 0], [3] * 40, [0, 0, 5], [130, 1, 1, 700]])
@pytest.mark.parametrize("dtype,decay,H,Hv", [("bf16", "token", 2, 2), ("fp32", "token", 1, 2), ("bf16", "head", 2, 4)])
def test_packed(lengths, dtype, decay, H, Hv):
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(int).tolist()
    _case(f"packed {lengths[:8]} {dtype} {decay}")
    d = _inputs(1, cu[-1], H, Hv, 128, 64, dtype, decay, seed=sum(lengths), n_seqs=len(lengths))
    _check(d, dtype, cu=cu, saved=len(lengths) % 2 == 0)


@pytest.mark.parametrize("B,T,H,decay", [(1, 2500, 2, "token"), (2, 4097, 1, "head"), (9, 1100, 16, "token")])
def test_long(B, T, H, decay):
    _case(f"long B{B} T{T} H{H} {decay}")
    d = _inputs(B, T, H, H, 128, 128, "bf16", decay, seed=T, shift=-4.0)
    keep = [(0, 0), (B - 1, H - 1)]
    import torch
    import paper_2605_22791_amd as g2
    x = _dev(d, "bf16")
    ws = torch.empty(g2.gdr2_linattn_workspace_bytes(g2._problem(x["q"], x["v"], None), 0, 1), dtype=torch.uint8, device="cuda")
    args = x["q"], x["k"], x["v"], x["g"]
    o, ST = g2.gdr2_linattn_fwd(*args, x["S0"], ws=ws, save=True)
    gr = g2.gdr2_linattn_bwd(*args, x["S0"], x["do"], x["dST"], ws=ws, saved=True)
    again = g2.gdr2_linattn_bwd(*args, x["S0"], x["do"], x["dST"])
    assert all(torch.equal(gr[n], again[n]) for n in gr)
    for b, h in keep:
        c = {n: d[n][b:b + 1, :, h:h + 1] for n in ("q", "k", "v", "do")}
        g = d["g"][b:b + 1, :, h:h + 1] if decay == "token" else d["g"][h:h + 1]
        S0, dST = d["S0"][b:b + 1, h:h + 1], d["dST"][b:b + 1, h:h + 1]
        oo, SS = linattn_fwd(c["q"], c["k"], c["v"], g, S0, 128 ** -0.5)
        gg = linattn_bwd(c["q"], c["k"], c["v"], g, S0, c["do"], dST, 128 ** -0.5)
        sub = lambda t: t[b:b + 1, :, h:h + 1]  # noqa: E731
        _close("o", sub(o), oo, "bf16")
        _close("S_T", ST[b:b + 1, h:h + 1], SS, "bf16")
        for n in ("dq", "dk", "dv"):
            _close(n, sub(gr[n]), gg[n], "bf16")
        _close("dS0", gr["dS0"][b:b + 1, h:h + 1], gg["dS0"], "bf16")
        if decay == "token":
            _close("dlog_decay", sub(gr["dlog_decay"]), gg["dg"], "bf16", TOL_DECAY)


def test_gradient_by_differences():
    """The decays' and the inputs' gradients along random directions, from the fp32 forward: a
    difference over 2 h = 2e-2 of a smooth loss, good to h^2 and to fp32's 1e-7 / h: 1e-3."""
    import torch
    import paper_2605_22791_amd as g2
    _case("differences of the fp32 forward")
    d = _dev(_inputs(1, 90, 2, 4, 64, 64, "fp32", "token", seed=16), "fp32")
    args = {n: d[n] for n in ("q", "k", "v", "g", "S0")}
    gr = g2.gdr2_linattn_bwd(*args.values(), d["do"], d["dST"])

    def loss(a):
        o, S = g2.gdr2_linattn_fwd(*a.values())
        return float((o.double() * d["do"].double()).sum() + (S.double() * d["dST"].double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(1)
    for n, m in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("g", "dlog_decay"), ("S0", "dS0")):
        e = gr[m] / gr[m].norm() + 0.1 * torch.randn(gr[m].shape, generator=gen, device="cuda") / gr[m].numel() ** 0.5
        fd = (loss({**args, n: args[n] + 1e-2 * e}) - loss({**args, n: args[n] - 1e-2 * e})) / 2e-2
        want = float((gr[m].double() * e.double()).sum())
        print(n, fd, want, flush=True)
        assert abs(fd - want) < 1e-3 * abs(want)


@pytest.mark.parametrize("B,T,H,Hv,Dk,Dv,dtype,decay", [
    (1, 1, 2, 2, 128, 128, "bf16", "token"), (5, 1, 2, 6, 64, 128, "bf16", "head"), (3, 1, 2, 2, 128, 64, "fp32", "token"),
    (2, 7, 2, 2, 64, 64, "bf16", "token"), (2, 33, 1, 2, 128, 128, "fp32", "head"), (70, 1, 8, 8, 128, 128, "bf16", "token"),
    (40, 3, 16, 16, 128, 128, "bf16", "token"), (300, 2, 2, 2, 64, 128, "fp32", "token")])
def test_step(B, T, H, Hv, Dk, Dv, dtype, decay):
    import paper_2605_22791_amd as g2
    _case(f"step B{B} T{T} H{H} Hv{Hv} Dk{Dk} Dv{Dv} {dtype} {decay}")
    d = _inputs(B, T, H, Hv, Dk, Dv, dtype, decay, seed=B + T)
    if decay == "token":
        d["g"][0, 0, 0] = -np.inf
    x = _dev(d, dtype)
    S = x["S0"].clone()
    o = g2.gdr2_linattn_step(x["q"], x["k"], x["v"], x["g"], S)
    oo, SS = linattn_fwd(d["q"], d["k"], d["v"], d["g"], d["S0"], Dk ** -0.5)
    _close("o", o, oo, dtype)
    _close("S", S, SS, dtype)


@pytest.mark.parametrize("lengths", [[1, 0, 4, 1, 16, 1, 2], [0, 0, 1], [1] * 50, [40, 1, 1]])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_step_packed(lengths, dtype):
    import torch
    import paper_2605_22791_amd as g2
    _case(f"step packed {lengths[:8]} {dtype}")
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(int).tolist()
    d = _inputs(1, cu[-1], 2, 4, 128, 128, dtype, "token", seed=len(lengths), n_seqs=len(lengths))
    x = _dev(d, dtype)
    S = x["S0"].clone()
    o = g2.gdr2_linattn_step(x["q"], x["k"], x["v"], x["g"], S, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    oo, SS = linattn_packed_fwd(d["q"], d["k"], d["v"], d["g"], cu, d["S0"], 128 ** -0.5)
    _close("o", o, oo, dtype)
    _close("S", S, SS, dtype)


def test_chunk_then_steps():
    """A prompt by chunks, then tokens one by one, is the whole sequence."""
    import paper_2605_22791_amd as g2
    _case("prompt, then steps")
    d = _inputs(2, 140, 2, 2, 128, 128, "bf16", "token", seed=17)
    x = _dev(d, "bf16")
    cut = lambda a, b: [x[n][:, a:b].contiguous() for n in ("q", "k", "v", "g")]  # noqa: E731
    o, S = g2.gdr2_linattn_fwd(*cut(0, 130), x["S0"])
    oo, SS = linattn_fwd(d["q"], d["k"], d["v"], d["g"], d["S0"], 128 ** -0.5)
    _close("prompt", o, oo[:, :130], "bf16")
    for t in range(130, 140):
        _close(f"token {t}", g2.gdr2_linattn_step(*cut(t, t + 1), S), oo[:, t:t + 1], "bf16")
    _close("S", S, SS, "bf16")


def test_rows_past_the_tensors_are_not_read_or_written():
    """Buffers whose surroundings hold NaN: nothing of it is read, nothing of it changes."""
    import torch
    import paper_2605_22791_amd as g2
    _case("guarded buffers")
    d = _inputs(1, 77, 2, 2, 128, 64, "bf16", "token", seed=18)
    x = _dev(d, "bf16")

    def guarded(t):
        pad = 4096
        big = torch.full((t.numel() + 2 * pad,), float("nan"), dtype=t.dtype, device="cuda")
        big[pad:pad + t.numel()] = t.reshape(-1)
        return big, big[pad:pad + t.numel()].view(t.shape)

    pairs = {n: guarded(x[n]) for n in ("q", "k", "v", "g", "do", "S0", "dST")}
    x = {n: p[1] for n, p in pairs.items()}
    outs = {n: guarded(torch.zeros_like(x[m])) for n, m in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("dlog_decay", "g"),
                                                         ("dS0", "S0"), ("o", "v"), ("S_T", "S0"))}
    g2.gdr2_linattn_fwd(x["q"], x["k"], x["v"], x["g"], x["S0"], o=outs["o"][1], S_T=outs["S_T"][1])
    grads = {n: outs[n][1] for n in ("dq", "dk", "dv", "dlog_decay", "dS0")}
    g2.gdr2_linattn_bwd(x["q"], x["k"], x["v"], x["g"], x["S0"], x["do"], x["dST"], grads=grads)
    torch.cuda.synchronize()
    for n, (big, inner) in outs.items():
        assert torch.isfinite(inner).all(), n
        assert torch.isnan(big[:4096]).all() and torch.isnan(big[-4096:]).all(), n


def test_bits_streams_and_graph():
    """Run to run the same bits; on another stream; replayed from a graph with other work between."""
    import torch
    import paper_2605_22791_amd as g2
    _case("bits, streams, graph")
    x = _dev(_inputs(2, 300, 4, 8, 128, 128, "bf16", "head", seed=19), "bf16")
    args = x["q"], x["k"], x["v"], x["g"]
    prob = g2._problem(x["q"], x["v"], None)
    ws = torch.empty(g2.gdr2_linattn_workspace_bytes(prob, 0, 1), dtype=torch.uint8, device="cuda")
    o, S = g2.gdr2_linattn_fwd(*args, x["S0"])
    gr = g2.gdr2_linattn_bwd(*args, x["S0"], x["do"], x["dST"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2, S2 = g2.gdr2_linattn_fwd(*args, x["S0"], ws=ws, save=True)
        gr2 = g2.gdr2_linattn_bwd(*args, x["S0"], x["do"], x["dST"], ws=ws, saved=True)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(S, S2) and all(torch.equal(gr[n], gr2[n]) for n in gr)
    St = x["S0"].clone()
    ot = torch.empty_like(o[:, :1])
    one = [t[:, :1].contiguous() for t in args[:3]] + [x["g"]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g2.gdr2_linattn_fwd(*args, x["S0"], o=o2, S_T=S2, ws=ws)
        g2.gdr2_linattn_step(*one, St, o=ot)
    want = x["S0"].clone()
    St.copy_(want)
    for _ in range(3):
        o2.zero_()
        graph.replay()
        w = g2.gdr2_linattn_step(*one, want)
        torch.cuda.synchronize()
        assert torch.equal(o2, o) and torch.equal(S2, S) and torch.equal(St, want) and torch.equal(ot, w)


def test_refusals_launch_nothing():
    import torch
    import paper_2605_22791_amd as g2
    _case("refusals")
    x = _dev(_inputs(2, 20, 2, 2, 64, 64, "bf16", "token", seed=20), "bf16")
    q, k, v, g, S0 = (x[n] for n in ("q", "k", "v", "g", "S0"))
    cu = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    bad = [lambda: g2.gdr2_linattn_fwd(q, k[:, :, ::2], v, g), lambda: g2.gdr2_linattn_fwd(q, k, v, g.double()),
           lambda: g2.gdr2_linattn_fwd(q, k, v.float(), g), lambda: g2.gdr2_linattn_fwd(q, k, v, g[:1]),
           lambda: g2.gdr2_linattn_fwd(q, k, v, g, S0[:1]), lambda: g2.gdr2_linattn_fwd(q, k, v, g, save=True),
           lambda: g2.gdr2_linattn_fwd(q.transpose(1, 2), k.transpose(1, 2), v, g),
           lambda: g2.gdr2_linattn_fwd(q, k, v, g, ws=torch.empty(16, dtype=torch.uint8, device="cuda")),
           lambda: g2.gdr2_linattn_bwd(q, k, v, g, S0, x["do"].float()), lambda: g2.gdr2_linattn_step(q, k, v, g, None),
           lambda: g2.gdr2_linattn_bwd(q, k, v, g, S0, x["do"], saved=True),
           lambda: g2.gdr2_linattn_fwd(q, k, v, g, cu_seqlens=cu.long())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(g2.Gdr2Error):   # packed with B = 2
        g2.gdr2_linattn_fwd(q, k, v, g, cu_seqlens=cu)
    h = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(4 * 2 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 2, 64)
    with pytest.raises(g2.Gdr2Error):   # not 16-byte aligned
        g2.gdr2_linattn_fwd(off, h, h, torch.zeros((1, 4, 2), device="cuda"))


@pytest.mark.parametrize("n", [63, 64, 65, 130])
@pytest.mark.parametrize("at", [0, -1])
def test_packed_many_sequences(n, at):
    """Around the most sequences that a wave looks up by itself; a long one, of several segments, first or last."""
    lengths = [(3 * i) % 7 for i in range(n)]
    lengths[at] = 450
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(int).tolist()
    _case(f"packed {n} sequences, the long one at {at}")
    d = _inputs(1, cu[-1], 1, 2, 64, 64, "bf16", "token", seed=n, n_seqs=n)
    _check(d, "bf16", cu=cu, saved=n % 2 == 0)
