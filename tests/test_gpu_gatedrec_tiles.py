"""The gated linear recurrence on the GPU at the sizes of training: from 4096 workgroups of 64 tokens on the forward takes
tiles of 128 tokens, with the look over eight tiles unless the chain is long beside its channels; and batches whose
sequences differ a thousandfold in length.  The reference is the definition, token by token, in 64 bits on the GPU.

Tolerances as in tests/test_gpu_gatedrec.py: bf16 outputs are one rounding (2^-8 / sqrt 3 at a mean mantissa, 1.7e-3 of the
norm) of a result good to fp32: 2e-3; fp32 ones 5e-6, for memories of up to some 60 tokens."""

import pytest

pytestmark = pytest.mark.gpu

OPTIONS = [(gate, normalize, dtype) for gate in (False, True) for normalize in (False, True) for dtype in ("bf16", "fp32")]


def _inputs(B, T, D, n, gate, dtype, seed):
    """Tensors on the GPU: x, g, i, h0, do, dhT."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return dict(x=f(B, T, D).to(dt), g=-torch.nn.functional.softplus(f(B, T, D) - 2), i=torch.sigmoid(f(B, T, D)).to(dt) if gate else None,
                h0=f(n, D), do=f(B, T, D).to(dt), dhT=f(n, D))


def _reference(t, lengths, normalize):
    """In 64 bits: the sequences side by side, (longest, sequences, D), rows past a sequence's end leaving the state alone."""
    import torch
    D, n, L = t["x"].shape[2], len(lengths), max(lengths)
    on = torch.arange(L, device="cuda")[:, None] < torch.tensor(lengths, device="cuda")

    def side(x):
        to = torch.zeros((n, L, D), dtype=torch.float64, device="cuda")
        to[on.T] = x.reshape(-1, D).double()
        return to.transpose(0, 1).contiguous()

    def flat(x):
        return x.transpose(0, 1)[on.T].reshape(t["x"].shape)

    g, x, do = side(t["g"]), side(t["x"]), side(t["do"])
    i = torch.ones_like(x) if t["i"] is None else side(t["i"])
    a, m = torch.exp(g), torch.sqrt(-torch.expm1(2 * g)) if normalize else torch.ones_like(g)
    u, h, before, after = m * i * x, t["h0"].double(), torch.empty_like(x), torch.empty_like(x)
    on3 = on[:, :, None]
    for k in range(L):
        before[k] = h
        h = torch.where(on3[k], a[k] * h + u[k], h)
        after[k] = h
    c, dh = t["dhT"].double(), torch.empty_like(x)
    for k in reversed(range(L)):
        dh[k] = do[k] + c
        c = torch.where(on3[k], a[k] * dh[k], c)
    dg = a * before * dh
    if normalize:
        dg = dg - torch.where(on3, a * a / m, 0.0) * i * x * dh
    want = {"o": flat(after), "h_T": h, "dx": flat(m * i * dh), "dlog_decay": flat(dg), "dh0": c}
    if t["i"] is not None:
        want["dgate"] = flat(m * x * dh)
    return want


def _in_parts(t, parts, normalize):
    """_reference of a packed batch, its sequences' lengths in runs that are side by side each."""
    import torch
    out, row, seq = [], 0, 0
    for lengths in parts:
        part = {n: None if x is None else x[seq:seq + len(lengths)] if n in ("h0", "dhT") else x[:, row:row + sum(lengths)]
                for n, x in t.items()}
        out.append(_reference(part, lengths, normalize))
        row, seq = row + sum(lengths), seq + len(lengths)
    return {n: torch.cat([w[n] for w in out], 0 if n in ("h_T", "dh0") else 1) for n in out[0]}


def _check(t, lengths, packed, normalize, want=None):
    import torch
    import paper_2605_22791_amd as g2
    want = want or _reference(t, lengths, normalize)
    cu = None
    if packed:
        cu = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
    how = dict(cu_seqlens=cu, normalize=normalize)
    B, T, D = t["x"].shape
    p = g2.Gdr2Gatedrec(B, T, D, g2.GDR2_BF16 if t["x"].dtype == torch.bfloat16 else g2.GDR2_FP32, int(normalize))
    need = g2.gdr2_gatedrec_workspace_bytes(p, len(lengths) if packed else 0, 1)
    for saved in (False, True):
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        o, h = g2.gdr2_gatedrec_fwd(t["x"], t["g"], t["i"], t["h0"], ws=ws, save=saved, **how)
        if not saved:
            ws.fill_(0xFF)
        got = {"o": o, "h_T": h, **g2.gdr2_gatedrec_bwd(t["x"], t["g"], t["i"], t["h0"], t["do"], t["dhT"], ws=ws, saved=saved, **how)}
        for n, w in want.items():
            e = float((got[n].double() - w).norm() / w.norm())
            print(f"{n} {e:.1e}", end="  ", flush=True)
            assert e < (2e-3 if got[n].dtype == torch.bfloat16 else 5e-6), (n, e, saved)


@pytest.mark.parametrize("gate,normalize,dtype", OPTIONS)
@pytest.mark.parametrize("B,T,D", [(16, 1500, 1155), (5, 3301, 2050), (1, 17001, 2046)])
def test_tiles_of_128(B, T, D, gate, normalize, dtype):
    print(f"\n[gpu case] {B} x {T} x {D} gate {gate} normalize {normalize} {dtype}", flush=True)
    _check(_inputs(B, T, D, B, gate, dtype, T), [T] * B, False, normalize)


@pytest.mark.parametrize("gate,normalize,dtype", OPTIONS)
@pytest.mark.parametrize("lengths,D", [([3000, 1, 700, 2500, 64, 128, 129, 3000, 3000, 1, 127, 4000], 1667),
                                       ([2000, 5000, 1, 3000, 333, 128, 128, 3500, 4096], 1990)], ids=["odd", "even"])
def test_tiles_of_128_packed(lengths, D, gate, normalize, dtype):
    print(f"\n[gpu case] packed {lengths} D {D} gate {gate} normalize {normalize} {dtype}", flush=True)
    _check(_inputs(1, sum(lengths), D, len(lengths), gate, dtype, D), lengths, True, normalize)


@pytest.mark.parametrize("D", [64, 200])
def test_one_long_sequence_among_short_ones(D):
    """The mean length says nothing of the longest: its chain is walked with the look over eight tiles."""
    parts = [3, 1, 17] * 60, [30000], [5, 64, 2] * 60
    lengths = sum(parts, [])
    print(f"\n[gpu case] one long sequence among {len(lengths)}, D {D}", flush=True)
    t = _inputs(1, sum(lengths), D, len(lengths), True, "bf16", D)
    _check(t, lengths, True, True, _in_parts(t, parts, True))
