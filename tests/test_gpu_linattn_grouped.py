"""bf16 training with grouped value heads over long scans on a full card, whole tensors against 64 bits.

Enough heads that a sequence is cut into few segments, of 6 to 18 chunks, and every CU has two of them:
what a wave of such a scan reads before it has landed is the chunk before.

Tolerances: as in test_gpu_linattn.py, bf16 outputs also for each chunk of up to 64 rows of one head by
itself (2e-3, or 1.1 times what rounding the reference's values costs there)."""

import numpy as np
import pytest
import torch

from oracle.linattn import linattn_bwd, linattn_fwd
from tests.test_gpu_linattn import TOL32, TOL_DECAY

BLOCK = 32


def _walk(q, k, v, g, S, scale):
    """o and the last state in 64 bits, (B, T, H, D) on the value heads, block after block; torch differentiates it."""
    B, T, H, _ = q.shape
    out = []
    for t in range(0, T, BLOCK):
        qb, kb, vb = (x[:, t:t + BLOCK].transpose(1, 2).contiguous() for x in (q, k, v))
        G = g[:, t:t + BLOCK].transpose(1, 2).cumsum(dim=-1)
        n = G.shape[-1]
        below = torch.ones((n, n), dtype=torch.bool, device=q.device).tril()
        D = torch.exp(torch.where(below, G.unsqueeze(-1) - G.unsqueeze(-2), float("-inf")))
        P = torch.matmul(qb, kb.transpose(-1, -2).contiguous()) * D
        out.append((torch.matmul(P, vb) + torch.matmul(qb, S) * torch.exp(G).unsqueeze(-1)).transpose(1, 2))
        w = torch.exp(G[..., -1:] - G).unsqueeze(-1)
        S = torch.exp(G[..., -1])[..., None, None] * S + torch.matmul((kb * w).transpose(-1, -2).contiguous(), vb)
    return scale * (torch.cat(out, dim=1) if out else v), S


def _reference(x, cu=None):
    """dict o, S_T and the gradients in 64 bits."""
    p = {n: x[n].double().requires_grad_(True) for n in ("q", "k", "v", "g", "S0")}
    G = x["v"].shape[2] // x["q"].shape[2]
    q, k = (p[n].repeat_interleave(G, dim=2) for n in ("q", "k"))
    g = p["g"] if p["g"].dim() == 3 else p["g"] * torch.ones((*x["v"].shape[:2], 1), dtype=torch.float64, device=q.device)
    scale = q.shape[-1] ** -0.5
    if cu is None:
        o, S = _walk(q, k, p["v"], g, p["S0"], scale)
    else:
        parts = [_walk(*(t[:, a:b] for t in (q, k, p["v"], g)), p["S0"][i:i + 1], scale)
                 for i, (a, b) in enumerate(zip(cu, cu[1:]))]
        o, S = (torch.cat([y[i] for y in parts], dim=1 - i) for i in (0, 1))
    ((o * x["do"].double()).sum() + (S * x["dST"].double()).sum()).backward()
    names = {"q": "dq", "k": "dk", "v": "dv", "g": "dlog_decay", "S0": "dS0"}
    return {"o": o.detach(), "S_T": S.detach(), **{m: p[n].grad for n, m in names.items()}}


def _inputs(B, T, H, Hv, Dk, Dv, decay, seed, n_seqs=0, device="cuda", io=torch.bfloat16):
    r = torch.Generator(device=device).manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=r, device=device)  # noqa: E731
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)  # noqa: E731
    ns = n_seqs or B
    g = f(B, T, Hv) if decay == "token" else f(Hv)
    return dict(q=unit(f(B, T, H, Dk)).to(io), k=unit(f(B, T, H, Dk)).to(io), v=f(B, T, Hv, Dv).to(io),
                g=-torch.nn.functional.softplus(g - 3.0), S0=0.3 * f(ns, Hv, Dk, Dv), do=f(B, T, Hv, Dv).to(io),
                dST=0.3 * f(ns, Hv, Dk, Dv))


@pytest.mark.parametrize("decay", ["token", "head"])
def test_the_reference_is_the_oracle(decay):
    x = _inputs(2, 75, 2, 4, 8, 6, decay, 1, device="cpu", io=torch.float32)
    got = _reference(x)
    n = {m: t.numpy() for m, t in x.items()}
    o, S = linattn_fwd(n["q"], n["k"], n["v"], n["g"], n["S0"], 8 ** -0.5)
    want = linattn_bwd(n["q"], n["k"], n["v"], n["g"], n["S0"], n["do"], n["dST"], 8 ** -0.5)
    want = {"o": o, "S_T": S, "dlog_decay": want.pop("dg"), **want}
    for m, t in want.items():
        assert np.linalg.norm(got[m].numpy() - t) < 1e-12 * np.linalg.norm(t), m


def _close(name, got, want, cuts):
    d = got.double() - want
    rounding = want.to(torch.bfloat16).double() - want
    size = float(want.norm())
    e = float(d.norm()) / size
    if got.dtype == torch.bfloat16:
        tol = max(2e-3, 1.1 * float(rounding.norm()) / size)
    else:
        tol = TOL_DECAY if name == "dlog_decay" else TOL32
    print(f"{name} {e:.2e}", end=" ", flush=True)
    assert e < tol, (name, e, tol)
    if got.dtype == torch.bfloat16:
        worst = 0.0
        for a, b in zip(cuts, cuts[1:]):
            for t in range(a, b, 64):
                c = slice(t, min(t + 64, b))
                off, own, all_ = (y[:, c].pow(2).sum(dim=(1, 3)).sqrt() for y in (d, rounding, want))
                worst = max(worst, float((off / torch.maximum(2e-3 * all_, 1.1 * own)).max()))
        print(f"(a chunk's share of its bound {worst:.2f})", end=" ", flush=True)
        assert worst < 1.0, (name, worst)


def _check(x, cu=None):
    import paper_2605_22791_amd as g2
    args = x["q"], x["k"], x["v"], x["g"], x["S0"]
    kw = {} if cu is None else {"cu_seqlens": torch.tensor(cu, dtype=torch.int32, device="cuda")}
    need = g2.gdr2_linattn_workspace_bytes(g2._problem(x["q"], x["v"], None), 0 if cu is None else len(cu) - 1, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    o, S = g2.gdr2_linattn_fwd(*args, ws=ws, save=True, **kw)
    got = g2.gdr2_linattn_bwd(*args, x["do"], x["dST"], ws=ws, saved=True, **kw)
    again = g2.gdr2_linattn_bwd(*args, x["do"], x["dST"], **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], again[n]) for n in got)
    want = _reference(x, cu)
    for n, t in {"o": o, "S_T": S, **got}.items():
        _close(n, t, want[n], [0, x["q"].shape[1]] if cu is None else cu)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,H,Hv,Dk,Dv,decay", [
    (9, 1100, 8, 16, 128, 128, "token"), (16, 1100, 8, 32, 128, 128, "token"), (16, 1090, 16, 32, 64, 64, "head"),
    (12, 1300, 8, 16, 64, 128, "token"), (12, 1300, 8, 16, 128, 64, "token")])
def test_grouped_heads_over_long_scans(B, T, H, Hv, Dk, Dv, decay):
    print(f"\n[gpu case] grouped B{B} T{T} H{H} Hv{Hv} Dk{Dk} Dv{Dv} {decay}", flush=True)
    _check(_inputs(B, T, H, Hv, Dk, Dv, decay, seed=T + Hv))


@pytest.mark.gpu
def test_packed_grouped_heads_over_long_scans():
    lengths = [1500, 37, 2048, 0, 300, 911, 64, 2500, 129, 3000, 203]
    cu = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    print(f"\n[gpu case] grouped, packed {lengths}", flush=True)
    _check(_inputs(1, cu[-1], 16, 32, 128, 128, "token", seed=3, n_seqs=len(lengths)), cu)
