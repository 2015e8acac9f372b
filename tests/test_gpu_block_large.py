"""Linear attention and the block norms at sizes past 32-bit offsets.

Linear attention: one sequence of 262141 tokens, 64 value heads of 128 on 32: v, o and their
gradients are 4 GB, the value heads' parts of dq and dk 8 GB in the workspace.  A token near the end forgets the state before it, so that what follows, which
has the highest offsets, is the fp64 oracle's run on those tokens alone; so are its gradients.
Block norms: 2^32 elements and a few rows; the last rows against the oracle on them alone.
Tolerances: as in the other tests of the two."""

import numpy as np
import pytest

from oracle.blocknorm import blocknorm_bwd, blocknorm_fwd
from oracle.linattn import linattn_bwd, linattn_fwd
from tests.helpers import rel_l2

pytestmark = pytest.mark.gpu


def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def test_linattn_past_32bit_offsets():
    import torch
    import paper_2605_22791_amd as g2
    T, H, D, tail = (1 << 18) - 3, 32, 128, 200
    print(f"\n[gpu case] linear attention T{T} H{H} Hv{2 * H} D{D}: 64-bit offsets", flush=True)
    r = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, do = (torch.empty(1, T, n * H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=r) for n in (1, 1, 2, 2))
    q *= D ** -0.5
    k *= D ** -0.5
    g = -torch.nn.functional.softplus(torch.randn(1, T, 2 * H, generator=r, device="cuda") - 2.0)
    g[:, T - tail] = -float("inf")
    o, S = g2.gdr2_linattn_fwd(q, k, v, g)
    d = g2.gdr2_linattn_bwd(q, k, v, g, None, do, want_dS0=False)
    torch.cuda.synchronize()
    for h in (0, H - 1):
        key, value = slice(h, h + 1), slice(2 * h, 2 * h + 2)
        qs, ks, vs, gs, ds = (_host(x[:, T - tail:, n]) for x, n in ((q, key), (k, key), (v, value), (g, value), (do, value)))
        oo, SS = linattn_fwd(qs, ks, vs, gs, None, D ** -0.5)
        dd = linattn_bwd(qs, ks, vs, gs, None, ds, None, D ** -0.5)
        assert rel_l2(_host(o[:, T - tail:, value]), oo) < 2e-3
        assert rel_l2(_host(S[:, value]), SS) < 5e-6
        for n, x in (("dq", key), ("dk", key), ("dv", value)):
            assert rel_l2(_host(d[n][:, T - tail:, x]), dd[n]) < 2e-3, n
        assert rel_l2(_host(d["dlog_decay"][:, T - tail:, value]), dd["dg"]) < 2e-5


def test_blocknorm_past_32bit_offsets():
    import torch
    import paper_2605_22791_amd as g2
    rows, D, last = (1 << 22) + 5, 1024, 6
    print(f"\n[gpu case] block norms {rows} rows of {D}: 64-bit offsets", flush=True)
    r = torch.Generator(device="cuda").manual_seed(6)
    y, z, dh = (torch.empty(rows, D, dtype=torch.bfloat16, device="cuda").normal_(generator=r) for _ in range(3))
    w = torch.rand(D, generator=r, device="cuda") + 0.5
    h, _ = g2.gdr2_blocknorm_fwd(y, w_post=w, gate=z)
    d = g2.gdr2_blocknorm_bwd(y, dh, w_post=w, gate=z)
    torch.cuda.synchronize()
    ys, zs, ds, ws = _host(y[-last:]), _host(z[-last:]), _host(dh[-last:]), _host(w)
    hh = blocknorm_fwd(ys, w_post=ws, z=zs)[0]
    dd = blocknorm_bwd(ys, ds, None, w_post=ws, z=zs)
    assert rel_l2(_host(h[-last:]), hh) < 2e-3
    assert rel_l2(_host(d["dy"][-last:]), dd["dy"]) < 2e-3
    assert rel_l2(_host(d["dgate"][-last:]), dd["dgate"]) < 2e-3
