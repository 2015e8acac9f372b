"""bf16 outputs of linear attention beside the 64-bit values rounded to bf16, and what they may not depend on.

Tolerance: an evaluation in 32 bits errs by a few 2^-23 of a value's typical size, say 5e-7 in the mean; a value
then takes its other neighbour in bf16 with that over a unit (2^-8 to 2^-7 of it) as its probability, and is off by
the unit: in the mean square (5e-7 * 0.8 * 0.8 * 0.0055)^(1/2) = 4.2e-5 of the norm.  6e-5 leaves that half as
much again of the error's square; products of 16-bit operands (2e-6) give 8.4e-5."""

import pytest
import torch

from tests.test_gpu_linattn_grouped import _inputs, _reference

pytestmark = pytest.mark.gpu

TOL = 6e-5


@pytest.mark.parametrize("Dk,Dv", [(128, 128), (64, 64), (64, 128), (128, 64)])
@pytest.mark.parametrize("B,T,H,Hv", [(4, 1000, 16, 16), (8, 1400, 16, 32)])
def test_rounded_as_from_32_bits(B, T, H, Hv, Dk, Dv):
    import paper_2605_22791_amd as g2
    print(f"\n[gpu case] bits B{B} T{T} H{H} Hv{Hv} Dk{Dk} Dv{Dv}", flush=True)
    x = _inputs(B, T, H, Hv, Dk, Dv, "token", seed=Dk + 2 * Dv)
    args = x["q"], x["k"], x["v"], x["g"], x["S0"]
    got = {"o": g2.gdr2_linattn_fwd(*args)[0], **g2.gdr2_linattn_bwd(*args, x["do"], x["dST"])}
    want = _reference(x)
    for n in ("o", "dq", "dk", "dv"):
        near = want[n].to(torch.bfloat16).double()
        e = float((got[n].double() - near).norm() / near.norm())
        print(f"{n} {e:.2e}", end=" ", flush=True)
        assert e < TOL, (n, e)


@pytest.mark.parametrize("cu", [None, [0, 37, 2085, 2085, 2385, 3300]])
def test_outputs_do_not_depend_on_the_states_asked_for(cu):
    import paper_2605_22791_amd as g2
    print(f"\n[gpu case] with and without S_T, dS0 {cu}", flush=True)
    x = _inputs(1, 3300, 8, 16, 128, 128, "token", seed=9, n_seqs=0 if cu is None else len(cu) - 1)
    kw = {} if cu is None else {"cu_seqlens": torch.tensor(cu, dtype=torch.int32, device="cuda")}
    args = x["q"], x["k"], x["v"], x["g"], x["S0"]
    o, _ = g2.gdr2_linattn_fwd(*args, **kw)
    alone, none = g2.gdr2_linattn_fwd(*args, want_state=False, **kw)
    assert none is None and torch.equal(o, alone)
    d = g2.gdr2_linattn_bwd(*args, x["do"], x["dST"], **kw)
    without = g2.gdr2_linattn_bwd(*args, x["do"], x["dST"], want_dS0=False, **kw)
    assert without["dS0"] is None and all(torch.equal(d[n], without[n]) for n in ("dq", "dk", "dv", "dlog_decay"))
