"""How far a non-finite value of one token reaches (include/gdr2_linattn.h); all else keeps its bits."""

import pytest
import torch

from tests.test_gpu_linattn_grouped import _inputs

pytestmark = pytest.mark.gpu

AT, CHUNK = 1500, slice(1472, 1536)  # the token, its chunk of 64


def _run(x):
    import paper_2605_22791_amd as g2
    args = x["q"], x["k"], x["v"], x["g"], x["S0"]
    o, S = g2.gdr2_linattn_fwd(*args)
    return {"o": o, "S_T": S, **g2.gdr2_linattn_bwd(*args, x["do"], x["dST"])}


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("dtype,B,H", [("bf16", 16, 32), ("fp32", 1, 4)])  # bf16: sequences in one segment
@pytest.mark.parametrize("decay", ["token", "head"])
def test_reach(value, name, dtype, B, H, decay):
    print(f"\n[gpu case] {value} in {name} {dtype} {decay}", flush=True)
    x = _inputs(B, 2500, H, H, 64, 64, decay, seed=4, io=torch.bfloat16 if dtype == "bf16" else torch.float32)
    clean = _run(x)
    b, h = B - 1, 2
    x[name] = x[name].clone()
    x[name][b, AT, h, 7] = value
    got = _run(x)
    forth = name in ("k", "v")
    before, behind, outside = [slice(0, CHUNK.start)], [slice(CHUNK.stop, None)], [slice(0, CHUNK.start), slice(CHUNK.stop, None)]
    kept = {"o": before if forth else outside, "dq": before if forth else outside, "dk": outside if forth else behind,
            "dv": outside if forth else behind,
            "dlog_decay": ([slice(0, AT - 1023)] if dtype == "bf16" else before) if forth else behind}
    for n, t in got.items():
        same = t == clean[n]
        if n in ("S_T", "dS0"):
            mine = same[b, h].all() if (n == "S_T") != forth else True
            same[b, h] = True
        elif n == "dlog_decay" and decay == "head":
            mine = True
            same[h] = True
        else:
            mine = all(same[b, s, h].all() for s in kept[n])
            same[b, :, h] = True
        assert bool(mine), f"{n} of the head itself"
        assert bool(same.all()), f"{n} of other heads"
