"""The gated recurrence, dropout with the residual sum, the block norms and the gated feed-forward block one
after the other, as a layer has them; and the example that trains and decodes such layers."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle.dropout import dropout_keep

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "recurrent_block.py")
    spec = importlib.util.spec_from_file_location("recurrent_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_layer_against_64_bits(dtype):
    """x -> norm -> recurrence -> x + dropout -> norm -> feed-forward -> x + dropout, and every gradient.

    fp32: four operators, each good to some 5e-6 of what it is given, behind one another, forward and
    backward: 5e-5.  bf16: the values that are rounded on the way, each by 2^-8 / sqrt 3 = 2.3e-3 in the mean square:
    n, o, n, h, y forward, and backward dy, dg and du (one factor), dn, do, dx, dn: up to twelve in one
    gradient, sqrt(12) 2.3e-3 = 8e-3 if they fall differently; 1.2e-2."""
    import paper_2605_22791_amd as g2
    print(f"layer {dtype}", flush=True)
    B, T, D, Fh, p, seed = 2, 300, 136, 264, 0.2, 5
    gen = torch.Generator(device="cuda").manual_seed(3)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x0, w1, w2 = f(B, T, D), 1 + 0.1 * f(D), 1 + 0.1 * f(D)
    g = -torch.nn.functional.softplus(f(B, T, D) - 2)
    i = torch.sigmoid(f(B, T, D)).to(dtype)
    wg, wu, wd = (f(Fh, D) * D ** -0.5).to(dtype), (f(Fh, D) * D ** -0.5).to(dtype), (f(D, Fh) * Fh ** -0.5).to(dtype)
    dout = f(B, T, D)

    # the operators; the stream is 32-bit, the norms' inputs are it
    _, n1 = g2.gdr2_blocknorm_fwd(x0, w_pre=w1)
    o, h = g2.gdr2_gatedrec_fwd(n1.to(dtype), g, i, normalize=True)
    x1 = g2.gdr2_dropout_fwd(o, p, seed, offset=1, residual=x0)
    _, n2 = g2.gdr2_blocknorm_fwd(x1, w_pre=w2)
    n2d = n2.to(dtype)
    y = g2.gdr2_gatedff_fwd(n2d, wg, wu, wd)
    x2 = g2.gdr2_dropout_fwd(y, p, seed, offset=2, residual=x1)
    ff = g2.gdr2_gatedff_bwd(n2d, wg, wu, wd, g2.gdr2_dropout_bwd(dout, p, seed, offset=2, dtype=dtype))
    b2 = g2.gdr2_blocknorm_bwd(x1, dout, ff["dx"].float(), w_pre=w2)  # dout: the residual's gradient
    rec = g2.gdr2_gatedrec_bwd(n1.to(dtype), g, i, None, g2.gdr2_dropout_bwd(b2["dy"], p, seed, offset=1, dtype=dtype),
                               normalize=True, want_dh0=False)
    b1 = g2.gdr2_blocknorm_bwd(x0, b2["dy"], rec["dx"].float(), w_pre=w1)
    got = dict(x2=x2, h=h, x0=b1["dy"], w1=b1["dw_pre"], w2=b2["dw_pre"], g=rec["dlog_decay"], i=rec["dgate"], wg=ff["dw_gate"],
               wu=ff["dw_up"], wd=ff["dw_down"])

    # 64 bits
    q = {n: t.double().requires_grad_(True) for n, t in dict(x0=x0, w1=w1, w2=w2, g=g, i=i, wg=wg, wu=wu, wd=wd).items()}
    keep = [torch.from_numpy(dropout_keep(x0.numel(), p, seed, k).reshape(B, T, D)).cuda() for k in (1, 2)]
    norm = lambda t, w: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
    u = torch.sqrt(-torch.expm1(2 * q["g"])) * q["i"] * norm(q["x0"], q["w1"])
    s, os = torch.zeros((B, D), dtype=torch.float64, device="cuda"), []
    for t in range(T):
        s = torch.exp(q["g"][:, t]) * s + u[:, t]
        os.append(s)
    a1 = q["x0"] + torch.where(keep[0], torch.stack(os, 1) / (1 - p), 0.0)
    m2 = norm(a1, q["w2"]).reshape(B * T, D)
    yy = (torch.nn.functional.silu(m2 @ q["wg"].T) * (m2 @ q["wu"].T)) @ q["wd"].T
    a2 = a1 + torch.where(keep[1], yy.reshape(B, T, D) / (1 - p), 0.0)
    a2.backward(dout.double())
    want = dict(x2=a2.detach(), h=s.detach(), **{n: t.grad for n, t in q.items()})
    tol = 5e-5 if dtype == torch.float32 else 1.2e-2
    for n in want:
        e = float((got[n].double() - want[n]).norm() / want[n].norm())
        print(f"{n} {e:.1e}", end="  ", flush=True)
        assert e < tol, (n, e)


def test_a_layer_in_one_graph():
    """The whole run captured once and replayed, other elements dropped each time."""
    import paper_2605_22791_amd as g2
    print("a layer in a graph", flush=True)
    B, T, D, Fh = 1, 700, 192, 256
    f = lambda *s: torch.randn(s, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, wg, wu, wd, w = torch.randn((B, T, D), device="cuda"), f(Fh, D), f(Fh, D), f(D, Fh), torch.ones(D, device="cuda")
    g, at = -torch.rand((B, T, D), device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def run(at):
        _, n = g2.gdr2_blocknorm_fwd(x, w_pre=w)
        n = n.to(torch.bfloat16)
        o, _ = g2.gdr2_gatedrec_fwd(n, g)
        x1 = g2.gdr2_dropout_fwd(o, 0.3, 9, offset=at, residual=x)
        _, n = g2.gdr2_blocknorm_fwd(x1, w_pre=w)
        n = n.to(torch.bfloat16)
        y = g2.gdr2_gatedff_fwd(n, wg, wu, wd)
        d = g2.gdr2_gatedff_bwd(n, wg, wu, wd, y)
        r = g2.gdr2_gatedrec_bwd(n, g, None, None, d["dx"])
        return [x1, y, r["dx"], r["dlog_decay"], d["dw_gate"], d["dw_down"]]

    run(at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(at)
    for k in range(4):
        at.fill_(k)
        graph.replay()
        want = run(k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_training_runs(example):
    print("training 20 steps", flush=True)
    _, losses = example.train(steps=20)
    assert all(np.isfinite(losses))


@pytest.mark.parametrize("prompt", [1, 63, 64, 100])
def test_decoding_agrees_with_one_call(example, prompt):
    print(f"decoding after a prompt of {prompt}", flush=True)
    torch.manual_seed(1)
    model = example.Model().to("cuda")
    tokens = torch.randint(0, 32, (3, 130), device="cuda")
    with torch.no_grad():
        whole, _ = model(tokens)
    apart = example.decode(model, tokens, prompt)
    # both round the same values to bfloat16 on their way: nine in a layer (v, i, z as one, f, o, a, its
    # projection, n, h, y, n) and the logits, each by 2^-8 / sqrt 3 in the mean square at most, and they agree but where
    # a sum of another order falls on the other side: sqrt(19) 2.3e-3 = 1e-2 if every rounding fell differently
    assert float((apart - whole).norm() / whole.norm()) < 1e-2


def test_gradients_follow_differences(example):
    """One step against the gradient lowers the loss by |gradient|^2 times its length, to first order, the same
    elements dropped."""
    torch.manual_seed(2)
    model = example.Model(layers=1).to("cuda")
    tokens = torch.randint(0, 32, (2, 200), device="cuda")

    def loss():
        logits, _ = model(tokens[:, :-1], drop=(0.1, 3, 4))
        return torch.nn.functional.cross_entropy(logits.reshape(-1, 32), tokens[:, 1:].reshape(-1))

    a = loss()
    a.backward()
    size = sum(float((q.grad.double() ** 2).sum()) for q in model.parameters())
    step = 0.05 * float(a.detach()) / size  # a predicted fall of 5 %: well over bfloat16's 0.4 %, small beside curvature
    with torch.no_grad():
        for q in model.parameters():
            q -= step * q.grad
        b = loss()
    fall = (float(a.detach()) - float(b)) / (step * size)
    assert 0.5 < fall < 1.5, fall


def test_a_second_derivative_is_refused(example):
    print("second derivatives", flush=True)
    x = torch.randn(1, 20, 64, device="cuda").to(torch.bfloat16).requires_grad_(True)
    w, wd = torch.randn(72, 64, device="cuda").to(torch.bfloat16), torch.randn(64, 72, device="cuda").to(torch.bfloat16)
    for y in (example.Recurrence.apply(x, -torch.rand(1, 20, 64, device="cuda"), x.detach(), None)[0],
              example.FeedForward.apply(x, w, w, wd), example.Dropout.apply(x, x.detach().float(), 0.1, 1, 2)):
        with pytest.raises(RuntimeError, match="second derivative"):
            d, = torch.autograd.grad(y.float().sum(), x, create_graph=True)
            (x.float() ** 2 + d.float() ** 2).sum().backward()
