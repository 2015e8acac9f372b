"""Layers of a gated linear recurrence and a gated feed-forward block, trained and decoded.

A layer, with a 32-bit residual stream x and its norm n in bfloat16:

    v, i, f, z = projections of n, i through the logistic function       (torch)
    o    = gated recurrence of v with input gate i, g = -softplus(f + bias)   gdr2_gatedrec_fwd / _bwd / _step
    a    = o gated by silu(z)                                            gdr2_blocknorm_fwd / _bwd
    x    = x + dropout(a W)                                              gdr2_dropout_fwd / _bwd
    n    = norm of x                                                     gdr2_blocknorm_fwd / _bwd
    x    = x + dropout(feed-forward of n)                                gdr2_gatedff_fwd / _bwd, gdr2_dropout_fwd / _bwd
    n    = norm of x, for the next layer                                 gdr2_blocknorm_fwd / _bwd

`python examples/recurrent_block.py` trains two layers to say the token before the current one, then
decodes: the prompt in one call, the rest token by token, beside the logits of one call over
everything.  Needs a GPU and the built library.
"""

import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2605_22791_amd as g2  # noqa: E402
from linear_block import BlockNorm, once  # noqa: E402


def _code(t):
    return g2.GDR2_BF16 if t.dtype == torch.bfloat16 else g2.GDR2_FP32


class Recurrence(torch.autograd.Function):
    """o, h_T of the normalized gated recurrence; the workspace takes the forward's states to the backward."""

    @staticmethod
    def forward(ctx, v, g, i, h0):
        B, T, D = v.shape
        p = g2.Gdr2Gatedrec(B, T, D, _code(v), 1)
        ws = torch.empty(g2.gdr2_gatedrec_workspace_bytes(p, 0, 1), dtype=torch.uint8, device=v.device)
        o, h = g2.gdr2_gatedrec_fwd(v, g, i, h0, normalize=True, ws=ws, save=True)
        ctx.save_for_backward(v, g, i, h0, ws)
        return o, h

    @staticmethod
    def backward(ctx, do, dh):
        once()
        v, g, i, h0, ws = ctx.saved_tensors
        d = g2.gdr2_gatedrec_bwd(v, g, i, h0, do.contiguous(), dh.contiguous(), normalize=True, want_dh0=h0 is not None, ws=ws,
                                 saved=True)
        return d["dx"], d["dlog_decay"], d["dgate"], d["dh0"]


class FeedForward(torch.autograd.Function):
    """The gated feed-forward block; the workspace takes its hidden values to the backward."""

    @staticmethod
    def forward(ctx, n, w_gate, w_up, w_down):
        p = g2.Gdr2Gatedff(n.numel() // n.shape[-1], n.shape[-1], w_gate.shape[0], _code(n), g2.GDR2_ACT_SILU)
        ws = torch.empty(g2.gdr2_gatedff_workspace_bytes(p, 1), dtype=torch.uint8, device=n.device)
        y = g2.gdr2_gatedff_fwd(n, w_gate, w_up, w_down, ws=ws, save=True)
        ctx.save_for_backward(n, w_gate, w_up, w_down, ws)
        return y

    @staticmethod
    def backward(ctx, dy):
        once()
        *args, ws = ctx.saved_tensors
        d = g2.gdr2_gatedff_bwd(*args, dy.contiguous(), ws=ws, saved=True)
        return d["dx"], d["dw_gate"], d["dw_up"], d["dw_down"]


def recurrence(v, g, i, h0):
    """o, h_T; nothing is kept where no gradient will be asked for."""
    return Recurrence.apply(v, g, i, h0) if torch.is_grad_enabled() else g2.gdr2_gatedrec_fwd(v, g, i, h0, normalize=True)


def feed_forward(n, w_gate, w_up, w_down):
    """Decoding, a call that keeps nothing: few rows then take the kernels made for them."""
    return (FeedForward.apply if torch.is_grad_enabled() else g2.gdr2_gatedff_fwd)(n, w_gate, w_up, w_down)


class Dropout(torch.autograd.Function):
    """residual + dropout(y); the backward forms the mask again from the seed and the offset."""

    @staticmethod
    def forward(ctx, y, residual, p, seed, offset):
        ctx.how = p, seed, offset, y.dtype
        return g2.gdr2_dropout_fwd(y, p, seed, offset=offset, residual=residual)

    @staticmethod
    def backward(ctx, d):
        once()
        p, seed, offset, dtype = ctx.how
        d = d.contiguous()
        return g2.gdr2_dropout_bwd(d, p, seed, offset=offset, dtype=dtype), d, None, None, None


class Layer(torch.nn.Module):
    def __init__(self, width, inner, hidden, site):
        super().__init__()
        self.site = site  # tells this layer's dropouts from the others'
        par = lambda *s: torch.nn.Parameter(torch.randn(s) * s[-1] ** -0.5)  # noqa: E731
        self.w_in, self.w_out = par(4 * inner, width), par(width, inner)
        self.bias = torch.nn.Parameter(torch.linspace(-5.0, 1.0, inner))  # slow and fast channels
        self.w_mid, self.w_next = (torch.nn.Parameter(torch.ones(width)) for _ in range(2))  # of the norms
        self.w_gate, self.w_up, self.w_down = par(hidden, width), par(hidden, width), par(width, hidden)

    def forward(self, n, x, h, step, drop):
        """n, x (B, T, width), a state or None, whether to go token by token, and (p, seed, number of the pass); returns
        n, x of the next layer and the state after."""
        dt = n.dtype
        v, i, f, z = (n @ self.w_in.t().to(dt)).chunk(4, dim=-1)
        v, i, z = v.contiguous(), torch.sigmoid(i).contiguous(), z.contiguous()
        g = -F.softplus(f.float() + self.bias).contiguous()
        if step:
            o = g2.gdr2_gatedrec_step(v, g, i, h, normalize=True)
        else:
            o, h = recurrence(v, g, i, h)
        a, _ = BlockNorm.apply(o, None, z, None, None, None)
        p, seed, number = drop
        at = (number << 16) + 2 * self.site  # an offset of its own for each dropout of each pass
        x = Dropout.apply(a @ self.w_out.t().to(dt), x, p, seed, at)
        _, n = BlockNorm.apply(x, None, None, None, None, self.w_mid)
        y = feed_forward(n.to(dt), self.w_gate.to(dt), self.w_up.to(dt), self.w_down.to(dt))
        x = Dropout.apply(y, x, p, seed, at + 1)
        _, n = BlockNorm.apply(x, None, None, None, None, self.w_next)
        return n.to(dt), x, h


class Model(torch.nn.Module):
    def __init__(self, vocab=32, width=192, inner=320, hidden=512, layers=2):
        super().__init__()
        self.embed = torch.nn.Parameter(torch.randn(vocab, width))
        self.w_first = torch.nn.Parameter(torch.ones(width))
        self.layers = torch.nn.ModuleList(Layer(width, inner, hidden, k) for k in range(layers))
        self.w_logits = torch.nn.Parameter(torch.randn(width, vocab) * width ** -0.5)

    def forward(self, tokens, states=None, step=False, drop=(0.0, 0, 0)):
        x = self.embed[tokens].float()
        _, n = BlockNorm.apply(x, None, None, None, None, self.w_first)
        n = n.to(torch.bfloat16)
        after = []
        for layer, h in zip(self.layers, states or [None] * len(self.layers)):
            n, x, h = layer(n, x, h, step, drop)
            after.append(h)
        return (n @ self.w_logits.to(n.dtype)).float(), after


def train(steps=150, batch=16, length=96, seed=0, p=0.1, device="cuda"):
    """Trains to say, at each of `length` random tokens, the one before it, which only the state can hold; returns
    the model and the losses."""
    torch.manual_seed(seed)
    model = Model().to(device)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for number in range(steps):
        tokens = torch.randint(0, model.embed.shape[0], (batch, length), device=device)
        logits, _ = model(tokens, drop=(p, seed, number))
        loss = F.cross_entropy(logits[:, 1:].reshape(-1, logits.shape[-1]), tokens[:, :-1].reshape(-1))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return model, losses


@torch.no_grad()
def decode(model, tokens, prompt):
    """Logits of tokens (B, T): the first `prompt` in one call, the others one at a time."""
    logits, states = model(tokens[:, :prompt])
    out = [logits]
    for t in range(prompt, tokens.shape[1]):
        logits, states = model(tokens[:, t:t + 1], states, step=True)
        out.append(logits)
    return torch.cat(out, dim=1)


def main():
    model, losses = train()
    print("loss: first %.3f, last %.3f" % (losses[0], losses[-1]))
    tokens = torch.randint(0, model.embed.shape[0], (4, 150), device="cuda")
    with torch.no_grad():
        whole, _ = model(tokens)
    apart = decode(model, tokens, 100)
    print("decoding beside the call over everything: relative difference %.2g" % float((apart - whole).norm() / whole.norm()))


if __name__ == "__main__":
    main()
