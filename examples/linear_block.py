"""Blocks of linear attention from the two operators, trained and decoded.

A block, with a 32-bit residual stream x and its norm n in bfloat16:

    q, k, v, z, f = projections of n          (torch)
    o    = linear attention of q, k, v, g = -softplus(f + bias)     gdr2_linattn_fwd / _bwd / _step
    a    = norm of o over each head, gated by z                     gdr2_blocknorm_fwd / _bwd
    x, n = x + c * (a W), and its norm for the next block           gdr2_blocknorm_fwd / _bwd

`python examples/linear_block.py` trains two blocks to say the token before the current
one, then decodes: the prompt in one chunk call, the rest token by token, beside the logits
of the chunk call over everything.  Needs a GPU and the built library.
"""

import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2605_22791_amd as g2  # noqa: E402


def once():
    """Of a backward: the kernels' results carry no graph, so under create_graph=True terms would be left out silently."""
    if torch.is_grad_enabled():
        raise RuntimeError("the operators have no second derivative: create_graph=True is not supported")


class Attention(torch.autograd.Function):
    """o, S_T of linear attention; the workspace takes the forward's states to the backward."""

    @staticmethod
    def forward(ctx, q, k, v, g, S0):
        B, T, H, Dk = q.shape
        p = g2.Gdr2Problem(B, T, H, Dk, v.shape[3], g2.CHUNK, Dk ** -0.5,
                           g2.GDR2_BF16 if q.dtype == torch.bfloat16 else g2.GDR2_FP32, v.shape[2])
        ws = torch.empty(g2.gdr2_linattn_workspace_bytes(p, 0, 1), dtype=torch.uint8, device=q.device)
        o, S = g2.gdr2_linattn_fwd(q, k, v, g, S0, ws=ws, save=True)
        ctx.save_for_backward(q, k, v, g, S0, ws)
        return o, S

    @staticmethod
    def backward(ctx, do, dS):
        once()
        q, k, v, g, S0, ws = ctx.saved_tensors
        d = g2.gdr2_linattn_bwd(q, k, v, g, S0, do.contiguous(), dS.contiguous(), want_dS0=S0 is not None, ws=ws,
                                saved=True)
        return d["dq"], d["dk"], d["dv"], d["dlog_decay"], d["dS0"]


class BlockNorm(torch.autograd.Function):
    """h, n of the block norms (None for what a call does not have)."""

    @staticmethod
    def forward(ctx, y, w_post, gate, x, res_scale, w_pre):
        h, n = g2.gdr2_blocknorm_fwd(y, w_post=w_post, gate=gate, x=x, res_scale=res_scale, w_pre=w_pre)
        ctx.save_for_backward(y, w_post, gate, x, res_scale, w_pre)
        return h, n

    @staticmethod
    def backward(ctx, dh, dn):
        once()
        y, w_post, gate, x, res_scale, w_pre = ctx.saved_tensors
        d = g2.gdr2_blocknorm_bwd(y, dh.contiguous(), None if w_pre is None else dn.contiguous(), w_post=w_post, gate=gate,
                                  x=x, res_scale=res_scale, w_pre=w_pre)
        return d["dy"], d["dw_post"], d["dgate"], d["dx"], d["dres_scale"], d["dw_pre"]


class Block(torch.nn.Module):
    def __init__(self, width, heads, dim):
        super().__init__()
        self.heads, self.dim = heads, dim
        inner = heads * dim
        self.w_in = torch.nn.Parameter(torch.randn(width, 4 * inner + heads) * width ** -0.5)
        self.w_out = torch.nn.Parameter(torch.randn(inner, width) * inner ** -0.5)
        self.bias = torch.nn.Parameter(torch.linspace(-4.0, 0.0, heads))  # slow and fast heads
        self.w_post = torch.nn.Parameter(torch.ones(dim))
        self.scale = torch.nn.Parameter(torch.full((width,), 0.5))
        self.w_next = torch.nn.Parameter(torch.ones(width))  # of the norm before the next block

    def forward(self, n, x, S=None, step=False):
        """n, x (B, T, width) and a state or None; returns n, x of the next block and the state after."""
        B, T, _ = n.shape
        inner = self.heads * self.dim
        q, k, v, z, f = (n @ self.w_in.to(n.dtype)).split([inner] * 4 + [self.heads], dim=-1)
        q, k, v, z = (t.reshape(B, T, self.heads, self.dim) for t in (q, k, v, z))
        g = -F.softplus(f.float() + self.bias)
        if step:
            o = g2.gdr2_linattn_step(q.contiguous(), k.contiguous(), v.contiguous(), g.contiguous(), S)
        else:
            o, S = Attention.apply(q.contiguous(), k.contiguous(), v.contiguous(), g.contiguous(), S)
        a, _ = BlockNorm.apply(o, self.w_post, z.contiguous(), None, None, None)
        y = a.reshape(B, T, inner) @ self.w_out.to(n.dtype)
        x, n = BlockNorm.apply(y, None, None, x, self.scale, self.w_next)
        return n, x, S


class Model(torch.nn.Module):
    def __init__(self, vocab=32, width=192, heads=3, dim=64, blocks=2):
        super().__init__()
        self.embed = torch.nn.Parameter(torch.randn(vocab, width))
        self.w_first = torch.nn.Parameter(torch.ones(width))
        self.blocks = torch.nn.ModuleList(Block(width, heads, dim) for _ in range(blocks))
        self.w_logits = torch.nn.Parameter(torch.randn(width, vocab) * width ** -0.5)

    def forward(self, tokens, states=None, step=False):
        e = self.embed[tokens]
        x = e.float()
        _, n = BlockNorm.apply(e.to(torch.bfloat16), None, None, None, None, self.w_first)
        states = states or [None] * len(self.blocks)
        after = []
        for block, S in zip(self.blocks, states):
            n, x, S = block(n, x, S, step)
            after.append(S)
        return (n @ self.w_logits.to(n.dtype)).float(), after


def train(steps=150, batch=16, length=96, seed=0, device="cuda"):
    """Trains to say, at each of `length` random tokens, the one before it, which only the state can hold; returns
    the model and the losses."""
    torch.manual_seed(seed)
    model = Model().to(device)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for _ in range(steps):
        tokens = torch.randint(0, model.embed.shape[0], (batch, length), device=device)
        logits, _ = model(tokens)
        loss = F.cross_entropy(logits[:, 1:].reshape(-1, logits.shape[-1]), tokens[:, :-1].reshape(-1))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return model, losses


@torch.no_grad()
def decode(model, tokens, prompt):
    """Logits of tokens (B, T): the first `prompt` in one chunk call, the others one at a time."""
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
    print("decoding beside the chunk call: relative difference %.2g" % float((apart - whole).norm() / whole.norm()))


if __name__ == "__main__":
    main()
