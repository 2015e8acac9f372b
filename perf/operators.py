"""What is timed of linear attention with a decay for each head and of the block norms.

A case is one call, or one training step (forward and backward), at one shape.

  op       "attend"   the recurrence S <- exp(g) S + k v^T, o = scale S^T q, on q, k (B, T, H, Dk)
                      and v (B, T, Hv, Dv), Hv a multiple of H:
             kind     "step" (a few tokens, the fp32 state updated in place), "prefill", "train"
             lengths  the sequences of a packed batch ("300,17,..."; B = 1, T their sum), or ""
             decay    "token": g (B, T, Hv), one value a token and head; "head": g (Hv,)
             shift    of the per-token decays, g = -softplus(N(0, 1) + shift)
             state    an initial state is given (training: and a gradient of the final one)
             saved    training: the forward keeps its segment states for the backward
           "norm"     rows of width D through RMSNorm, gate, residual sum and the next RMSNorm:
             kind     "fwd", "train"
             parts    which of them: p (norm after the block), g (SiLU gate), x (residual stream),
                      c (residual scale for each channel), n (norm before the next block)
             stream   the type of the residual stream
"""

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
ATTEND = dict(op="attend", B=1, T=1, H=16, Hv=16, Dk=128, Dv=128, dtype="bf16", lengths="", decay="token", shift=-2.0,
              state=False, saved=False)
NORM = dict(op="norm", rows=1, D=2048, dtype="bf16", stream="bf16", parts="pgxcn", kind="fwd")
EPS = 1e-6


def _attend(**kw):
    c = dict(ATTEND, **kw)
    if c["lengths"]:
        c["T"] = sum(_lengths(c))
    if "Hv" not in kw:
        c["Hv"] = c["H"]
    return c


def _norm(**kw):
    return dict(NORM, **kw)


def _lengths(case):
    return [int(x) for x in case["lengths"].split(",")]


def _states(case):
    return len(_lengths(case)) if case["lengths"] else case["B"]


def listed():
    return [
        # one user's next token at the 1.3B layer's heads: launch and call latency
        _attend(name="step_one", kind="step", state=True),
        # a full serving batch, one token each: the fp32 states go through memory once
        _attend(name="step_batch", kind="step", B=256, state=True),
        # continuous batching: most sequences take one token, some a few drafted or short-prompt tokens
        _attend(name="step_ragged", kind="step", state=True,
                lengths="1,1,4,1,1,1,8,1,1,1,5,1,1,1,1,3,1,1,1,1,1,16,1,1,1,4,1,1,1,1,1,8,1,1,1,1,2,1,1,1,1,5,1,1,1,1,1,1"),
        # one user's prompt, length as it comes, a fixed decay for each head
        _attend(name="prefill_prompt", kind="prefill", T=1000, decay="head"),
        # the prompts that arrived together, packed, grouped value heads, on top of earlier states
        _attend(name="prefill_packed", kind="prefill", H=8, Hv=16, state=True,
                lengths="37,2048,300,911,64,1500,129,3000,203"),
        # the 1.3B layer's training step at its 4K context
        _attend(name="train_layer", kind="train", B=8, T=4096, saved=True),
        # long-context training: one 64K sequence with slow decays
        _attend(name="train_long", kind="train", T=65536, state=True, shift=-4.0, saved=True),
        # 32-bit training of a small layer (numerical checks, ablations): odd length, grouped heads, fixed decays
        _attend(name="train_fp32", kind="train", B=2, T=1000, H=4, Hv=8, dtype="fp32", decay="head", state=True),
        # one token's head outputs through norm and output gate
        _norm(name="norm_step", rows=16, D=128, parts="pg"),
        # the same in training at the 1.3B layer's batch: a row for each token and head
        _norm(name="norm_heads_train", rows=8 * 4096 * 16, D=128, parts="pg", kind="train"),
        # between two blocks at that batch: norm, gate, layer scale, 32-bit residual stream, next norm
        _norm(name="norm_block_train", rows=8 * 4096, D=2048, stream="fp32", kind="train"),
        # an odd width in 32 bits, without gate
        _norm(name="norm_odd", rows=1999, D=1155, dtype="fp32", stream="fp32", parts="pxn", kind="train"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.4:
        c = dict(parts=rng.choice(["pg", "pg", "xn", "pxn", "xcn", "pgx", "pgxn", "pgxcn"]),
                 dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), kind=rng.choice(["fwd", "train", "train"]))
        c["stream"] = "fp32" if c["dtype"] == "fp32" or rng.random() < 0.4 else "bf16"
        c["D"] = rng.choice([64, 128, 128]) if c["parts"] == "pg" else _log(rng, 48, 8192)
        if c["parts"] != "pg" and rng.random() < 0.6:
            c["D"] = max(64, c["D"] // 64 * 64)
        c["rows"] = _log(rng, 1, 2 ** 26 // c["D"])
        return _norm(**c)
    kind = rng.choice(["step", "step", "prefill", "prefill", "train", "train", "train"])
    c = dict(kind=kind, H=rng.choice([2, 4, 8, 16, 16, 16]), shift=rng.choice([0.0, -2.0, -2.0, -4.0]),
             decay=rng.choice(["token", "token", "head"]))
    c["Dk"], c["Dv"] = rng.choice([(128, 128), (128, 128), (128, 128), (64, 128), (64, 64), (128, 64)])
    if rng.random() < 0.15:
        c["dtype"] = "fp32"
    if rng.random() < 0.2:
        c["Hv"] = c["H"] * 2
    Hv = c.get("Hv", c["H"])
    if kind == "step":
        c["state"] = True
        if rng.random() < 0.3:
            n = _log(rng, 2, 64)
            c["lengths"] = ",".join(str(rng.choice([1, 1, 1, 1, 1, rng.randint(2, 16)])) for _ in range(n))
        else:
            c["B"] = _log(rng, 1, 4096 // Hv)
            c["T"] = 1 if rng.random() < 0.7 else rng.randint(2, 16)
        return _attend(**c)
    # (token, value head) pairs: up to the training layer's count, 32-bit problems a 16th of it
    most = (8 * 4096 * 16) // (16 if c.get("dtype") == "fp32" else 1) // Hv
    if rng.random() < 0.3:
        total, left = _log(rng, 256, most), []
        while sum(left) < total and len(left) < 48:
            left.append(_log(rng, 16, min(4096, total)))
        left[-1] = max(1, left[-1] - max(0, sum(left) - total))
        c["lengths"] = ",".join(str(x) for x in left)
    else:
        c["T"] = _log(rng, 128, min(most, 65536))
        if rng.random() < 0.3:
            c["T"] = max(64, c["T"] // 64 * 64)
        c["B"] = _log(rng, 1, max(1, min(16, most // c["T"])))
    if kind == "train":
        c["saved"] = rng.random() < 0.7
    c["state"] = rng.random() < 0.4
    return _attend(**c)


def prepare(case, seed):
    """The tensors of one call, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if case["op"] == "norm":
        rows, D, parts, st = case["rows"], case["D"], case["parts"], DT[case["stream"]]
        x = dict(y=normal(rows, D).to(dt), w_post=None, gate=None, x=None, res_scale=None, w_pre=None, dh=None, dn=None)
        if "p" in parts:
            x["w_post"] = 1.0 + 0.1 * normal(D)
        if "g" in parts:
            x["gate"] = normal(rows, D).to(dt)
        if "x" in parts:
            x["x"] = (2.0 * normal(rows, D)).to(st)
        if "c" in parts:
            x["res_scale"] = 0.3 + 0.1 * normal(D)
        if "n" in parts:
            x["w_pre"] = 1.0 + 0.1 * normal(D)
        if case["kind"] == "train":
            x["dh"] = normal(rows, D).to(st if "x" in parts else dt)
            x["dn"] = normal(rows, D).to(dt) if "n" in parts else None
        return dict(case=dict(case), x=x)

    B, T, H, Hv, Dk, Dv = (case[n] for n in ("B", "T", "H", "Hv", "Dk", "Dv"))

    def rows(t):  # unit rows, as the layer hands q and k to its operator
        return (t / torch.sqrt((t * t).sum(dim=-1, keepdim=True))).to(dt)

    x = dict(q=rows(normal(B, T, H, Dk)), k=rows(normal(B, T, H, Dk)), v=normal(B, T, Hv, Dv).to(dt), S0=None, dout=None,
             dST=None, cu=None)
    if case["decay"] == "token":
        x["g"] = -torch.nn.functional.softplus(normal(B, T, Hv) + case["shift"])
    else:  # memories of about 8 to 500 tokens over the heads
        x["g"] = -torch.exp2(torch.linspace(-3.0, -9.0, Hv, device="cuda") + 0.1 * normal(Hv))
    if case["state"]:
        x["S0"] = 0.2 * normal(_states(case), Hv, Dk, Dv)
    if case["kind"] == "train":
        x["dout"] = normal(B, T, Hv, Dv).to(dt)
        if case["state"]:
            x["dST"] = 0.1 * normal(_states(case), Hv, Dk, Dv)
    if case["lengths"]:
        cu = [0]
        for n in _lengths(case):
            cu.append(cu[-1] + n)
        x["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    return dict(case=dict(case), x=x, longest=max(_lengths(case)) if case["lengths"] else T)


# ------------------------------------------------------------------ the framework's operators
def _own_attend(c, x):
    import paper_2605_22791_amd as g2
    args = x["q"], x["k"], x["v"], x["g"]
    if c["kind"] == "step":
        o = g2.gdr2_linattn_step(*args, x["S0"], cu_seqlens=x["cu"])
        return {"o": o, "S": x["S0"]}
    ws = None
    if c["saved"]:
        p = g2.Gdr2Problem(c["B"], c["T"], c["H"], c["Dk"], c["Dv"], g2.CHUNK, c["Dk"] ** -0.5,
                           g2.GDR2_BF16 if c["dtype"] == "bf16" else g2.GDR2_FP32, c["Hv"])
        need = g2.gdr2_linattn_workspace_bytes(p, _states(c) if c["lengths"] else 0, 1)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    o, S = g2.gdr2_linattn_fwd(*args, x["S0"], cu_seqlens=x["cu"], ws=ws, save=c["saved"])
    out = {"o": o, "S": S}
    if c["kind"] == "train":
        out.update(g2.gdr2_linattn_bwd(*args, x["S0"], x["dout"], x["dST"], cu_seqlens=x["cu"], ws=ws, saved=c["saved"]))
    return out


def _own_norm(c, x):
    import paper_2605_22791_amd as g2
    parts = {n: x[n] for n in ("w_post", "gate", "x", "res_scale", "w_pre")}
    h, n = g2.gdr2_blocknorm_fwd(x["y"], **parts, eps=EPS)
    out = {"h": h} if n is None else {"h": h, "n": n}
    if c["kind"] == "train":
        d = g2.gdr2_blocknorm_bwd(x["y"], x["dh"], x["dn"], **parts, eps=EPS)
        out.update({name: t for name, t in d.items() if t is not None})
    return out


# ------------------------------------------------------------------ the plain forms, in 32 bits
def _decays(g):
    """exp of the sums of g over s < j <= r, (..., r, s); zero above the diagonal."""
    n = g.shape[-1]
    below = torch.ones((n, n), dtype=torch.bool, device=g.device).tril(-1)
    sums = torch.where(below, g.unsqueeze(-1), 0.0).cumsum(dim=-2)
    return torch.where(below.triu(1 - n) | torch.eye(n, dtype=torch.bool, device=g.device), torch.exp(sums), 0.0)


def _plain_linear(q, k, v, g, S0, scale):
    """(N, T, H, D) sequences in blocks of up to 64 tokens; the states between blocks by one product over the blocks."""
    N, T, H, _ = q.shape
    C = min(64, T)

    def blocks(t):
        t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, -T % C))
        return t.reshape(N, -1, C, H, t.shape[-1]).permute(0, 3, 1, 2, 4)

    q, k, v, g = blocks(q), blocks(k), blocks(v), blocks(g.unsqueeze(-1)).squeeze(-1)
    D = _decays(g)
    inside = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * D, v)
    new = torch.matmul((k * D[..., -1, :].unsqueeze(-1)).transpose(-1, -2), v)
    between = _decays(torch.nn.functional.pad(g.sum(dim=-1), (1, 0)))
    every = torch.cat([S0.unsqueeze(2), new], dim=2)
    states = torch.matmul(between, every.flatten(3)).reshape(every.shape)
    o = inside + torch.matmul(q, states[:, :, :-1]) * torch.exp(g.cumsum(dim=-1)).unsqueeze(-1)
    return scale * o.permute(0, 2, 3, 1, 4).reshape(N, -1, H, v.shape[-1])[:, :T], states[:, :, -1]


def _plain_attend(s):
    c, x = s["case"], s["x"]
    dt, train = DT[c["dtype"]], c["kind"] == "train"
    G, ns = c["Hv"] // c["H"], _states(c)
    S0 = x["S0"] if x["S0"] is not None else torch.zeros((ns, c["Hv"], c["Dk"], c["Dv"]), device="cuda")
    p = dict(dq=x["q"].float(), dk=x["k"].float(), dv=x["v"].float(), dlog_decay=x["g"], dS0=S0)
    if train:
        p = {n: t.detach().clone().requires_grad_(True) for n, t in p.items()}
    with torch.set_grad_enabled(train):
        q, k, v = p["dq"].repeat_interleave(G, dim=2), p["dk"].repeat_interleave(G, dim=2), p["dv"]
        g = p["dlog_decay"] if c["decay"] == "token" else p["dlog_decay"].expand(c["B"], c["T"], c["Hv"])
        if c["lengths"]:  # a row for each sequence, zero past its end
            at = x["cu"][:-1, None].long() + torch.arange(s["longest"], device="cuda")
            there = at < x["cu"][1:, None]
            at = torch.where(there, at, 0)
            q, k, v = (torch.where(there[..., None, None], t[0, at], 0.0) for t in (q, k, v))
            g = torch.where(there[..., None], g[0, at], 0.0)
        o, S = _plain_linear(q, k, v, g, p["dS0"], c["Dk"] ** -0.5)
        if c["lengths"]:
            o = o[there].unsqueeze(0)
        if train:
            total = (o * x["dout"].float()).sum()
            if x["dST"] is not None:
                total = total + (S * x["dST"]).sum()
            d = dict(zip(p, torch.autograd.grad(total, list(p.values()))))
            d.update({n: d[n].to(dt) for n in ("dq", "dk", "dv")})
            return {"o": o.detach().to(dt), "S": S.detach(), **d}
    if c["kind"] == "step":
        S = x["S0"].copy_(S)
    return {"o": o.to(dt), "S": S}


def _plain_norm(s):
    c, x = s["case"], s["x"]
    dt, st = DT[c["dtype"]], DT[c["stream"]]
    names = dict(y="dy", w_post="dw_post", gate="dgate", x="dx", res_scale="dres_scale", w_pre="dw_pre")
    train = c["kind"] == "train"
    p = {n: None if x[n] is None else x[n].float() for n in names}
    if train:
        p = {n: None if t is None else t.detach().clone().requires_grad_(True) for n, t in p.items()}
    with torch.set_grad_enabled(train):
        a = p["y"]
        if p["w_post"] is not None:
            a = a * torch.rsqrt((a * a).mean(dim=-1, keepdim=True) + EPS) * p["w_post"]
        if p["gate"] is not None:
            a = a * (p["gate"] / (1.0 + torch.exp(-p["gate"])))
        if p["res_scale"] is not None:
            a = a * p["res_scale"]
        h = a if p["x"] is None else p["x"] + a
        ht = dt if p["x"] is None else st
        out = {"h": h.detach().to(ht)}
        n = None
        if p["w_pre"] is not None:
            n = h * torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + EPS) * p["w_pre"]
            out["n"] = n.detach().to(dt)
        if train:
            total = (h * x["dh"].float()).sum()
            if n is not None:
                total = total + (n * x["dn"].float()).sum()
            with_grad = {m: t for m, t in p.items() if t is not None}
            d = dict(zip(with_grad, torch.autograd.grad(total, list(with_grad.values()))))
            out.update({names[m]: t if m[:2] in ("w_", "re") else t.to(st if m == "x" else dt) for m, t in d.items()})
    return out


def run(s):
    c, x = s["case"], s["x"]
    if own:
        return _own_norm(c, x) if c["op"] == "norm" else _own_attend(c, x)
    return _plain_norm(s) if c["op"] == "norm" else _plain_attend(s)


def work(case):
    """Each input read once and each output written once; the recurrence takes 5 Dk Dv operations a
    token and head (decay, update, read-out) and its adjoint 12, a norm's element about 10 and 25."""
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n, parts, t = case["rows"] * case["D"], case["parts"], 2 if case["stream"] == "bf16" else 4
        h = t if "x" in parts else e
        fwd = e + ("g" in parts) * e + ("x" in parts) * t + h + ("n" in parts) * e
        bwd = 2 * e + ("g" in parts) * 2 * e + ("x" in parts) * 2 * t + h + ("n" in parts) * e
        train = case["kind"] == "train"
        wide = 4 * case["D"] * sum(p in parts for p in "pcn") * (2 if train else 1)
        return {"bytes": n * (fwd + (bwd if train else 0)) + wide, "flops": n * (35.0 if train else 10.0)}
    B, T, H, Hv, Dk, Dv = (case[n] for n in ("B", "T", "H", "Hv", "Dk", "Dv"))
    key, val, state = B * T * H * Dk, B * T * Hv * Dv, _states(case) * Hv * Dk * Dv * 4
    g = 4 * (B * T * Hv if case["decay"] == "token" else Hv)
    flops = 5.0 * B * T * Hv * Dk * Dv
    nbytes = 2 * key * e + 2 * val * e + g + state + (state if case["state"] else 0)
    if case["kind"] == "train":
        nbytes += 4 * key * e + 3 * val * e + 2 * g + state + (2 * state if case["state"] else 0)
        flops += 12.0 * B * T * Hv * Dk * Dv
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ the definitions, in 64 bits
BLOCK = 32


def _walk(q, k, v, g, S, scale):
    """One set of sequences (B, T, H, D), state (B, H, Dk, Dv), block after block."""
    B, T, H, _ = q.shape

    def blocks(t):
        t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, -T % BLOCK))
        return t.reshape(B, -1, BLOCK, H, t.shape[-1]).permute(0, 3, 1, 2, 4).contiguous()

    q, k, v, g = blocks(q), blocks(k), blocks(v), blocks(g.unsqueeze(-1))
    up = torch.exp(g.cumsum(dim=-2))
    q, kT = q * up, (k / up).transpose(-1, -2).contiguous()
    own_part = torch.matmul(torch.tril(torch.matmul(q, kT)), v)
    gain, last = torch.matmul(kT, v), up[..., -1:, :]
    outs = []
    for qn, a, n, d in zip(*(t.unbind(dim=2) for t in (q, own_part, gain, last))):
        outs.append(a + torch.matmul(qn, S))
        S = d * (S + n)
    o = scale * torch.stack(outs, dim=2)
    return o.permute(0, 2, 3, 1, 4).reshape(B, -1, H, v.shape[-1])[:, :T], S


def _exact_attend(c, x):
    train, G = c["kind"] == "train", c["Hv"] // c["H"]
    p = {n: x[n].double() for n in ("q", "k", "v", "g")}
    p["S"] = x["S0"].double() if x["S0"] is not None else torch.zeros(
        (_states(c), c["Hv"], c["Dk"], c["Dv"]), dtype=torch.float64, device="cuda")
    if train:
        p = {n: t.requires_grad_(True) for n, t in ((n, t.detach()) for n, t in p.items())}
    with torch.set_grad_enabled(train):
        q, k = (p[n].repeat_interleave(G, dim=2) for n in ("q", "k"))
        g = p["g"] if c["decay"] == "token" else p["g"] * torch.ones((c["B"], c["T"], 1), dtype=torch.float64, device="cuda")
        scale = c["Dk"] ** -0.5
        if c["lengths"]:
            os, Ss, at = [], [], 0
            for i, n in enumerate(_lengths(c)):
                o, S = _walk(*(t[:, at:at + n] for t in (q, k, p["v"], g)), p["S"][i:i + 1], scale)
                os.append(o)
                Ss.append(S)
                at += n
            o, S = torch.cat(os, dim=1), torch.cat(Ss)
        else:
            o, S = _walk(q, k, p["v"], g, p["S"], scale)
        out = {"o": o.detach(), "S": S.detach()}
        if train:
            loss = (o * x["dout"].double()).sum()
            if x["dST"] is not None:
                loss = loss + (S * x["dST"].double()).sum()
            loss.backward()
            names = {"dq": "q", "dk": "k", "dv": "v", "dlog_decay": "g", "dS0": "S"}
            out.update({n: p[m].grad for n, m in names.items()})
    return out


def _exact_norm(c, x):
    """The formulas and their gradients, written out."""
    y, wp, z, r, cs, wn, dh, dn = (None if x[n] is None else x[n].double() for n in (
        "y", "w_post", "gate", "x", "res_scale", "w_pre", "dh", "dn"))
    one = torch.ones((), dtype=torch.float64, device="cuda")
    ry = one if wp is None else 1.0 / torch.sqrt((y ** 2).mean(dim=-1, keepdim=True) + EPS)
    u = y * ry * (one if wp is None else wp)
    sg = one if z is None else torch.sigmoid(z)
    gate = one if z is None else z * sg
    a = u * gate
    ca = a * (one if cs is None else cs)
    h = ca if r is None else r + ca
    out = {"h": h}
    if wn is not None:
        rh = 1.0 / torch.sqrt((h ** 2).mean(dim=-1, keepdim=True) + EPS)
        out["n"] = h * rh * wn
    if c["kind"] != "train":
        return out
    full = dh
    if wn is not None:
        t = dn * wn
        full = dh + rh * (t - h * rh ** 2 * (t * h).mean(dim=-1, keepdim=True))
        out["dw_pre"] = (dn * h * rh).sum(dim=0)
    if r is not None:
        out["dx"] = full
    if cs is not None:
        out["dres_scale"] = (full * a).sum(dim=0)
    da = full * (one if cs is None else cs)
    if z is not None:
        out["dgate"] = da * u * sg * (1.0 + z * (1.0 - sg))
    du = da * gate
    if wp is None:
        out["dy"] = du
    else:
        out["dw_post"] = (du * y * ry).sum(dim=0)
        t = du * wp
        out["dy"] = ry * (t - y * ry ** 2 * (t * y).mean(dim=-1, keepdim=True))
    return out


def exact(case, seed):
    x = prepare(case, seed)["x"]
    return _exact_norm(case, x) if case["op"] == "norm" else _exact_attend(case, x)
