"""What is timed of the gated linear recurrence, the gated feed-forward block and dropout with the residual sum.

A case is one call, or one training step (forward and backward), at one shape.

  op       "rec"      h_t = exp(g_t) h_{t-1} + m_t i_t x_t for each channel, on x, i, g (B, T, D):
             kind     "step" (a few tokens, the fp32 state updated in place), "prefill", "train"
             lengths  the sequences of a packed batch ("300,17,..."; B = 1, T their sum), or ""
             gate     there is an input gate i (else 1)
             unit     m = sqrt(1 - exp(2 g)), which keeps the variance (else 1)
             shift    of the decays, g = -softplus(N(0, 1) + shift)
             state    an initial state is given (training: and a gradient of the final one)
             saved    training: the forward keeps its states for the backward
           "ff"       y = (act(x Wg^T) * (x Wu^T)) Wd^T on rows of width D, F hidden channels:
             kind     "fwd", "train"
             act      "silu", "gelu"
             saved    training: the forward keeps its hidden values for the backward
           "drop"     y = residual + keep * x / (1 - p), keep from a counter-based generator:
             kind     "fwd", "train"
             stream   the type of the residual stream; "" without one
"""

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
REC = dict(op="rec", kind="train", B=1, T=1, D=2048, dtype="bf16", lengths="", gate=True, unit=True, shift=-2.0,
           state=False, saved=False)
FF = dict(op="ff", kind="fwd", rows=1, D=2048, F=5504, dtype="bf16", act="silu", saved=False)
DROP = dict(op="drop", kind="train", rows=1, D=2048, dtype="bf16", stream="bf16", p=0.1)


def _rec(**kw):
    c = dict(REC, **kw)
    if c["lengths"]:
        c["T"] = sum(_lengths(c))
    return c


def _lengths(case):
    return [int(x) for x in case["lengths"].split(",")] if case["lengths"] else [case["T"]] * case["B"]


def listed():
    return [
        # one user's next token: launch and call latency
        _rec(name="rec_step_one", kind="step", state=True),
        # a full serving batch, one token each
        _rec(name="rec_step_batch", kind="step", B=256, state=True),
        # the prompts that arrived together, packed, on top of earlier states
        _rec(name="rec_prefill_packed", kind="prefill", state=True, lengths="37,2048,300,911,64,1500,129,3000,203"),
        # a layer's training step at a 4K context
        _rec(name="rec_train_layer", B=8, T=4096, saved=True),
        # long-context training: one 64K sequence with slow decays, no input gate, the input as it is
        _rec(name="rec_train_long", T=65536, state=True, gate=False, unit=False, shift=-4.0, saved=True),
        # 32-bit training of a small layer (numerical checks, ablations): odd length and width
        _rec(name="rec_train_fp32", B=2, T=1001, D=1155, dtype="fp32", state=True),
        # one user's next token: the weights go through memory once
        dict(FF, name="ff_step"),
        # one user's prompt, length as it comes
        dict(FF, name="ff_prompt", rows=1000),
        # a layer's training step at the batch of rec_train_layer
        dict(FF, name="ff_train", kind="train", rows=8 * 4096, saved=True),
        # 32-bit training of a small block, odd row count, GELU, hidden values formed again
        dict(FF, name="ff_train_fp32", kind="train", rows=777, D=520, F=1368, dtype="fp32", act="gelu"),
        # a fine-tuning step's short batch of odd width in 32 bits, without a residual stream
        dict(DROP, name="drop_small", rows=257, D=1155, dtype="fp32", stream=""),
        # between two blocks at the training batch: 32-bit residual stream beside bf16 blocks
        dict(DROP, name="drop_train", rows=8 * 4096, stream="fp32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rec", "rec", "rec", "ff", "ff", "drop"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    if op == "drop":
        D = _log(rng, 32, 8192)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        return dict(DROP, rows=_log(rng, 1, 2 ** 26 // D), D=D, dtype=dtype, kind=rng.choice(["fwd", "train", "train"]),
                    stream=rng.choice(["", "fp32", "fp32" if dtype == "fp32" else "bf16"]), p=rng.choice([0.05, 0.1, 0.1, 0.3, 0.5]))
    if op == "ff":
        D = _log(rng, 128, 4096) // 8 * 8
        F = min(16384, int(D * rng.uniform(1.0, 4.0))) // 8 * 8
        if rng.random() < 0.5:
            D, F = max(128, D // 128 * 128), max(128, F // 128 * 128)
        most = (8 * 4096 * 2048 * 5504) // (32 if dtype == "fp32" else 1) // (D * F)
        kind = rng.choice(["fwd", "fwd", "train", "train", "train"])
        return dict(FF, D=D, F=F, rows=_log(rng, 1 if kind == "fwd" else 64, max(64, min(65536, most))), dtype=dtype, kind=kind,
                    act=rng.choice(["silu", "silu", "gelu"]), saved=kind == "train" and rng.random() < 0.6)
    kind = rng.choice(["step", "prefill", "prefill", "train", "train", "train"])
    c = dict(kind=kind, dtype=dtype, D=_log(rng, 64, 8192), gate=rng.random() < 0.6, unit=rng.random() < 0.5,
             shift=rng.choice([0.0, -2.0, -2.0, -4.0]), state=kind == "step" or rng.random() < 0.4)
    if rng.random() < 0.7:
        c["D"] = max(64, c["D"] // 64 * 64)
    if kind == "step":
        if rng.random() < 0.3:
            c["lengths"] = ",".join(str(rng.choice([1, 1, 1, 1, 1, rng.randint(2, 16)])) for _ in range(_log(rng, 2, 64)))
        else:
            c["B"] = _log(rng, 1, 512)
            c["T"] = 1 if rng.random() < 0.7 else rng.randint(2, 16)
        return _rec(**c)
    most = min(2 ** 26 // c["D"], 65536)
    if rng.random() < 0.3:
        total, left = _log(rng, min(256, most), most), []
        while sum(left) < total and len(left) < 48:
            left.append(_log(rng, 1, min(8192, total)))
        left[-1] = max(1, left[-1] - max(0, sum(left) - total))
        c["lengths"] = ",".join(str(x) for x in left)
    else:
        c["T"] = _log(rng, min(128, most), most)
        c["B"] = _log(rng, 1, max(1, min(16, most // c["T"])))
    c["saved"] = kind == "train" and rng.random() < 0.7
    return _rec(**c)


def prepare(case, seed):
    """The tensors of one call, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if case["op"] == "drop":
        rows, D, st = case["rows"], case["D"], DT[case["stream"] or case["dtype"]]
        x = dict(x=normal(rows, D).to(dt), residual=None, dy=None)
        if case["stream"]:
            x["residual"] = (2.0 * normal(rows, D)).to(st)
        if case["kind"] == "train":
            x["dy"] = normal(rows, D).to(st)
        # a seed over the whole 64 bits; the offset a training loop's step count
        return dict(case=dict(case), x=x, key=(seed * 0x9E3779B97F4A7C15 + 0x1234567) % 2 ** 64, offset=(5 << 32) + seed % 1000)
    if case["op"] == "ff":
        rows, D, F = case["rows"], case["D"], case["F"]
        x = dict(x=normal(rows, D).to(dt), w_gate=(normal(F, D) * D ** -0.5).to(dt), w_up=(normal(F, D) * D ** -0.5).to(dt),
                 w_down=(normal(D, F) * F ** -0.5).to(dt), dy=normal(rows, D).to(dt) if case["kind"] == "train" else None)
        return dict(case=dict(case), x=x)
    B, T, D = case["B"], case["T"], case["D"]
    n = len(_lengths(case))
    x = dict(x=normal(B, T, D).to(dt), g=-torch.nn.functional.softplus(normal(B, T, D) + case["shift"]), gate=None, h0=None,
             dout=None, dhT=None, cu=None)
    if case["gate"]:
        x["gate"] = torch.sigmoid(normal(B, T, D)).to(dt)
    if case["state"]:
        x["h0"] = normal(n, D)
    if case["kind"] == "train":
        x["dout"] = normal(B, T, D).to(dt)
        if case["state"]:
            x["dhT"] = normal(n, D)
    if case["lengths"]:
        cu = [0]
        for m in _lengths(case):
            cu.append(cu[-1] + m)
        x["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    return dict(case=dict(case), x=x)


# ------------------------------------------------------------------ the framework's operators
def _own_rec(c, x):
    import paper_2605_22791_amd as g2
    how = dict(cu_seqlens=x["cu"], normalize=c["unit"])
    if c["kind"] == "step":
        o = g2.gdr2_gatedrec_step(x["x"], x["g"], x["gate"], x["h0"], **how)
        return {"o": o, "h": x["h0"]}
    ws = None
    if c["saved"]:
        p = g2.Gdr2Gatedrec(c["B"], c["T"], c["D"], g2.GDR2_BF16 if c["dtype"] == "bf16" else g2.GDR2_FP32, c["unit"])
        need = g2.gdr2_gatedrec_workspace_bytes(p, len(_lengths(c)) if c["lengths"] else 0, 1)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    o, h = g2.gdr2_gatedrec_fwd(x["x"], x["g"], x["gate"], x["h0"], ws=ws, save=c["saved"], **how)
    out = {"o": o, "h": h}
    if c["kind"] == "train":
        d = g2.gdr2_gatedrec_bwd(x["x"], x["g"], x["gate"], x["h0"], x["dout"], x["dhT"], ws=ws, saved=c["saved"],
                                 want_dh0=c["state"], **how)
        out.update({n: t for n, t in d.items() if t is not None})
    return out


def _own_ff(c, x):
    import paper_2605_22791_amd as g2
    args = x["x"], x["w_gate"], x["w_up"], x["w_down"]
    ws = None
    if c["saved"]:
        p = g2.Gdr2Gatedff(c["rows"], c["D"], c["F"], g2.GDR2_BF16 if c["dtype"] == "bf16" else g2.GDR2_FP32,
                           g2.GDR2_ACT_SILU if c["act"] == "silu" else g2.GDR2_ACT_GELU)
        ws = torch.empty(g2.gdr2_gatedff_workspace_bytes(p, 1), dtype=torch.uint8, device="cuda")
    out = {"y": g2.gdr2_gatedff_fwd(*args, act=c["act"], ws=ws, save=c["saved"])}
    if c["kind"] == "train":
        out.update(g2.gdr2_gatedff_bwd(*args, x["dy"], act=c["act"], ws=ws, saved=c["saved"]))
    return out


def _own_drop(s):
    import paper_2605_22791_amd as g2
    c, x = s["case"], s["x"]
    out = {"y": g2.gdr2_dropout_fwd(x["x"], c["p"], s["key"], offset=s["offset"], residual=x["residual"])}
    if c["kind"] == "train":
        out["dx"] = g2.gdr2_dropout_bwd(x["dy"], c["p"], s["key"], offset=s["offset"], dtype=x["x"].dtype)
    return out


# ------------------------------------------------------------------ the plain forms, in 32 bits
def _scan(a, u, longest):
    """h_t = a_t h_{t-1} + u_t along the first axis, by doubling; a is zero where a sequence of up to `longest` starts."""
    step = 1
    while step < longest:
        back_a = torch.nn.functional.pad(a[:-step], (0, 0, step, 0))
        back_u = torch.nn.functional.pad(u[:-step], (0, 0, step, 0))
        u = torch.addcmul(u, a, back_u)
        a = a * back_a
        step *= 2
    return u


def _plain_rec(s):
    c, x = s["case"], s["x"]
    dt, D = DT[c["dtype"]], c["D"]
    N, longest = c["B"] * c["T"], max(_lengths(c))
    if c["lengths"]:
        ends = x["cu"][1:].long()
        starts = x["cu"][:-1].long()
    else:
        starts = torch.arange(c["B"], device="cuda") * c["T"]
        ends = starts + c["T"]
    g = x["g"].reshape(N, D)
    a = torch.exp(g)
    m = torch.sqrt(-torch.expm1(2.0 * g)) if c["unit"] else None
    xi = x["x"].reshape(N, D).float()
    i = None if x["gate"] is None else x["gate"].reshape(N, D).float()
    mi = (m if i is None else m * i) if m is not None else i
    u = xi if mi is None else mi * xi
    h0 = x["h0"]
    inner = a.index_fill(0, starts, 0.0)
    first = u if h0 is None else u.index_add(0, starts, a[starts] * h0)
    h = _scan(inner, first, longest)
    last = h[ends - 1]
    out = {"o": h.to(dt).reshape(x["x"].shape), "h": last}
    if c["kind"] == "step":
        out["h"] = h0.copy_(last)
    if c["kind"] != "train":
        return out
    do = x["dout"].reshape(N, D).float()
    if x["dhT"] is not None:
        do = do.index_add(0, ends - 1, x["dhT"])
    # a_{t+1} meets dh_{t+1}: the decays one row earlier, zero at each sequence's end, and time reversed
    later = torch.nn.functional.pad(inner[1:], (0, 0, 0, 1))
    dh = _scan(later.flip(0), do.flip(0), longest).flip(0)
    before = torch.nn.functional.pad(h[:-1], (0, 0, 1, 0)).index_fill(0, starts, 0.0)
    if h0 is not None:
        before = before.index_copy(0, starts, h0)
    dg = a * before
    if m is not None:
        dg = dg - a * a / m * (xi if i is None else i * xi)
    out["dlog_decay"] = (dg * dh).reshape(x["g"].shape)
    out["dx"] = (dh if mi is None else dh * mi).to(dt).reshape(x["x"].shape)
    if i is not None:
        out["dgate"] = (dh * (xi if m is None else m * xi)).to(dt).reshape(x["x"].shape)
    if h0 is not None:
        out["dh0"] = a[starts] * dh[starts]
    return out


def _plain_ff(c, x):
    dt = DT[c["dtype"]]
    xf, wg, wu, wd = (x[n].float() for n in ("x", "w_gate", "w_up", "w_down"))
    g, u = torch.mm(xf, wg.t()), torch.mm(xf, wu.t())
    if c["act"] == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        slope = s * (1.0 + g * (1.0 - s))
    else:
        s = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        slope = s + g * torch.exp(-0.5 * g * g) * (0.5 / math.pi) ** 0.5
    a = g * s
    h = a * u
    out = {"y": torch.mm(h, wd.t()).to(dt)}
    if c["kind"] == "train":
        dy = x["dy"].float()
        dh = torch.mm(dy, wd)
        dg, du = dh * u * slope, dh * a
        out["dx"] = (torch.mm(dg, wg) + torch.mm(du, wu)).to(dt)
        out["dw_gate"] = torch.mm(dg.t(), xf).to(dt)
        out["dw_up"] = torch.mm(du.t(), xf).to(dt)
        out["dw_down"] = torch.mm(dy.t(), h).to(dt)
    return out


M32 = 0xFFFFFFFF


def _words(n, key, offset):
    """The first n words of Philox 4x32-10 (Salmon et al., SC 2011): counter (block, offset), key; int64 tensors of 32-bit values."""
    block = torch.arange((n + 3) // 4, device="cuda")
    c0, c1 = block & M32, block >> 32
    c2, c3 = torch.full_like(block, offset & M32), torch.full_like(block, offset >> 32)
    k0, k1 = key & M32, key >> 32
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64; the upper words through the shift and the mask
        c0, c1, c2, c3 = (q >> 32) & M32 ^ c1 ^ k0, q & M32, (p >> 32) & M32 ^ c3 ^ k1, p & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack([c0, c1, c2, c3], dim=1).reshape(-1)[:n]


def _plain_drop(s):
    c, x = s["case"], s["x"]
    keep = (_words(x["x"].numel(), s["key"], s["offset"]) >= round(c["p"] * 2 ** 32)).reshape(x["x"].shape)
    scale = 1.0 / (1.0 - c["p"])
    y = torch.where(keep, x["x"].float() * scale, 0.0)
    if x["residual"] is not None:
        y = x["residual"].float() + y
    out = {"y": y.to(DT[c["stream"] or c["dtype"]])}
    if c["kind"] == "train":
        out["dx"] = torch.where(keep, x["dy"].float() * scale, 0.0).to(DT[c["dtype"]])
    return out


def run(s):
    c, x = s["case"], s["x"]
    if own:
        return _own_rec(c, x) if c["op"] == "rec" else _own_ff(c, x) if c["op"] == "ff" else _own_drop(s)
    return _plain_rec(s) if c["op"] == "rec" else _plain_ff(c, x) if c["op"] == "ff" else _plain_drop(s)


def work(case):
    """Each input read once and each output written once; the recurrence takes about 20 operations an element and
    40 for its gradients, a product of the feed-forward 2 rows D F (three forward, six backward), dropout about 40."""
    e, train = 2 if case["dtype"] == "bf16" else 4, case["kind"] == "train"
    if case["op"] == "drop":
        n, r = case["rows"] * case["D"], {"": 0, "bf16": 2, "fp32": 4}[case["stream"]]
        return {"bytes": n * (e + r + (r or e) + (train and (r or e) + e)), "flops": 40.0 * n * (2 if train else 1)}
    if case["op"] == "ff":
        wide, weights = case["rows"] * case["D"] * e, 3 * case["D"] * case["F"] * e
        return {"bytes": (4 if train else 2) * wide + (2 if train else 1) * weights,
                "flops": (18.0 if train else 6.0) * case["rows"] * case["D"] * case["F"]}
    n, state = case["B"] * case["T"] * case["D"], 4 * len(_lengths(case)) * case["D"]
    g = case["gate"] * e
    nbytes = n * (2 * e + g + 4) + state * (2 if case["state"] else 1)
    if train:
        nbytes += n * (3 * e + 2 * g + 8) + (2 * state if case["state"] else 0)
    return {"bytes": nbytes, "flops": (60.0 if train else 20.0) * n}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_rec(c, x):
    """Token by token over all sequences at once, a row of a padded tensor for each."""
    lengths, D = _lengths(c), c["D"]
    L = max(lengths)
    length = torch.tensor(lengths, device="cuda")
    there = torch.arange(L, device="cuda") < length[:, None]

    def rows(t):
        to = torch.zeros((len(lengths), L, D), dtype=torch.float64, device="cuda")
        to[there] = t.reshape(-1, D).double()
        return to.transpose(0, 1).contiguous()

    def back(t, like):
        return t.transpose(0, 1)[there].reshape(like.shape)

    g = rows(x["g"])
    a, on = g.exp(), there.t()[:, :, None]
    m = torch.sqrt(1.0 - (2.0 * g).exp()) if c["unit"] else torch.ones_like(a)
    i = torch.ones_like(a) if x["gate"] is None else rows(x["gate"])
    xs = rows(x["x"])
    put = m * i * xs
    h = torch.zeros((len(lengths), D), dtype=torch.float64, device="cuda") if x["h0"] is None else x["h0"].double()
    before, hs = torch.empty_like(a), torch.empty_like(a)
    for t in range(L):
        before[t] = h
        h = torch.where(on[t], a[t] * h + put[t], h)
        hs[t] = h
    out = {"o": back(hs, x["x"]), "h": h}
    if c["kind"] != "train":
        return out
    do = rows(x["dout"])
    carry = torch.zeros_like(h) if x["dhT"] is None else x["dhT"].double()
    dh = torch.zeros_like(a)
    for t in reversed(range(L)):
        dh[t] = torch.where(on[t], do[t] + carry, 0.0)
        carry = torch.where(on[t], a[t] * dh[t], carry)
    dg = dh * a * before
    if c["unit"]:
        dg = dg - dh * i * xs * torch.where(on, (2.0 * g).exp() / m, 0.0)
    out["dlog_decay"] = back(dg, x["g"])
    out["dx"] = back(dh * m * i, x["x"])
    if x["gate"] is not None:
        out["dgate"] = back(dh * m * xs, x["x"])
    if x["h0"] is not None:
        out["dh0"] = carry
    return out


def _exact_ff(c, x):
    p = {n: x[n].double().requires_grad_(c["kind"] == "train") for n in ("x", "w_gate", "w_up", "w_down")}
    with torch.set_grad_enabled(c["kind"] == "train"):
        g, u = p["x"] @ p["w_gate"].T, p["x"] @ p["w_up"].T
        a = torch.nn.functional.silu(g) if c["act"] == "silu" else torch.nn.functional.gelu(g)
        y = (a * u) @ p["w_down"].T
        out = {"y": y.detach()}
        if c["kind"] == "train":
            y.backward(x["dy"].double())
            out.update({"d" + n: t.grad for n, t in p.items()})
    return out


def _exact_drop(c, x, key, offset):
    """The generator with its products in halves of 16 bits."""
    def product(v, k):
        low, high = v & 0xFFFF, v >> 16
        k0, k1 = k & 0xFFFF, k >> 16
        mid = high * k0 + (low * k0 >> 16)
        rest = low * k1 + (mid & 0xFFFF)
        return high * k1 + (mid >> 16) + (rest >> 16), (rest & 0xFFFF) << 16 | low * k0 & 0xFFFF

    n = x["x"].numel()
    e = torch.arange(n, device="cuda")
    b = e // 4
    state = [b % 2 ** 32, b // 2 ** 32, torch.full_like(b, offset % 2 ** 32), torch.full_like(b, offset // 2 ** 32)]
    for r in range(10):
        h0, l0 = product(state[0], 0xD2511F53)
        h1, l1 = product(state[2], 0xCD9E8D57)
        k0, k1 = (key % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (key // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        state = [h1 ^ state[1] ^ k0, l1, h0 ^ state[3] ^ k1, l0]
    word = torch.zeros_like(e)
    for k in range(4):
        word = torch.where(e % 4 == k, state[k], word)
    keep = (word >= round(c["p"] * 2 ** 32)).reshape(x["x"].shape)
    y = torch.where(keep, x["x"].double() / (1.0 - c["p"]), 0.0)
    out = {"y": y if x["residual"] is None else x["residual"].double() + y}
    if c["kind"] == "train":
        out["dx"] = torch.where(keep, x["dy"].double() / (1.0 - c["p"]), 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "drop":
        return _exact_drop(case, s["x"], s["key"], s["offset"])
    return _exact_rec(case, s["x"]) if case["op"] == "rec" else _exact_ff(case, s["x"])
