"""Performance cases of the training operators around the compressed linears.

Four operators, each with its plain form in elementary torch operations (32 bits inside, one rounding at the end), the
calls a user makes of the library, and its definition in 64 bits:

  q8      a matrix kept as an 8-bit checkpoint (one scale per row and group of 128 columns) and read back
  swiglu  H = silu(G) * U; a training step keeps G and U in 8 bits and takes dG, dU from them
  norm    h' = h + alpha * gate * N_post(b), y = N_pre(h'): the residual join between two blocks with both RMS norms; a
          training step keeps h and b in 8 bits
  ce      softmax cross entropy of X W^T over a vocabulary without the logits in memory, and its gradients

The 8-bit format is part of the definition: with a = max |x| over the group (binary32), scale = a / 127 and
code = round_to_even(x * (127 / a)), every step one binary32 operation; a group with a < 2^-100 is all zeros.

`own` False: the plain forms.  True: the library.
"""
import torch

own = False

GROUP = 128          # columns that share one scale of an 8-bit checkpoint
TINY = 2.0 ** -100   # a group whose largest magnitude is below this is stored as zeros
EPS = 1e-5


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one layer's input of a small model's micro-batch (4096 tokens of width 896) kept in 8 bits
        {"name": "q8_bf16_4096x896", "op": "q8", "dtype": "bf16", "rows": 4096, "cols": 896, "pad": 0},
        # a column slice of a wider fp32 buffer whose last group is partly filled
        {"name": "q8_f32_3001x2056_strided", "op": "q8", "dtype": "f32", "rows": 3001, "cols": 2056, "pad": 120},
        # decoding: a handful of rows, nothing kept; the call's latency is what counts
        {"name": "swiglu_fwd_bf16_8x4864", "op": "swiglu", "mode": "fwd", "dtype": "bf16", "rows": 8, "cols": 4864, "stacked": True},
        # a fine-tuning batch of 16384 tokens behind a stacked gate/up product
        {"name": "swiglu_step_bf16_16384x8192", "op": "swiglu", "mode": "step", "dtype": "bf16", "rows": 16384, "cols": 8192, "stacked": True},
        # fp32 with an odd number of rows and a partly filled last group
        {"name": "swiglu_step_f32_1027x1000", "op": "swiglu", "mode": "step", "dtype": "f32", "rows": 1027, "cols": 1000, "stacked": False},
        # decoding through a sandwich-norm block
        {"name": "norm_fwd_bf16_16x896", "op": "norm", "mode": "fwd", "dtype": "bf16", "rows": 16, "cols": 896, "join": True, "post": True, "gate": True},
        # the whole residual join at the width and batch of the largest layer of this repository
        {"name": "norm_step_bf16_16384x3072", "op": "norm", "mode": "step", "dtype": "bf16", "rows": 16384, "cols": 3072, "join": True, "post": True, "gate": True},
        # a plain pre-norm transformer's join (no norm behind the block, no gate) in fp32, odd sizes
        {"name": "norm_step_f32_2049x2040", "op": "norm", "mode": "step", "dtype": "f32", "rows": 2049, "cols": 2040, "join": True, "post": False, "gate": False},
        # scoring a short text: the vocabulary matrix is read once, the products are few
        {"name": "ce_score_64x2048x128256", "op": "ce", "mode": "score", "tokens": 64, "d": 2048, "vocab": 128256, "weighted": False, "logit_scale": 1.0},
        # a ragged micro-batch over an odd vocabulary with per-token weights and scaled logits
        {"name": "ce_step_333x904x32003", "op": "ce", "mode": "step", "tokens": 333, "d": 904, "vocab": 32003, "weighted": True, "logit_scale": 0.5},
        # a small model with a large vocabulary, its whole batch of 8 x 512 tokens
        {"name": "ce_step_4096x896x151936", "op": "ce", "mode": "step", "tokens": 4096, "d": 896, "vocab": 151936, "weighted": False, "logit_scale": 1.0},
        # half a fine-tuning batch at the largest width
        {"name": "ce_step_8192x3072x128256", "op": "ce", "mode": "step", "tokens": 8192, "d": 3072, "vocab": 128256, "weighted": False, "logit_scale": 1.0},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["q8", "swiglu", "norm", "ce"])
    if op == "ce":
        while True:
            t, d, v = _spread(rng, 1, 8192), 8 * _spread(rng, 8, 512), _spread(rng, 500, 152000)
            if t * d * v <= 8192 * 3072 * 128256 and t * v <= 8192 * 128256:
                break
        return {"op": "ce", "mode": rng.choice(["score", "step", "step"]), "tokens": t, "d": d, "vocab": v,
                "weighted": rng.random() < 0.3, "logit_scale": rng.choice([1.0, 1.0, 0.5])}
    while True:
        rows, cols = _spread(rng, 1, 32768), 8 * _spread(rng, 8, 1024 if op == "norm" else 2048)
        if rows * cols <= (1 << 26 if op == "norm" else 1 << 27):
            break
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"]), "rows": rows, "cols": cols}
    if op == "q8":
        case["pad"] = rng.choice([0, 0, 8, 120])
    elif op == "swiglu":
        case.update(mode=rng.choice(["fwd", "step", "step"]), stacked=rng.random() < 0.5)
    else:
        case.update(mode=rng.choice(["fwd", "step", "step"]), join=rng.random() < 0.8, post=rng.random() < 0.6, gate=rng.random() < 0.4)
        if not case["join"]:
            case.update(post=False, gate=False)
    return case


def work(case):
    """Each input read once, each output written once; a training step's own checkpoints (8 bits and the scales) are
    written by its forward half and read by its backward half."""
    op = case["op"]
    if op == "ce":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        fwd_bytes, fwd_flops = 2 * (t * d + v * d) + 8 * t + 8 * t, 2 * t * d * v
        if case["mode"] == "score":
            return {"bytes": fwd_bytes, "flops": fwd_flops}
        # backward: the logits again, D W and D^T X; X and W read, dX and dW written
        return {"bytes": 2 * fwd_bytes + 2 * (t * d + v * d), "flops": 4 * fwd_flops}
    n, e = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
    q = n + 4 * case["rows"] * -(-case["cols"] // GROUP)    # one checkpoint: codes and scales
    if op == "q8":
        return {"bytes": 2 * n * e + 2 * q, "flops": 4 * n}
    if op == "swiglu":
        if case["mode"] == "fwd":
            return {"bytes": 3 * n * e, "flops": 6 * n}
        return {"bytes": 3 * n * e + 2 * q + n * e + 2 * q + 2 * n * e, "flops": 24 * n}
    join = 1 if case["join"] else 0
    fwd = n * e * (2 + 2 * join)                        # h, y and with a join b, h'
    if case["mode"] == "fwd":
        return {"bytes": fwd, "flops": 10 * n}
    qs = q * (1 + (1 if case["join"] else 0))           # h and b
    return {"bytes": fwd + 2 * qs + n * e * (3 + join), "flops": 40 * n}   # dy, dh' read; dh and db written


# ------------------------------------------------------------------------------------------------------- inputs
def _io(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _activations(g, rows, cols):
    """Residual-stream-like values: every row its own size, one channel in 64 much larger than the rest."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    x[:, ::64] *= 8.0
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    io, op = _io(case), case["op"]
    s = {"case": dict(case)}
    if op == "ce":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        W = (rnd(v, d) * d ** -0.5).to(io)
        # targets as frequent as words are (low ids often), a third of the tokens a prompt that is not trained on
        y = (torch.rand(t, generator=g, device="cuda") ** 4 * v).long().clamp_(max=v - 1)
        # hidden states as a half-trained model has them: the target's logit is raised by 0 to 12
        X = (rnd(t, d) + 12.0 * torch.rand(t, 1, generator=g, device="cuda") * W[y].float()).to(io)
        y[torch.arange(t, device="cuda") % 96 < 32] = -100
        y[t - 1] = v - 1
        s.update(X=X, W=W, targets=y, weight=(torch.rand(t, generator=g, device="cuda") * 2) if case["weighted"] else None)
        s["out"] = dict(loss=torch.empty(t, device="cuda"), lse=torch.empty(t, device="cuda"), total=torch.empty(2, device="cuda"))
        if case["mode"] == "step":
            s["out"].update(dX=torch.empty_like(X), dW=torch.empty_like(W))
        return s
    rows, cols = case["rows"], case["cols"]
    new = lambda *sh, dt=io: torch.empty(*sh, dtype=dt, device="cuda")  # noqa: E731
    code = lambda: (new(rows, cols, dt=torch.int8), new(rows, -(-cols // GROUP), dt=torch.float32))  # noqa: E731
    if op == "q8":
        s["X"] = _activations(g, rows, cols + case["pad"]).to(io)[:, :cols]
        s["q"] = code()
        s["out"] = {"X": new(rows, cols)}
    elif op == "swiglu":
        GU = (rnd(rows, 2 * cols) * 1.5).to(io)
        dGU = new(rows, 2 * cols)
        s["G"], s["U"] = (GU[:, :cols], GU[:, cols:]) if case["stacked"] else (GU[:, :cols].contiguous(), GU[:, cols:].contiguous())
        s["out"] = {"H": new(rows, cols)}
        if case["mode"] == "step":
            s["dH"] = (rnd(rows, cols) * 0.1).to(io)
            s["qG"], s["qU"] = code(), code()
            s["out"]["dG"], s["out"]["dU"] = (dGU[:, :cols], dGU[:, cols:]) if case["stacked"] else (new(rows, cols), new(rows, cols))
    else:
        s["h"] = _activations(g, rows, cols).to(io)
        s["b"] = (rnd(rows, cols) * torch.exp(0.5 * rnd(rows, 1))).to(io) if case["join"] else None
        s["w_pre"] = (1.0 + 0.2 * rnd(cols)).to(io)
        s["w_post"] = (1.0 + 0.2 * rnd(cols)).to(io) if case["post"] else None
        s["gate"] = (0.5 + 0.2 * rnd(cols)).to(io) if case["gate"] else None
        s["alpha"] = 0.7 if case["join"] else 1.0
        s["out"] = {"y": new(rows, cols)}
        if case["join"]:
            s["out"]["h_out"] = new(rows, cols)
        if case["mode"] == "step":
            f32 = torch.float32
            s["dy"], s["dh_next"] = (rnd(rows, cols) * 0.1).to(io), (rnd(rows, cols) * 0.1).to(io)
            s["qh"], s["qb"] = code(), code() if case["join"] else (None, None)
            s["rstd_pre"], s["rstd_post"] = new(rows, dt=f32), new(rows, dt=f32) if case["post"] else None
            s["out"].update(dh=new(rows, cols), dw_pre=new(cols, dt=f32))
            if case["join"]:
                s["out"]["db"] = new(rows, cols)
            if case["post"]:
                s["out"]["dw_post"] = new(cols, dt=f32)
            if case["gate"]:
                s["out"]["dgate"] = new(cols, dt=f32)
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _q8(x):
    """The values that the 8-bit checkpoint of x (binary32) stands for."""
    rows, cols = x.shape
    pad = -cols % GROUP
    xg = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, GROUP)
    a = xg.abs().amax(-1, keepdim=True)
    live = a >= TINY
    inv = torch.where(live, 127.0 / a, 0.0)
    scale = torch.where(live, a / 127.0, 0.0)
    return (torch.round(xg * inv) * scale).view(rows, -1)[:, :cols]


def _plain_swiglu(s):
    io = _io(s["case"])
    G, U = s["G"].float(), s["U"].float()
    out = {"H": (G / (1 + torch.exp(-G)) * U).to(io)}
    if s["case"]["mode"] == "step":
        G, U, dH = _q8(G), _q8(U), s["dH"].float()
        sg = 1 / (1 + torch.exp(-G))
        out["dG"] = (dH * U * sg * (1 + G * (1 - sg))).to(io)
        out["dU"] = (dH * G * sg).to(io)
    return out


def _plain_norm(s):
    c, io, alpha = s["case"], _io(s["case"]), s["alpha"]
    h, w_pre = s["h"].float(), s["w_pre"].float()
    out = {}
    if c["join"]:
        b = s["b"].float()
        r_b = torch.rsqrt((b * b).mean(-1, keepdim=True) + EPS) if c["post"] else 1.0
        w_post = s["w_post"].float() if c["post"] else 1.0
        gate = s["gate"].float() if c["gate"] else 1.0
        t = h + alpha * (gate * (b * r_b * w_post))
        out["h_out"] = t.to(io)
    else:
        t = h
    r_h = torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS)
    out["y"] = (t * r_h * w_pre).to(io)
    if c["mode"] == "fwd":
        return out
    dy, dt = s["dy"].float(), s["dh_next"].float()
    tq = _q8(h)
    if c["join"]:
        bhat = _q8(b) * r_b
        tq = tq + alpha * (gate * (bhat * w_post))
    that = tq * r_h
    gy = dy * w_pre
    dt = dt + r_h * (gy - that * (gy * that).mean(-1, keepdim=True))
    out["dh"] = dt.to(io)
    out["dw_pre"] = (dy * that).sum(0)
    if c["join"]:
        e = alpha * dt * gate
        col = (dt * bhat).sum(0) * alpha
        p = e * w_post
        out["db"] = (r_b * (p - bhat * (p * bhat).mean(-1, keepdim=True)) if c["post"] else p).to(io)
        if c["post"]:
            out["dw_post"] = col * gate
        if c["gate"]:
            out["dgate"] = col * w_post
    return out


def _plain_ce(s):
    c = s["case"]
    X, W, y = s["X"].float(), s["W"].float(), s["targets"]
    logits = X @ W.t()
    logits *= c["logit_scale"]
    valid = (y >= 0) & (y < c["vocab"])
    yc = torch.where(valid, y, 0)[:, None]
    top = logits.amax(-1, keepdim=True)
    target = logits.gather(1, yc)[:, 0]
    p = logits.sub_(top).exp_()
    z = p.sum(-1, keepdim=True)
    lse = (top + torch.log(z))[:, 0]
    loss = torch.where(valid, lse - target, 0.0)
    w = torch.where(valid, s["weight"] if c["weighted"] else 1.0, 0.0)
    out = {"loss": loss, "lse": lse, "total": torch.stack([(w * loss).sum(), w.sum()])}
    if c["mode"] == "step":
        f = torch.where(out["total"][1] > 0, c["logit_scale"] / out["total"][1], 0.0)
        p.div_(z).scatter_add_(1, yc, torch.full_like(loss, -1.0)[:, None]).mul_(w[:, None])
        out["dX"] = ((p @ W) * f).to(torch.bfloat16)
        out["dW"] = ((p.t() @ X) * f).to(torch.bfloat16)
    return out


# ------------------------------------------------------------------------------------------------------- the library
def _library(s):
    from paper_2605_01255_b200 import binding as B
    c, o = s["case"], s["out"]
    op = c["op"]
    if op == "ce":
        if "desc" not in s:   # the plan and the scratch memory that a program keeps
            s["desc"] = B.make_ce_desc(c["tokens"], c["d"], c["vocab"], logit_scale=c["logit_scale"])
            s["ws"] = B.alloc_ce_workspace(s["desc"], B.ACX_OP_CE_BWD if c["mode"] == "step" else B.ACX_OP_CE_FWD)
        d = s["desc"]
        B.acx_linear_ce_fwd(d, s["X"], s["W"], s["targets"], o["loss"], o["lse"], total=o["total"], weight=s["weight"], ws=s["ws"])
        if c["mode"] == "step":
            B.acx_linear_ce_bwd(d, s["X"], s["W"], s["targets"], o["lse"], o["dX"], o["dW"], weight=s["weight"],
                                denom=o["total"][1:], ws=s["ws"])
        return o
    if "desc" not in s:
        s["desc"] = B.make_rows_desc(c["rows"], c["cols"], c["dtype"])
        s["ws"] = B.alloc_rows_workspace(s["desc"], B.ACX_OP_NORM_BWD) if op == "norm" else None
    d = s["desc"]
    if op == "q8":
        B.acx_q8_store(d, s["X"], *s["q"])
        B.acx_q8_load(d, *s["q"], o["X"])
    elif op == "swiglu":
        if c["mode"] == "fwd":
            B.acx_swiglu_fwd(d, s["G"], s["U"], o["H"])
        else:
            B.acx_swiglu_fwd(d, s["G"], s["U"], o["H"], *s["qG"], *s["qU"])
            B.acx_swiglu_bwd(d, s["dH"], *s["qG"], *s["qU"], o["dG"], o["dU"])
    elif c["mode"] == "fwd":
        B.acx_norm_join_fwd(d, s["h"], s["b"], s["w_post"], s["gate"], s["w_pre"], o.get("h_out"), o["y"], eps=EPS, alpha=s["alpha"])
    else:
        B.acx_norm_join_fwd(d, s["h"], s["b"], s["w_post"], s["gate"], s["w_pre"], o.get("h_out"), o["y"], *s["qh"], *s["qb"],
                            s["rstd_post"], s["rstd_pre"], eps=EPS, alpha=s["alpha"])
        B.acx_norm_join_bwd(d, s["dy"], s["dh_next"], s["w_post"], s["gate"], s["w_pre"], *s["qh"], *s["qb"], s["rstd_post"],
                            s["rstd_pre"], o["dh"], o.get("db"), o.get("dw_post"), o.get("dgate"), o["dw_pre"], alpha=s["alpha"], ws=s["ws"])
    return o


def run(state):
    if own:
        return _library(state)
    op = state["case"]["op"]
    if op == "q8":
        return {"X": _q8(state["X"].float()).to(_io(state["case"]))}
    return {"swiglu": _plain_swiglu, "norm": _plain_norm, "ce": _plain_ce}[op](state)


# ------------------------------------------------------------------------------------------------------- 64 bits
def _codes64(x):
    """Checkpointed values in 64 bits.  The codes and scales are whole decisions of the format (binary32 steps, see the
    head of this file); the value a code stands for is their exact product."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    for c0 in range(0, cols, GROUP):
        part = x[:, c0:c0 + GROUP].float()
        a = torch.max(part.max(1).values, -part.min(1).values)
        a = torch.where(a < TINY, torch.inf, a)            # an infinite divisor makes every code of the group 0
        k = torch.round(part * (127.0 / a)[:, None])
        out[:, c0:c0 + GROUP] = k.double() * torch.where(a.isinf(), 0.0, a / 127.0).double()[:, None]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "q8":
        return {"X": _codes64(s["X"])}
    if op == "swiglu":
        G, U = s["G"].double(), s["U"].double()
        out = {"H": G * torch.sigmoid(G) * U}
        if case["mode"] == "step":
            G, U, dH = _codes64(s["G"]), _codes64(s["U"]), s["dH"].double()
            sg = torch.sigmoid(G)
            out["dU"] = G * sg * dH
            out["dG"] = (sg + G * sg * torch.sigmoid(-G)) * U * dH
        return out
    if op == "norm":
        n = case["cols"]
        t, out = s["h"].double(), {}
        if case["join"]:
            k = torch.full((n,), s["alpha"], dtype=torch.float64, device="cuda")     # what multiplies the block's output per column
            k = k * s["gate"].double() if case["gate"] else k
            k_w = k * s["w_post"].double() if case["post"] else k
            b = s["b"].double()
            len_b = torch.sqrt(b.square().sum(1, keepdim=True) / n + EPS) if case["post"] else torch.ones_like(b[:, :1])
            t = t + k_w * b / len_b
            out["h_out"] = t
        len_t = torch.sqrt(t.square().sum(1, keepdim=True) / n + EPS)
        out["y"] = s["w_pre"].double() * t / len_t
        if case["mode"] == "fwd":
            return out
        t = _codes64(s["h"])
        if case["join"]:
            b = _codes64(s["b"]) / len_b
            t = t + k_w * b
        t = t / len_t
        dy = s["dy"].double()
        out["dw_pre"] = (dy * t).sum(0)
        v = dy * s["w_pre"].double()
        d = s["dh_next"].double() + (v - t * ((v * t).sum(1, keepdim=True) / n)) / len_t
        out["dh"] = d
        if case["join"]:
            v = d * k_w
            out["db"] = (v - b * ((v * b).sum(1, keepdim=True) / n)) / len_b if case["post"] else v
            if case["post"]:
                out["dw_post"] = (d * b * k).sum(0)
            if case["gate"]:
                out["dgate"] = (d * b).sum(0) * s["alpha"] * (s["w_post"].double() if case["post"] else 1.0)
        return out
    t, V = case["tokens"], case["vocab"]
    X, W, y = s["X"].double(), s["W"].double(), s["targets"]
    trained = (y >= 0) & (y < V)
    w = (s["weight"].double() if case["weighted"] else torch.ones(t, dtype=torch.float64, device="cuda")) * trained
    count = w.sum()
    loss, lse = (torch.empty(t, dtype=torch.float64, device="cuda") for _ in range(2))
    step = case["mode"] == "step"
    dX, dW = (torch.zeros_like(X), torch.zeros_like(W)) if step else (None, None)
    for r0 in range(0, t, 2048):    # blocks of tokens: the 64-bit logits of all of them would be large
        r = slice(r0, min(t, r0 + 2048))
        L = case["logit_scale"] * (X[r] @ W.T)
        lse[r] = torch.logsumexp(L, 1)
        hot = torch.zeros_like(L)
        at = torch.nonzero(trained[r])[:, 0]
        hot[at, y[r][at]] = 1.0
        loss[r] = torch.where(trained[r], lse[r] - (L * hot).sum(1), 0.0)
        if step:
            D = (torch.softmax(L, 1) - hot) * (w[r] * case["logit_scale"] / count.clamp(min=1e-300))[:, None]
            dX[r] = D @ W
            dW += D.T @ X[r]
        del L, hot
    out = {"loss": loss, "lse": lse, "total": torch.stack([(w * loss).sum(), count])}
    if step:
        out["dX"], out["dW"] = dX, dW
    return out
