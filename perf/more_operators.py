"""Performance cases of the operators that a language model's training step has around its linears.

Three operators, each with its plain form in elementary torch operations (32 bits inside, one rounding at the end), the
calls a user makes of the library, and its definition in 64 bits:

  attn    softmax attention over packed documents: causal, bidirectional or with a visible prefix, scores capped by a tanh
          or biased by the distance, several query heads per key head; a training step takes dQ, dK, dV too
  embed   rows of an embedding table, scaled; a training step takes the table's gradient, the sum over each word's tokens
  clip    the norm over many gradients, and the gradients scaled down to a largest norm

`own` False: the plain forms.  True: the library.
"""
import random

import torch

own = False


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # scoring one short text with a small model's heads, every token sees every other: the call's latency
        {"name": "attn_fwd_77x14x2x64_bidirectional", "op": "attn", "mode": "fwd", "tokens": 77, "heads": 14, "kv_heads": 2, "d": 64, "docs": 1,
         "cut": 0, "causal": False, "prefix": False, "cap": 0.0, "alibi": False, "stacked": True},
        # a small model's micro-batch, packed from eleven documents of uneven lengths
        {"name": "attn_step_4096x14x2x64_documents", "op": "attn", "mode": "step", "tokens": 4096, "heads": 14, "kv_heads": 2, "d": 64, "docs": 11,
         "cut": 1, "causal": True, "prefix": False, "cap": 0.0, "alibi": False, "stacked": True},
        # prompts that see themselves whole, capped scores, an odd head width and odd lengths
        {"name": "attn_step_3001x6x2x72_prefix_cap", "op": "attn", "mode": "step", "tokens": 3001, "heads": 6, "kv_heads": 2, "d": 72, "docs": 5,
         "cut": 2, "causal": True, "prefix": True, "cap": 30.0, "alibi": False, "stacked": False},
        # one long document through the widest heads of this repository's layers
        {"name": "attn_step_8192x24x8x128_causal", "op": "attn", "mode": "step", "tokens": 8192, "heads": 24, "kv_heads": 8, "d": 128, "docs": 1,
         "cut": 0, "causal": True, "prefix": False, "cap": 0.0, "alibi": False, "stacked": True},
        # scoring a long text by a model whose heads know positions from the distance
        {"name": "attn_fwd_16384x32x8x64_distance", "op": "attn", "mode": "fwd", "tokens": 16384, "heads": 32, "kv_heads": 8, "d": 64, "docs": 1,
         "cut": 0, "causal": True, "prefix": False, "cap": 0.0, "alibi": True, "stacked": True},
        # the rows of a handful of new tokens
        {"name": "embed_fwd_bf16_8x896", "op": "embed", "mode": "fwd", "dtype": "bf16", "grad": "bf16", "tokens": 8, "d": 896, "vocab": 32000, "scale": 1.0},
        # a fine-tuning batch over a large vocabulary
        {"name": "embed_step_bf16_16384x2048x128256", "op": "embed", "mode": "step", "dtype": "bf16", "grad": "f32", "tokens": 16384, "d": 2048,
         "vocab": 128256, "scale": 1.0},
        # fp32, ragged, a vocabulary of odd size, rows scaled by the root of the width
        {"name": "embed_step_f32_5003x1000x32003", "op": "embed", "mode": "step", "dtype": "f32", "grad": "f32", "tokens": 5003, "d": 1000,
         "vocab": 32003, "scale": 31.62},
        # the vectors of a small model: many tiny gradients, the calls' latency
        {"name": "clip_vectors_49x896", "op": "clip", "kind": "vectors", "layers": 24, "d": 896, "kv": 128, "inter": 4864, "r": 64, "vocab": 0,
         "cut": 0, "max_norm": 1.0},
        # the gradient factors of a small model's compressed linears
        {"name": "clip_factors_24x896_r64", "op": "clip", "kind": "factors", "layers": 24, "d": 896, "kv": 128, "inter": 4864, "r": 64, "vocab": 0,
         "cut": 0, "max_norm": 1.0},
        # factors of a larger model and the bf16 gradient of its head
        {"name": "clip_factors_16x2048_r128_head", "op": "clip", "kind": "factors", "layers": 16, "d": 2048, "kv": 512, "inter": 8192, "r": 128,
         "vocab": 128256, "cut": 0, "max_norm": 1.0},
        # full bf16 gradients of all kinds of sizes, the norm below the largest one allowed
        {"name": "clip_ragged_401", "op": "clip", "kind": "ragged", "layers": 401, "d": 120001, "kv": 0, "inter": 0, "r": 0, "vocab": 0, "cut": 3,
         "max_norm": 1e6},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["attn", "attn", "embed", "clip"])
    if op == "attn":
        while True:
            t, d = _spread(rng, 1, 16384), 8 * rng.choice([4, 8, 8, 9, 10, 12, 15, 16, 16])
            kv = rng.choice([1, 2, 3, 4, 8])
            h = kv * rng.choice([1, 2, 3, 4, 7])
            docs = min(t, _spread(rng, 1, 64))
            mode = rng.choice(["fwd", "step", "step"])
            case = {"op": "attn", "mode": mode, "tokens": t, "heads": h, "kv_heads": kv, "d": d, "docs": docs, "cut": rng.randrange(1000)}
            if h <= 32 and t * t * h * d <= 8192 * 8192 * 24 * 128:   # the plain form takes all pairs
                break
        mask = rng.choice(["causal", "causal", "prefix", "all"])
        case.update(causal=mask != "all", prefix=mask == "prefix", cap=rng.choice([0.0, 0.0, 50.0]), alibi=rng.random() < 0.3,
                    stacked=rng.random() < 0.5)
        return case
    if op == "embed":
        while True:
            t, d, v = _spread(rng, 1, 32768), 8 * _spread(rng, 8, 512), _spread(rng, 100, 152000)
            if v * d <= 128256 * 2048 and t * d <= 16384 * 2048:
                break
        return {"op": "embed", "mode": rng.choice(["fwd", "step", "step"]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "grad": rng.choice(["bf16", "f32"]), "tokens": t, "d": d, "vocab": v, "scale": rng.choice([1.0, 1.0, 22.6])}
    kind = rng.choice(["vectors", "factors", "factors", "ragged"])
    case = {"op": "clip", "kind": kind, "layers": rng.randrange(1, 25), "d": 8 * rng.randrange(32, 256), "cut": rng.randrange(1000),
            "max_norm": rng.choice([1.0, 1.0, 1e6])}
    case.update(kv=case["d"] // 4, inter=3 * case["d"], r=rng.choice([16, 64, 128]), vocab=rng.choice([0, 0, 32003]))
    if kind == "ragged":
        case.update(layers=_spread(rng, 1, 700), d=_spread(rng, 10, 200000), kv=0, inter=0, r=0, vocab=0)
    return case


def _lengths(case):
    """Lengths of the packed documents: uneven cuts of the tokens, none empty."""
    rng = random.Random(case["cut"])
    cuts = sorted(rng.sample(range(1, case["tokens"]), case["docs"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [case["tokens"]])]


def _prefixes(case):
    rng = random.Random(case["cut"] + 1)
    return [rng.randrange(0, n + 1) if case["prefix"] else 0 for n in _lengths(case)]


def _gradients(case):
    """(elements, dtype, weight in the squared norm) of every gradient."""
    c = case
    if c["kind"] == "ragged":
        rng = random.Random(c["cut"])
        return [(_spread(rng, 1, c["d"]), "bf16" if rng.random() < 0.7 else "f32", 1.0) for _ in range(c["layers"])]
    if c["kind"] == "vectors":
        return [(c["d"], "f32", 1.0)] * (2 * c["layers"] + 1)
    d, kv, n, r = c["d"], c["kv"], c["inter"], c["r"]
    out = []
    for _ in range(c["layers"]):
        # factors A (outputs x r) of q, k, v, o, gate, up, down: the squared norm of A S^T is (d_in + r + 1) / r times A's on average
        out += [(o * r, "f32", (i + r + 1) / r) for o, i in ((d, d), (kv, d), (kv, d), (d, d), (n, d), (n, d), (d, n))]
        out += [(d, "f32", 1.0)] * 2
    return out + ([(c["vocab"] * d, "bf16", 1.0)] if c["vocab"] else [])


def _buckets(case):
    """The gradients lie one behind the other in one buffer for each type, every one of them on a 16-byte boundary:
    (type, offset) of each, and the buffers' sizes."""
    size, at = {}, []
    for n, t, _ in _gradients(case):
        at.append((t, size.get(t, 0)))
        size[t] = size.get(t, 0) + -(-n // 8) * 8
    return at, size


def work(case):
    op = case["op"]
    if op == "attn":
        pairs = 0
        for n, p in zip(_lengths(case), _prefixes(case)):
            # causal: row i sees max(i + 1, p) keys
            pairs += n * n if not case["causal"] else n * (n + 1) // 2 + p * (p - 1) // 2
        t, h, k, d = case["tokens"], case["heads"], case["kv_heads"], case["d"]
        fwd = 2 * t * d * (2 * h + 2 * k) + 4 * t * h
        if case["mode"] == "fwd":
            return {"bytes": fwd, "flops": 4 * pairs * h * d}
        # backward: q, k, v, o, dO, lse read; dQ, dK, dV written; five products
        return {"bytes": fwd + 2 * t * d * (4 * h + 4 * k) + 4 * t * h, "flops": 14 * pairs * h * d}
    if op == "embed":
        t, d, e = case["tokens"], case["d"], 2 if case["dtype"] == "bf16" else 4
        fwd = 2 * t * d * e + 8 * t
        if case["mode"] == "fwd":
            return {"bytes": fwd, "flops": t * d}
        return {"bytes": fwd + t * d * e + 8 * t + case["vocab"] * d * (2 if case["grad"] == "bf16" else 4), "flops": 3 * t * d}
    g = _gradients(case)
    return {"bytes": sum(2 * n * (2 if t == "bf16" else 4) for n, t, _ in g), "flops": 3 * sum(n for n, _, _ in g)}


# ------------------------------------------------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    new = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    op = case["op"]
    s = {"case": dict(case)}
    if op == "attn":
        t, h, k, d, bf = case["tokens"], case["heads"], case["kv_heads"], case["d"], torch.bfloat16

        def split(x):
            """q, k, v as the columns of one product's output, or each by itself."""
            parts = [p.unflatten(1, (-1, d)) for p in x.split([h * d, k * d, k * d], 1)]
            return parts if case["stacked"] else [p.contiguous() for p in parts]
        qkv = rnd(t, (h + 2 * k) * d)
        qkv[:, h * d:(h + k) * d:16] += 2.0      # keys have channels with a mean of their own
        s["q"], s["k"], s["v"] = split((1.2 * qkv).to(bf))
        off = torch.tensor([0] + _lengths(case), dtype=torch.int32).cumsum(0).to(torch.int32)
        s["offsets"] = off.cuda()
        s["prefix"] = torch.tensor(_prefixes(case), dtype=torch.int32).cuda() if case["prefix"] else None
        s["slopes"] = 2.0 ** (-8.0 * (1 + torch.arange(h, device="cuda")) / h) if case["alibi"] else None
        s["out"] = {"o": new(t, h, d, dt=bf), "lse": new(h, t)}
        if case["mode"] == "step":
            s["do"] = (0.1 * rnd(t, h, d)).to(bf)
            s["out"]["dq"], s["out"]["dk"], s["out"]["dv"] = split(new(t, (h + 2 * k) * d, dt=bf))
    elif op == "embed":
        t, d, v, io = case["tokens"], case["d"], case["vocab"], _TYPES[case["dtype"]]
        s["E"] = (0.05 * rnd(v, d)).to(io)
        # words as frequent as they are (low ids often), one token in eight the same separator, one in 50 padding
        ids = (torch.rand(t, generator=g, device="cuda") ** 4 * v).long().clamp_(max=v - 1)
        u = torch.rand(t, generator=g, device="cuda")
        ids = torch.where(u < 0.125, v // 2, ids)
        s["ids"] = torch.where(u > 0.98, -100, ids)
        s["out"] = {"Y": new(t, d, dt=io)}
        if case["mode"] == "step":
            s["dY"] = (0.1 * rnd(t, d)).to(io)
            s["out"]["dE"] = new(v, d, dt=_TYPES[case["grad"]])
    else:
        spec = _gradients(case)
        at, size = _buckets(case)
        flat, clipped = ({t: torch.zeros(n, dtype=_TYPES[t], device="cuda") for t, n in size.items()} for _ in range(2))
        parts = lambda b: [b[t][o:o + n] for (t, o), (n, _, _) in zip(at, spec)]  # noqa: E731
        s["grads"], s["clipped"], s["weights"] = parts(flat), parts(clipped), [w for _, _, w in spec]
        for i, x in enumerate(s["grads"]):
            x.copy_(0.01 * rnd(len(x)) * 2.0 ** (i % 5 - 2))
        s["out"] = {"total": new(2), "clipped": clipped}
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _visible(c, offsets, prefix):
    """Keys that each token sees (tokens x tokens, truth values): those of its document up to its own position or the
    prefix's end."""
    t = torch.arange(c["tokens"], device="cuda")
    doc = (t[:, None] >= offsets[None, :]).sum(1) - 1
    start, end = offsets[doc], offsets[doc + 1]
    if c["causal"]:
        own_end = t + 1
        end = torch.minimum(end, torch.maximum(own_end, start + prefix[doc]) if prefix is not None else own_end)
    return (t[None, :] >= start[:, None]) & (t[None, :] < end[:, None])


def _plain_attn(s):
    c, bf = s["case"], torch.bfloat16
    t, group, scale = c["tokens"], c["heads"] // c["kv_heads"], c["d"] ** -0.5
    seen = _visible(c, s["offsets"], s["prefix"])
    pos = torch.arange(t, device="cuda", dtype=torch.float32)
    out = {"o": torch.empty(t, c["heads"], c["d"], dtype=bf, device="cuda"), "lse": torch.empty(c["heads"], t, device="cuda")}
    step = c["mode"] == "step"
    if step:
        out["dq"] = torch.empty_like(out["o"])
        dk, dv = (torch.zeros(t, c["kv_heads"], c["d"], device="cuda") for _ in range(2))
    for h in range(c["heads"]):
        q, k, v = s["q"][:, h].float(), s["k"][:, h // group].float(), s["v"][:, h // group].float()
        z = (q @ k.t()) * scale
        if c["cap"]:
            th = torch.tanh(z / c["cap"])
            z = c["cap"] * th
        if c["alibi"]:
            z = z - s["slopes"][h] * (pos[:, None] - pos[None, :]).abs_()
        z = torch.where(seen, z, -torch.inf)
        top = z.amax(1, keepdim=True)
        p = z.sub_(top).exp_()
        total = p.sum(1, keepdim=True)
        o = (p @ v) / total
        out["o"][:, h] = o.to(bf)
        out["lse"][h] = (top + torch.log(total))[:, 0]
        if step:
            do = s["do"][:, h].float()
            p /= total
            dv[:, h // group] += p.t() @ do
            ds = p.mul_(do @ v.t() - (do * o).sum(1, keepdim=True)).mul_(scale)
            if c["cap"]:
                ds *= 1 - th * th
            out["dq"][:, h] = (ds @ k).to(bf)
            dk[:, h // group] += ds.t() @ q
    if step:
        out["dk"], out["dv"] = dk.to(bf), dv.to(bf)
    return out


def _plain_embed(s):
    c, ids = s["case"], s["ids"]
    inside = (ids >= 0) & (ids < c["vocab"])
    rows = torch.where(inside, ids, 0)
    scale = torch.where(inside, c["scale"], 0.0)[:, None]
    out = {"Y": (s["E"][rows].float() * scale).to(_TYPES[c["dtype"]])}
    if c["mode"] == "step":
        dE = torch.zeros(c["vocab"], c["d"], device="cuda")
        dE.index_add_(0, rows, s["dY"].float() * scale)
        out["dE"] = dE.to(_TYPES[c["grad"]])
    return out


def _plain_clip(s):
    sums = torch.stack([x.float().square().sum() for x in s["grads"]])
    norm = (sums * torch.tensor(s["weights"], device="cuda")).sum().sqrt()
    f = torch.clamp(s["case"]["max_norm"] / norm, max=1.0)
    for x, y in zip(s["grads"], s["clipped"]):
        y.copy_(x.float() * f)
    return {"total": torch.stack([norm, f]), "clipped": s["out"]["clipped"]}


# ------------------------------------------------------------------------------------------------------- the library
def _library(s):
    from paper_2605_01255_b200 import binding as B
    c, o = s["case"], s["out"]
    if c["op"] == "attn":
        if "desc" not in s:   # the plan's and the scratch memory that a program keeps
            s["desc"] = B.make_attn_desc(c["tokens"], c["heads"], c["kv_heads"], c["d"], docs=c["docs"], causal=c["causal"], softcap=c["cap"])
            s["plan"] = B.alloc_attn_workspace(s["desc"], B.ACX_OP_ATTN_PLAN)
            s["ws"] = B.alloc_attn_workspace(s["desc"], B.ACX_OP_ATTN_BWD) if c["mode"] == "step" else None
        d = s["desc"]
        B.acx_attn_plan(d, s["offsets"], s["plan"], prefix=s["prefix"])     # the documents of this batch
        B.acx_attn_fwd(d, s["q"], s["k"], s["v"], s["plan"], o["o"], o["lse"], slopes=s["slopes"])
        if c["mode"] == "step":
            B.acx_attn_bwd(d, s["q"], s["k"], s["v"], s["plan"], o["o"], s["do"], o["lse"], o["dq"], o["dk"], o["dv"], slopes=s["slopes"],
                           ws=s["ws"])
    elif c["op"] == "embed":
        if "desc" not in s:
            s["desc"] = B.make_embed_desc(c["tokens"], c["d"], c["vocab"], c["dtype"], c["grad"], scale=c["scale"])
            s["ws"] = B.alloc_embed_workspace(s["desc"], B.ACX_OP_EMBED_BWD) if c["mode"] == "step" else None
        B.acx_embed_fwd(s["desc"], s["ids"], s["E"], o["Y"])
        if c["mode"] == "step":
            B.acx_embed_bwd(s["desc"], s["ids"], s["dY"], o["dE"], ws=s["ws"])
    else:
        if "list" not in s:   # the gradients' buffers stay where they are from step to step
            s["list"] = B.make_grad_list(s["grads"], weights=s["weights"], out=s["clipped"])
            s["ws"] = B.alloc_grad_workspace(s["list"])
        B.acx_grad_clip(s["list"], c["max_norm"], o["total"], ws=s["ws"])
    return o


def run(state):
    if own:
        return _library(state)
    return {"attn": _plain_attn, "embed": _plain_embed, "clip": _plain_clip}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = dict(dtype=torch.float64, device="cuda")
    if case["op"] == "clip":
        squares = sum(w * float(x.double().square().sum()) for x, w in zip(s["grads"], s["weights"]))
        norm = squares ** 0.5
        f = 1.0 if norm <= case["max_norm"] else case["max_norm"] / norm
        at, size = _buckets(case)
        clipped = {t: torch.zeros(n, **f64) for t, n in size.items()}
        for (t, o), x in zip(at, s["grads"]):
            clipped[t][o:o + len(x)] = x.double() * f
        return {"total": torch.tensor([norm, f], **f64), "clipped": clipped}
    if case["op"] == "embed":
        keep = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["vocab"]))[:, 0]
        out = {"Y": torch.zeros(case["tokens"], case["d"], **f64)}
        out["Y"][keep] = case["scale"] * s["E"][s["ids"][keep]].double()
        if case["mode"] == "step":
            out["dE"] = torch.zeros(case["vocab"], case["d"], **f64)
            out["dE"].index_add_(0, s["ids"][keep], case["scale"] * s["dY"][keep].double())
        return out
    # attention: document by document, the heads of a key head together, blocks of rows
    h, kv, d, step = case["heads"], case["kv_heads"], case["d"], case["mode"] == "step"
    q, k, v = (s[n].double().transpose(0, 1) for n in "qkv")                # heads x tokens x d
    out = {"o": torch.zeros(case["tokens"], h, d, **f64), "lse": torch.zeros(h, case["tokens"], **f64)}
    if step:
        do = s["do"].double().transpose(0, 1)
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros(case["tokens"], kv, d, **f64), dv=torch.zeros(case["tokens"], kv, d, **f64))
    start = 0
    for n, pre in zip(_lengths(case), _prefixes(case)):
        j = torch.arange(n, device="cuda")
        for g in range(h):
            kg, vg = k[g * kv // h, start:start + n], v[g * kv // h, start:start + n]
            for r0 in range(0, n, 4096):
                i = j[r0:r0 + 4096]
                r = slice(start + r0, start + r0 + len(i))
                raw = q[g, r] @ kg.T / d ** 0.5
                z = case["cap"] * torch.tanh(raw / case["cap"]) if case["cap"] else raw
                slope = torch.ones_like(raw) if not case["cap"] else 1 - (z / case["cap"]).square()
                if case["alibi"]:
                    z = z - 2.0 ** (-8.0 * (g + 1) / h) * (i[:, None] - j).abs().double()
                if case["causal"]:
                    z = z.masked_fill((j > i[:, None]) & (j >= pre), -torch.inf)
                lse = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - lse)
                o = p @ vg
                out["o"][r, g], out["lse"][g, r] = o, lse[:, 0]
                if step:
                    dp = do[g, r] @ vg.T
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * slope / d ** 0.5
                    out["dq"][r, g] = ds @ kg
                    out["dk"][start:start + n, g * kv // h] += ds.T @ q[g, r]
                    out["dv"][start:start + n, g * kv // h] += p.T @ do[g, r]
                del raw, z, slope, p
        start += n
    return out
