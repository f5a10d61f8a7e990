"""A training step through everything between the linears and behind the last one: a stack of gated MLP blocks with
sandwich norms and a language-model head, every arithmetic step in libacx.

    y_0 = N(h_0) w_pre[0]
    block l:  [G | U] = y_l Wgu^T  (factor XS kept),  H = silu(G) U  (G, U kept in 8 bits),  b = H Wdn^T  (factor kept),
              h_{l+1} = h_l + alpha gate[l] N(b) w_post[l],  y_{l+1} = N(h_{l+1}) w_pre[l+1]  (h_l, b kept in 8 bits)
    loss = cross entropy of y_L Whead^T at the targets, mean over the trained tokens

The backward pass runs it in reverse from what was kept; the weight gradients of the linears come out as factors and go
straight into AdamW (`acx_reconstruct_adamw`), the head's and the vectors' are left in `grads`.

With `heads` the block has attention over packed documents in front, a sub-block between two norms of its own:
    [Q | K | V] = y Wqkv^T  (factor kept, and Q, K, V),  a = attention within the documents (kept, with its lse),  b = a Wo^T  (factor kept).
With `tied` the batch is word ids: h_0 = sqrt(d) Whead[ids], whose gradient is added to the head's.  With `max_norm` the gradients of
all linears (as factors), of the vectors and of the head are clipped together before any weight is updated; a step whose norm is not a
number (an infinity or a NaN among the gradients) is left out, weights, moments and step count as they were.

    python -m paper_2605_01255_b200.mlp_lm [steps] [full]     # a few steps on one synthetic batch: the loss falls; full: all of these
"""
from __future__ import annotations

import math
import sys
from dataclasses import dataclass, replace
from typing import Dict, List

import torch

from . import binding as B
from . import inputs as I


@dataclass
class Sizes:
    tokens: int
    d: int
    inter: int
    vocab: int
    layers: int
    r: int
    alpha: float = 1.0
    eps: float = 1e-5
    heads: int = 0            # query heads of the attention in front of every MLP, 0: none
    kv_heads: int = 0
    head_dim: int = 0
    docs: int = 1             # documents in a batch
    tied: bool = False        # the head's rows are the embeddings too
    max_norm: float = 0.0     # 0: no clipping


class MlpLm:
    """Weights, optimizer state, kept activations and call order; allocates everything once."""

    def __init__(self, s: Sizes, seed: int = 0, device="cuda"):
        self.s, self.dev, self.step_no = s, torch.device(device), 0
        g = torch.Generator(device=self.dev).manual_seed(seed)
        bf, f32 = torch.bfloat16, torch.float32
        new = lambda *shape, dt=bf: torch.empty(*shape, dtype=dt, device=self.dev)  # noqa: E731
        normal = lambda *shape: torch.randn(*shape, generator=g, device=self.dev)  # noqa: E731
        m, d, n, L = s.tokens, s.d, s.inter, s.layers
        # linears: fp32 master weights with AdamW moments, bf16 copies for the products
        self.master = [{"gu": normal(2 * n, d) * d ** -0.5, "dn": normal(d, n) * n ** -0.5} for _ in range(L)]
        self.moments = [{k: (torch.zeros_like(w), torch.zeros_like(w)) for k, w in lw.items()} for lw in self.master]
        self.w = [{k: w.to(bf) for k, w in lw.items()} for lw in self.master]
        self.head = (normal(s.vocab, d) * d ** -0.5).to(bf)
        # sub-blocks, each between two norms: (layer, what it is)
        self.subs = [(l, k) for l in range(L) for k in (("attn", "mlp") if s.heads else ("mlp",))]
        ns = len(self.subs)
        if s.heads:
            hd, wide = s.heads * s.head_dim, (s.heads + 2 * s.kv_heads) * s.head_dim
            for l in range(L):
                more = {"qkv": normal(wide, d) * d ** -0.5, "o": normal(d, hd) * hd ** -0.5}
                self.master[l].update(more)
                self.moments[l].update({k: (torch.zeros_like(w), torch.zeros_like(w)) for k, w in more.items()})
                self.w[l].update({k: w.to(bf) for k, w in more.items()})
        ones = lambda: torch.ones(d, dtype=bf, device=self.dev)  # noqa: E731
        self.w_pre = [ones() for _ in range(ns + 1)]
        self.w_post, self.gate = [ones() for _ in range(ns)], [ones() for _ in range(ns)]
        # what the backward pass needs: 8-bit checkpoints, the linears' factors, the norms' scales
        q8 = lambda cols: B.q8_empty(m, cols, self.dev)  # noqa: E731
        self.q_h = [q8(d) for _ in range(ns + 1)]
        self.q_b = [q8(d) for _ in range(ns)]
        self.q_g, self.q_u = [q8(n) for _ in range(L)], [q8(n) for _ in range(L)]
        self.rstd_pre = [new(m, dt=f32) for _ in range(ns + 1)]
        self.rstd_post = [new(m, dt=f32) for _ in range(ns)]
        self.xs = [{k: new(m, s.r) for k in lw} for lw in self.w]
        self.lse, self.loss, self.total = new(m, dt=f32), new(m, dt=f32), new(2, dt=f32)
        # scratch that every layer uses again
        self.h = [new(m, d), new(m, d)]
        self.y, self.b, self.gu, self.hid = new(m, d), new(m, d), new(m, 2 * n), new(m, n)
        self.dh = [new(m, d), new(m, d)]
        self.dy, self.db, self.dgu, self.dhid = new(m, d), new(m, d), new(m, 2 * n), new(m, n)
        # factors of the linears' gradients: one of a kind, or all of them where they wait for their common norm
        outs = {"gu": 2 * n, "dn": d, **({"qkv": wide, "o": d} if s.heads else {})}
        one = lambda: {k: new(rows, s.r, dt=f32) for k, rows in outs.items()}  # noqa: E731
        self.factor = one()
        self.factors = [one() if s.max_norm > 0 else self.factor for _ in range(L)]
        self.grads: Dict[str, List[torch.Tensor]] = {
            "w_pre": [new(d, dt=f32) for _ in range(ns + 1)], "w_post": [new(d, dt=f32) for _ in range(ns)],
            "gate": [new(d, dt=f32) for _ in range(ns)], "head": [new(s.vocab, d)]}
        self.rows_d, self.rows_n = B.make_rows_desc(m, d, "bf16"), B.make_rows_desc(m, n, "bf16")
        self.ce = B.make_ce_desc(m, d, s.vocab)
        self.ws_ce = B.alloc_ce_workspace(self.ce, B.ACX_OP_CE_BWD, self.dev)
        self.ws_norm = B.alloc_rows_workspace(self.rows_d, B.ACX_OP_NORM_BWD, self.dev)
        need = max((B.acx_workspace_bytes(self._desc(0, k), op) for lw in self.w[:1] for k in lw
                    for op in (B.ACX_OP_FWD, B.ACX_OP_BWD, B.ACX_OP_RECONSTRUCT)), default=0)
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device=self.dev)
        if s.heads:
            self.attn = B.make_attn_desc(m, s.heads, s.kv_heads, s.head_dim, s.docs)
            self.plan = B.alloc_attn_workspace(self.attn, B.ACX_OP_ATTN_PLAN, self.dev)
            self.ws_attn = B.alloc_attn_workspace(self.attn, B.ACX_OP_ATTN_BWD, self.dev)
            self.even = torch.tensor([m * i // s.docs for i in range(s.docs + 1)], dtype=torch.int32, device=self.dev)
            # the order of the tokens: a penalty on their distance, another one for every head
            self.slopes = 2.0 ** (-8.0 * torch.arange(1, s.heads + 1, dtype=f32, device=self.dev) / s.heads)
            self.qkv, self.o = [new(m, wide) for _ in range(L)], [new(m, hd) for _ in range(L)]
            self.lse_attn = [new(s.heads, m, dt=f32) for _ in range(L)]
            self.do, self.dqkv = new(m, hd), new(m, wide)
        if s.tied:
            self.table = B.make_embed_desc(m, d, s.vocab, bf, scale=d ** 0.5)
            self.ws_table = B.alloc_embed_workspace(self.table, B.ACX_OP_EMBED_BWD, self.dev)
        if s.max_norm > 0:
            # a factor counts as often as its gradient A S^T does on average over the sketches
            parts = [(a, B.grad_factor_weight(self.w[l][k].shape[1], s.r)) for l in range(L) for k, a in self.factors[l].items()]
            parts += [(t, 1.0) for ts in self.grads.values() for t in ts]
            self.clip = B.make_grad_list([t for t, _ in parts], [w for _, w in parts])
            self.norm, self.ws_clip = new(2, dt=f32), B.alloc_grad_workspace(self.clip)

    def _desc(self, layer: int, kind: str):
        d_out, d_in = self.w[layer][kind].shape
        return B.make_desc(self.s.tokens, d_in, d_out, self.s.r, I.sketch_seed(0, layer, ("gu", "dn", "qkv", "o").index(kind), self.step_no), "bf16")

    def _heads(self, t: torch.Tensor):
        """Query, key and value heads of [Q | K | V]: views."""
        s = self.s
        parts = t.split([s.heads * s.head_dim, s.kv_heads * s.head_dim, s.kv_heads * s.head_dim], dim=1)
        return [x.unflatten(1, (-1, s.head_dim)) for x in parts]

    def kept_bytes(self) -> Dict[str, int]:
        """Activation memory between forward and backward: what is kept, and what keeping the same tensors in bf16 would take."""
        size = lambda ts: sum(t.numel() * t.element_size() for t in ts)  # noqa: E731
        s = self.s
        kept = size(t for group in (self.q_h, self.q_b, self.q_g, self.q_u) for q in group for t in q)
        kept += size(self.rstd_pre) + size(self.rstd_post) + size(t for x in self.xs for t in x.values())
        kept += size([self.y, self.lse, self.loss, self.total])      # what the head's backward reads: its input is kept as it is
        # h, b, the norms' outputs (the linears' inputs), G, U and H of every layer; the logits are not counted on either side
        plain = 2 * s.tokens * (s.layers * (3 * s.d + 3 * s.inter) + 2 * s.d)
        if s.heads:
            attn = size(self.qkv) + size(self.o) + size(self.lse_attn)
            kept += attn + self.plan.numel() + size([self.slopes])
            plain += attn + s.layers * 2 * s.tokens * 3 * s.d
        return {"kept": kept, "bf16": plain, "logits_bf16": 2 * s.tokens * s.vocab}

    def forward(self, h0: torch.Tensor, targets: torch.Tensor, weight=None, offsets=None) -> torch.Tensor:
        """total = (sum of weight * loss, sum of weight) of the batch, on the device; keeps what `backward` needs.  h0: hidden states, or
        with `tied` word ids; offsets: where the documents start and the last one ends (int32, on the device), None: all equally long."""
        s, n = self.s, self.s.inter
        self.targets, self.weight, self.ids = targets, weight, h0
        if s.tied:
            B.acx_embed_fwd(self.table, h0, self.head, self.h[1])
            h0 = self.h[1]
        if s.heads:
            B.acx_attn_plan(self.attn, self.even if offsets is None else offsets, self.plan)
        B.acx_norm_join_fwd(self.rows_d, h0, None, None, None, self.w_pre[0], None, self.y, *self.q_h[0], None, None, None, self.rstd_pre[0],
                            eps=s.eps)
        h = h0
        for i, (l, kind) in enumerate(self.subs):
            if kind == "attn":
                B.acx_linear_fwd(self._desc(l, "qkv"), self.y, self.w[l]["qkv"], self.qkv[l], self.xs[l]["qkv"], self.ws)
                B.acx_attn_fwd(self.attn, *self._heads(self.qkv[l]), self.plan, self.o[l].view(s.tokens, s.heads, -1), self.lse_attn[l],
                               slopes=self.slopes)
                B.acx_linear_fwd(self._desc(l, "o"), self.o[l], self.w[l]["o"], self.b, self.xs[l]["o"], self.ws)
            else:
                B.acx_linear_fwd(self._desc(l, "gu"), self.y, self.w[l]["gu"], self.gu, self.xs[l]["gu"], self.ws)
                B.acx_swiglu_fwd(self.rows_n, self.gu[:, :n], self.gu[:, n:], self.hid, *self.q_g[l], *self.q_u[l])
                B.acx_linear_fwd(self._desc(l, "dn"), self.hid, self.w[l]["dn"], self.b, self.xs[l]["dn"], self.ws)
            B.acx_norm_join_fwd(self.rows_d, h, self.b, self.w_post[i], self.gate[i], self.w_pre[i + 1], self.h[i % 2], self.y,
                                *self.q_h[i + 1], *self.q_b[i], self.rstd_post[i], self.rstd_pre[i + 1], eps=s.eps, alpha=s.alpha)
            h = self.h[i % 2]
        B.acx_linear_ce_fwd(self.ce, self.y, self.head, targets, self.loss, self.lse, self.total, weight, self.ws_ce)
        return self.total

    def backward(self, lr: float = 0.0, **hyper) -> torch.Tensor:
        """Gradient of the mean loss with respect to h0; with lr > 0 every linear takes its AdamW step as soon as its factor is
        known (after the last use of its weights in this pass), or, where gradients are clipped, once all of them are: the host then
        waits for the norm, and a step whose norm is not a number is left out (in a graph's capture it cannot: every step is taken)."""
        s, n = self.s, self.s.inter
        clip = s.max_norm > 0
        B.acx_linear_ce_bwd(self.ce, self.y, self.head, self.targets, self.lse, self.dy, self.grads["head"][0], loss=self.loss,
                            weight=self.weight, denom=self.total[1:], ws=self.ws_ce)
        dh = None
        for i in range(len(self.subs) - 1, -1, -1):
            l, kind = self.subs[i]
            out = self.dh[i % 2]
            B.acx_norm_join_bwd(self.rows_d, self.dy, dh, self.w_post[i], self.gate[i], self.w_pre[i + 1], *self.q_h[i + 1], *self.q_b[i],
                                self.rstd_post[i], self.rstd_pre[i + 1], out, self.db, self.grads["w_post"][i], self.grads["gate"][i],
                                self.grads["w_pre"][i + 1], alpha=s.alpha, ws=self.ws_norm)
            dh = out
            second, first = ("o", "qkv") if kind == "attn" else ("dn", "gu")
            B.acx_linear_bwd(self._desc(l, second), self.db, self.w[l][second], self.xs[l][second], self.do if kind == "attn" else self.dhid,
                             self.factors[l][second], self.ws)
            if not clip:
                self._update(l, second, lr, hyper)
            if kind == "attn":
                o, do = (t.view(s.tokens, s.heads, -1) for t in (self.o[l], self.do))
                B.acx_attn_bwd(self.attn, *self._heads(self.qkv[l]), self.plan, o, do, self.lse_attn[l], *self._heads(self.dqkv),
                               slopes=self.slopes, ws=self.ws_attn)
                inner = self.dqkv
            else:
                B.acx_swiglu_bwd(self.rows_n, self.dhid, *self.q_g[l], *self.q_u[l], self.dgu[:, :n], self.dgu[:, n:])
                inner = self.dgu
            B.acx_linear_bwd(self._desc(l, first), inner, self.w[l][first], self.xs[l][first], self.dy, self.factors[l][first], self.ws)
            if not clip:
                self._update(l, first, lr, hyper)
        dh0 = self.dh[1] if dh is not self.dh[1] else self.dh[0]
        B.acx_norm_join_bwd(self.rows_d, self.dy, dh, None, None, self.w_pre[0], *self.q_h[0], None, None, None, self.rstd_pre[0], dh0, None, None,
                            None, self.grads["w_pre"][0], ws=self.ws_norm)
        if s.tied:
            B.acx_embed_bwd(self.table, self.ids, dh0, self.grads["head"][0], beta=1.0, ws=self.ws_table)
        if clip:
            B.acx_grad_clip(self.clip, s.max_norm, self.norm, ws=self.ws_clip)
            if lr > 0 and not (self.norm.is_cuda and torch.cuda.is_current_stream_capturing()):
                norm, f = self.norm.tolist()
                if not math.isfinite(norm) and not f < 1:      # (one beyond fp32 reads as infinity, but has its factor)
                    return dh0
            for l in range(s.layers):
                for kind in self.factors[l]:
                    self._update(l, kind, lr, hyper)
        if lr > 0:
            self.step_no += 1
        return dh0

    def _update(self, l: int, kind: str, lr: float, hyper) -> None:
        if lr > 0:
            m, v = self.moments[l][kind]
            B.acx_reconstruct_adamw(self._desc(l, kind), self.factors[l][kind], self.master[l][kind], m, v, self.w[l][kind],
                                    step=self.step_no + 1, lr=lr, ws=self.ws, **hyper)


def synthetic_batch(s: Sizes, seed: int = 1, device="cuda"):
    """Hidden states (with `tied` word ids) and targets of one batch; the first eighth of the tokens is not trained on."""
    g = torch.Generator(device=device).manual_seed(seed)
    h0 = torch.randn(s.tokens, s.d, generator=g, device=device).to(torch.bfloat16)
    y = torch.randint(0, s.vocab, (s.tokens,), generator=g, device=device)
    y[: s.tokens // 8] = -100
    if s.tied:
        return torch.randint(0, s.vocab, (s.tokens,), generator=g, device=device), y
    return h0, y


def main(argv) -> int:
    full = "full" in argv
    argv = [a for a in argv if a != "full"]
    steps = int(argv[0]) if argv else 20
    s = Sizes(tokens=4096, d=896, inter=4864, vocab=32000, layers=4, r=64)
    if full:
        s = replace(s, heads=14, kv_heads=2, head_dim=64, docs=5, tied=True, max_norm=1.0)
    model = MlpLm(s)
    h0, y = synthetic_batch(s)
    losses = []
    for _ in range(steps):
        losses.append(model.forward(h0, y).clone())
        model.backward(lr=1e-3)
    st = B.acx_last_device_status()
    if st != B.ACX_OK:
        raise SystemExit(B.status_string(st))
    means = [float(t[0] / t[1]) for t in losses]
    kept = model.kept_bytes()
    print("loss %s" % " ".join("%.3f" % x for x in means))
    print("activations kept %.1f MB (in bf16 %.1f MB); logits never stored %.1f MB" % tuple(kept[k] / 1e6 for k in ("kept", "bf16", "logits_bf16")))
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv[1:]))
