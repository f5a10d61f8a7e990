"""A training step through everything between the linears and behind the last one: a stack of gated MLP blocks with
sandwich norms and a language-model head, every arithmetic step in libacx.

    y_0 = N(h_0) w_pre[0]
    block l:  [G | U] = y_l Wgu^T  (factor XS kept),  H = silu(G) U  (G, U kept in 8 bits),  b = H Wdn^T  (factor kept),
              h_{l+1} = h_l + alpha gate[l] N(b) w_post[l],  y_{l+1} = N(h_{l+1}) w_pre[l+1]  (h_l, b kept in 8 bits)
    loss = cross entropy of y_L Whead^T at the targets, mean over the trained tokens

The backward pass runs it in reverse from what was kept; the weight gradients of the linears come out as factors and go
straight into AdamW (`acx_reconstruct_adamw`), the head's and the vectors' are left in `grads`.  Attention is not part of
this library, so the token mixing a real model has between these blocks is absent here.

    python -m paper_2605_01255_b200.mlp_lm [steps]      # a few steps on one synthetic batch: the loss falls
"""
from __future__ import annotations

import sys
from dataclasses import dataclass
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
        ones = lambda: torch.ones(d, dtype=bf, device=self.dev)  # noqa: E731
        self.w_pre = [ones() for _ in range(L + 1)]
        self.w_post, self.gate = [ones() for _ in range(L)], [ones() for _ in range(L)]
        # what the backward pass needs: 8-bit checkpoints, the linears' factors, the norms' scales
        q8 = lambda cols: B.q8_empty(m, cols, self.dev)  # noqa: E731
        self.q_h = [q8(d) for _ in range(L + 1)]
        self.q_b = [q8(d) for _ in range(L)]
        self.q_g, self.q_u = [q8(n) for _ in range(L)], [q8(n) for _ in range(L)]
        self.rstd_pre = [new(m, dt=f32) for _ in range(L + 1)]
        self.rstd_post = [new(m, dt=f32) for _ in range(L)]
        self.xs = [{"gu": new(m, s.r), "dn": new(m, s.r)} for _ in range(L)]
        self.lse, self.loss, self.total = new(m, dt=f32), new(m, dt=f32), new(2, dt=f32)
        # scratch that every layer uses again
        self.h = [new(m, d), new(m, d)]
        self.y, self.b, self.gu, self.hid = new(m, d), new(m, d), new(m, 2 * n), new(m, n)
        self.dh = [new(m, d), new(m, d)]
        self.dy, self.db, self.dgu, self.dhid = new(m, d), new(m, d), new(m, 2 * n), new(m, n)
        self.factor = {"gu": new(2 * n, s.r, dt=f32), "dn": new(d, s.r, dt=f32)}
        self.grads: Dict[str, List[torch.Tensor]] = {
            "w_pre": [new(d, dt=f32) for _ in range(L + 1)], "w_post": [new(d, dt=f32) for _ in range(L)],
            "gate": [new(d, dt=f32) for _ in range(L)], "head": [new(s.vocab, d)]}
        self.rows_d, self.rows_n = B.make_rows_desc(m, d, "bf16"), B.make_rows_desc(m, n, "bf16")
        self.ce = B.make_ce_desc(m, d, s.vocab)
        self.ws_ce = B.alloc_ce_workspace(self.ce, B.ACX_OP_CE_BWD, self.dev)
        self.ws_norm = B.alloc_rows_workspace(self.rows_d, B.ACX_OP_NORM_BWD, self.dev)
        need = max(B.acx_workspace_bytes(self._desc(0, k), op) for k in ("gu", "dn")
                   for op in (B.ACX_OP_FWD, B.ACX_OP_BWD, B.ACX_OP_RECONSTRUCT))
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device=self.dev)

    def _desc(self, layer: int, kind: str):
        s = self.s
        d_in, d_out = (s.d, 2 * s.inter) if kind == "gu" else (s.inter, s.d)
        return B.make_desc(s.tokens, d_in, d_out, s.r, I.sketch_seed(0, layer, 0 if kind == "gu" else 1, self.step_no), "bf16")

    def kept_bytes(self) -> Dict[str, int]:
        """Activation memory between forward and backward: what is kept, and what keeping the same tensors in bf16 would take."""
        size = lambda ts: sum(t.numel() * t.element_size() for t in ts)  # noqa: E731
        s = self.s
        kept = size(t for group in (self.q_h, self.q_b, self.q_g, self.q_u) for q in group for t in q)
        kept += size(self.rstd_pre) + size(self.rstd_post) + size(t for x in self.xs for t in x.values())
        kept += size([self.y, self.lse, self.loss, self.total])      # what the head's backward reads: its input is kept as it is
        # h, b, the norms' outputs (the linears' inputs), G, U and H of every layer; the logits are not counted on either side
        plain = 2 * s.tokens * (s.layers * (3 * s.d + 3 * s.inter) + 2 * s.d)
        return {"kept": kept, "bf16": plain, "logits_bf16": 2 * s.tokens * s.vocab}

    def forward(self, h0: torch.Tensor, targets: torch.Tensor, weight=None) -> torch.Tensor:
        """total = (sum of weight * loss, sum of weight) of the batch, on the device; keeps what `backward` needs."""
        s, n = self.s, self.s.inter
        self.targets, self.weight = targets, weight
        B.acx_norm_join_fwd(self.rows_d, h0, None, None, None, self.w_pre[0], None, self.y, *self.q_h[0], None, None, None, self.rstd_pre[0],
                            eps=s.eps)
        h = h0
        for l in range(s.layers):
            B.acx_linear_fwd(self._desc(l, "gu"), self.y, self.w[l]["gu"], self.gu, self.xs[l]["gu"], self.ws)
            B.acx_swiglu_fwd(self.rows_n, self.gu[:, :n], self.gu[:, n:], self.hid, *self.q_g[l], *self.q_u[l])
            B.acx_linear_fwd(self._desc(l, "dn"), self.hid, self.w[l]["dn"], self.b, self.xs[l]["dn"], self.ws)
            B.acx_norm_join_fwd(self.rows_d, h, self.b, self.w_post[l], self.gate[l], self.w_pre[l + 1], self.h[l % 2], self.y,
                                *self.q_h[l + 1], *self.q_b[l], self.rstd_post[l], self.rstd_pre[l + 1], eps=s.eps, alpha=s.alpha)
            h = self.h[l % 2]
        B.acx_linear_ce_fwd(self.ce, self.y, self.head, targets, self.loss, self.lse, self.total, weight, self.ws_ce)
        return self.total

    def backward(self, lr: float = 0.0, **hyper) -> torch.Tensor:
        """Gradient of the mean loss with respect to h0; with lr > 0 every linear takes its AdamW step as soon as its factor is
        known (after the last use of its weights in this pass)."""
        s, n = self.s, self.s.inter
        B.acx_linear_ce_bwd(self.ce, self.y, self.head, self.targets, self.lse, self.dy, self.grads["head"][0], loss=self.loss,
                            weight=self.weight, denom=self.total[1:], ws=self.ws_ce)
        dh = None
        for l in range(s.layers - 1, -1, -1):
            out = self.dh[l % 2]
            B.acx_norm_join_bwd(self.rows_d, self.dy, dh, self.w_post[l], self.gate[l], self.w_pre[l + 1], *self.q_h[l + 1], *self.q_b[l],
                                self.rstd_post[l], self.rstd_pre[l + 1], out, self.db, self.grads["w_post"][l], self.grads["gate"][l],
                                self.grads["w_pre"][l + 1], alpha=s.alpha, ws=self.ws_norm)
            dh = out
            B.acx_linear_bwd(self._desc(l, "dn"), self.db, self.w[l]["dn"], self.xs[l]["dn"], self.dhid, self.factor["dn"], self.ws)
            self._update(l, "dn", lr, hyper)
            B.acx_swiglu_bwd(self.rows_n, self.dhid, *self.q_g[l], *self.q_u[l], self.dgu[:, :n], self.dgu[:, n:])
            B.acx_linear_bwd(self._desc(l, "gu"), self.dgu, self.w[l]["gu"], self.xs[l]["gu"], self.dy, self.factor["gu"], self.ws)
            self._update(l, "gu", lr, hyper)
        dh0 = self.dh[1] if dh is not self.dh[1] else self.dh[0]
        B.acx_norm_join_bwd(self.rows_d, self.dy, dh, None, None, self.w_pre[0], *self.q_h[0], None, None, None, self.rstd_pre[0], dh0, None, None,
                            None, self.grads["w_pre"][0], ws=self.ws_norm)
        if lr > 0:
            self.step_no += 1
        return dh0

    def _update(self, l: int, kind: str, lr: float, hyper) -> None:
        if lr > 0:
            m, v = self.moments[l][kind]
            B.acx_reconstruct_adamw(self._desc(l, kind), self.factor[kind], self.master[l][kind], m, v, self.w[l][kind],
                                    step=self.step_no + 1, lr=lr, ws=self.ws, **hyper)


def synthetic_batch(s: Sizes, seed: int = 1, device="cuda"):
    """Hidden states and targets of one batch; the first eighth of the tokens is not trained on."""
    g = torch.Generator(device=device).manual_seed(seed)
    h0 = torch.randn(s.tokens, s.d, generator=g, device=device).to(torch.bfloat16)
    y = torch.randint(0, s.vocab, (s.tokens,), generator=g, device=device)
    y[: s.tokens // 8] = -100
    return h0, y


def main(argv) -> int:
    steps = int(argv[0]) if argv else 20
    s = Sizes(tokens=4096, d=896, inter=4864, vocab=32000, layers=4, r=64)
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
