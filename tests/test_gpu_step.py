"""Attention, the embedding table and the clipping as a training step uses them: together, in captured graphs, on several streams, with
batches that hold anything where no document is; and where offsets pass 32 bits."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import mlp_lm as M

BF, NAN = torch.bfloat16, float("nan")
gpu = pytest.mark.gpu
FULL = dict(heads=6, kv_heads=2, head_dim=24, docs=4, tied=True)


def offsets_of(*ends):
    return torch.tensor([0, *ends], dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------------ the step
def reference(model, ids, y, offsets):
    """Loss and gradients of the same network by autograd in float64."""
    s, dbl = model.s, torch.float64
    leaf = lambda t: t.detach().to(dbl).requires_grad_()  # noqa: E731
    p = {"head": leaf(model.head), "w": [{k: leaf(w) for k, w in lw.items()} for lw in model.w]}
    p.update({k: [leaf(t) for t in getattr(model, k)] for k in ("w_pre", "w_post", "gate")})
    norm = lambda x, w: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps) * w  # noqa: E731
    pos = torch.arange(s.tokens, device=ids.device)
    doc = torch.bucketize(pos, offsets.long()[1:], right=True)
    inside = pos < offsets[-1]
    seen = (doc[:, None] == doc[None, :]) & (pos[None, :] <= pos[:, None]) & inside[:, None]
    far = (pos[:, None] - pos[None, :]).abs().to(dbl)

    def attention(x, w):
        q, k, v = (t.unflatten(1, (-1, s.head_dim)) for t in (x @ w["qkv"].T).split([s.heads * s.head_dim] + 2 * [s.kv_heads * s.head_dim], dim=1))
        k, v = (t.repeat_interleave(s.heads // s.kv_heads, dim=1) for t in (k, v))
        z = torch.einsum("ihd,jhd->hij", q, k) * s.head_dim ** -0.5 - model.slopes.to(dbl)[:, None, None] * far
        a = torch.softmax(z.masked_fill(~seen, -1e300), dim=-1) * inside[None, :, None]
        return torch.einsum("hij,jhd->ihd", a, v).flatten(1) @ w["o"].T

    h0 = (p["head"][ids] * s.d ** 0.5).detach().requires_grad_()
    # h0 is a leaf here, so that its gradient is at hand; the table's part of it is added below
    h, x = h0, norm(h0, p["w_pre"][0])
    for i, (l, kind) in enumerate(model.subs):
        w = p["w"][l]
        if kind == "attn":
            b = attention(x, w)
        else:
            g, u = (x @ w["gu"].T).split(s.inter, dim=1)
            b = (g * torch.sigmoid(g) * u) @ w["dn"].T
        h = h + s.alpha * p["gate"][i] * norm(b, p["w_post"][i])
        x = norm(h, p["w_pre"][i + 1])
    loss = torch.nn.functional.cross_entropy(x @ p["head"].T, y, ignore_index=-100)
    loss.backward()
    p["h0"] = h0
    p["head"].grad.index_add_(0, ids, h0.grad * s.d ** 0.5)
    return loss, p


def rel(a, b):
    return float((a.to(torch.float64) - b).norm() / b.norm())


@gpu
def test_step_against_autograd():
    s = M.Sizes(tokens=333, d=136, inter=264, vocab=1003, layers=2, r=32, alpha=0.8, max_norm=0.25, **FULL)
    model = M.MlpLm(s)
    ids, y = M.synthetic_batch(s)
    offsets = offsets_of(1, 130, 130, 300)      # one token, 129, none, 170; the last 33 tokens are padding
    total = model.forward(ids, y, offsets=offsets)
    dh0 = model.backward()
    assert B.acx_last_device_status() == B.ACX_OK
    loss, p = reference(model, ids, y, offsets)
    norm, f = model.norm.double().tolist()
    # as for the step without attention (bf16 storage 2^-9 each, 8-bit checkpoints 0.8 % each, random), but eight checkpoints a
    # layer and some twenty roundings: sqrt(16) 0.8 % + sqrt(40) 0.2 % = 4.5 %, and a third to spare
    assert abs(float(total[0] / total[1]) - float(loss.detach())) <= 1e-2 * float(loss.detach())
    tol = 6e-2
    assert rel(dh0, p["h0"].grad) <= tol
    assert 0 < f < 1 and abs(norm * f - s.max_norm) <= 1e-6 * s.max_norm
    assert rel(model.grads["head"][0] / f, p["head"].grad) <= tol
    for k in ("w_pre", "w_post", "gate"):
        for a, b in zip(model.grads[k], p[k]):
            assert rel(a / f, b.grad) <= tol, k
    # the norm is that of what was clipped: every bf16 element off by 2^-8 at most, of its own size
    clipped = sum(float(t.double().square().sum()) for ts in model.grads.values() for t in ts)
    clipped += sum(model.w[l][k].shape[1] / s.r * float(a.double().square().sum()) for l in range(s.layers) for k, a in model.factors[l].items())
    assert abs(clipped ** 0.5 - s.max_norm) <= 2.0 ** -8 * s.max_norm
    # A = dW S with E[S S^T] = I, so |A|^2 is |dW|^2 on average, and a factor's weight d_in / r makes it what |A S^T|^2, the gradient that
    # the optimizer sees, is on average.  One sketch: a standard deviation of sqrt(2 / r) = 25 % at most (dW of rank one), three of them.
    for l, lw in enumerate(p["w"]):
        for k, w in lw.items():
            got = float((model.factors[l][k].double() / f).square().sum()) / float(w.grad.square().sum())
            assert 0.25 < got < 1.75, (l, k, got)


@gpu
def test_a_step_runs_and_updates():
    s = M.Sizes(tokens=512, d=128, inter=256, vocab=999, layers=2, r=32, max_norm=1.0, heads=4, kv_heads=1, head_dim=32, docs=3, tied=True)
    model = M.MlpLm(s)
    ids, y = M.synthetic_batch(s)
    before = [{k: w.clone() for k, w in lw.items()} for lw in model.w]
    for _ in range(3):
        t = model.forward(ids, y)
        dh0 = model.backward(lr=1e-3)
        assert torch.isfinite(t).all() and torch.isfinite(dh0.float()).all() and 0 < float(model.norm[1]) <= 1
    assert B.acx_last_device_status() == B.ACX_OK
    assert all(not torch.equal(w, b[k]) for lw, b in zip(model.w, before) for k, w in lw.items())


def test_weights_of_a_step_without_attention_stay_the_same():
    s = dict(tokens=32, d=64, inter=128, vocab=100, layers=2, r=16)
    a, b = M.MlpLm(M.Sizes(**s), device="cpu"), M.MlpLm(M.Sizes(**s, **FULL), device="cpu")
    assert torch.equal(a.head, b.head)
    for x, z in zip(a.w, b.w):
        assert set(z) == set(x) | {"qkv", "o"} and all(torch.equal(x[k], z[k]) for k in x)


def test_kept_bytes_are_the_bytes_the_backward_reads(monkeypatch):
    s = M.Sizes(tokens=96, d=64, inter=128, vocab=100, layers=2, r=16, **FULL)
    model = M.MlpLm(s, device="cpu")
    ids, y = M.synthetic_batch(s, device="cpu")
    read = {}

    def record(*written):
        def call(desc, *args, **kw):
            for t in [t for i, t in enumerate(args) if i not in written] + [kw.get(k) for k in ("loss", "weight", "denom", "slopes")]:
                if isinstance(t, torch.Tensor):
                    read[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
        return call

    for name in ("acx_norm_join_fwd", "acx_linear_fwd", "acx_swiglu_fwd", "acx_linear_ce_fwd", "acx_attn_plan", "acx_attn_fwd", "acx_embed_fwd"):
        monkeypatch.setattr(B, name, lambda *a, **k: None)
    model.forward(ids, y)
    for name, written in (("acx_linear_ce_bwd", (4, 5)), ("acx_norm_join_bwd", (11, 12, 13, 14, 15)), ("acx_linear_bwd", (3, 4, 5)),
                          ("acx_swiglu_bwd", (5, 6)), ("acx_attn_bwd", (7, 8, 9)), ("acx_embed_bwd", (2,))):
        monkeypatch.setattr(B, name, record(*written))
    model.backward()
    for t in [model.head, *model.w_pre, *model.w_post, *model.gate, *(w for lw in model.w for w in lw.values()),      # weights
              model.dy, model.db, model.dgu, model.dhid, model.do, model.dqkv, *model.dh, ids, y]:                    # gradients, the batch
        read.pop(t.untyped_storage().data_ptr(), None)
    assert model.kept_bytes()["kept"] == sum(read.values())


# ------------------------------------------------------------------------------------------------- graphs and streams
class Batch:
    """A lookup, attention over its documents, the way back into the table, and the clipping of all three gradients."""

    def __init__(self, T=700, H=4, K=2, d=64, vocab=501, docs=4, seed=0, scratch=None):
        self.T, self.docs, self.vocab = T, docs, vocab
        g = torch.Generator().manual_seed(seed)
        wide = (H + 2 * K) * d
        self.E = (0.8 * torch.randn(vocab, wide, generator=g)).to(BF).cuda()
        self.ids = torch.zeros(T, dtype=torch.int64, device="cuda")
        self.offsets = torch.zeros(docs + 1, dtype=torch.int32, device="cuda")
        self.do = torch.zeros(T, H, d, dtype=BF, device="cuda")
        self.attn, self.table = B.make_attn_desc(T, H, K, d, docs), B.make_embed_desc(T, wide, vocab, BF, torch.float32, scale=1.25)
        self.x, self.dx = torch.empty(T, wide, dtype=BF, device="cuda"), torch.empty(T, wide, dtype=BF, device="cuda")
        self.o, self.lse = torch.empty(T, H, d, dtype=BF, device="cuda"), torch.empty(H, T, device="cuda")
        self.dE = torch.empty(vocab, wide, device="cuda")
        self.total = torch.empty(2, device="cuda")
        self.list = B.make_grad_list([self.dE, self.dx], [1.0, 0.5])
        self.plan = B.alloc_attn_workspace(self.attn, B.ACX_OP_ATTN_PLAN)
        self.scratch = scratch or (B.alloc_attn_workspace(self.attn, B.ACX_OP_ATTN_BWD), B.alloc_embed_workspace(self.table, B.ACX_OP_EMBED_BWD),
                                   B.alloc_grad_workspace(self.list))
        cut = [H * d, (H + K) * d]
        heads = lambda t: [p.unflatten(1, (-1, d)) for p in torch.tensor_split(t, cut, dim=1)]  # noqa: E731
        self.qkv, self.dqkv = heads(self.x), heads(self.dx)

    def fill(self, seed):
        g = torch.Generator().manual_seed(1000 + seed)
        self.ids.copy_(torch.randint(-1, self.vocab + 1, (self.T,), generator=g))
        ends = torch.randint(0, self.T + 1, (self.docs + 1,), generator=g).sort().values
        self.offsets.copy_(ends.int())
        self.do.copy_(torch.randn(self.do.shape, generator=g).to(BF))

    def run(self):
        B.acx_embed_fwd(self.table, self.ids, self.E, self.x)
        B.acx_attn_plan(self.attn, self.offsets, self.plan)
        B.acx_attn_fwd(self.attn, *self.qkv, self.plan, self.o, self.lse)
        B.acx_attn_bwd(self.attn, *self.qkv, self.plan, self.o, self.do, self.lse, *self.dqkv, ws=self.scratch[0])
        B.acx_embed_bwd(self.table, self.ids, self.dx, self.dE, ws=self.scratch[1])
        B.acx_grad_clip(self.list, 0.5, self.total, ws=self.scratch[2])

    def results(self):
        return [t.clone() for t in (self.x, self.o, self.lse, self.dx, self.dE, self.total)]

    def eager(self, seed):
        self.fill(seed)
        self.run()
        return self.results()

    def capture(self):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.run()
        return graph


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_same_bits_and_captured_with_other_batches():
    b = Batch()
    want = [b.eager(seed) for seed in range(3)]
    assert same(b.eager(0), want[0])
    graph = b.capture()
    for seed in (2, 0, 1, 1):
        b.fill(seed)
        for t in (b.x, b.o, b.lse, b.dx, b.dE, b.total):
            t.fill_(NAN)
        graph.replay()
        assert same(b.results(), want[seed]), seed
    assert B.acx_last_device_status() == B.ACX_OK


@gpu
def test_two_graphs_that_share_scratch():
    a = Batch()
    b = Batch(seed=5, scratch=a.scratch)
    want_a, want_b = a.eager(3), b.eager(4)
    ga, gb = a.capture(), b.capture()
    for _ in range(3):
        ga.replay()
        gb.replay()
    assert same(a.results(), want_a) and same(b.results(), want_b)


@gpu
def test_two_steps_at_once():
    a, b = Batch(T=1500, docs=3), Batch(T=900, H=6, K=1, d=72, seed=7)
    want_a, want_b = a.eager(1), b.eager(2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                x.run()
    torch.cuda.synchronize()
    assert same(a.results(), want_a) and same(b.results(), want_b)
    assert B.acx_last_device_status() == B.ACX_OK


# --------------------------------------------------------------------------------------------------------- attention
def inputs(T, H, K, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, h, d, generator=g).to(BF).cuda() for h in (H, K, K, H)]


def run(desc, offsets, q, k, v, do, prefix=None, plan=None):
    if plan is None:
        plan = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN)
        B.acx_attn_plan(desc, offsets, plan, prefix=prefix)
    o, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, device="cuda")
    B.acx_attn_fwd(desc, q, k, v, plan, o, lse)
    g = [torch.full_like(t, NAN) for t in (q, k, v)]
    B.acx_attn_bwd(desc, q, k, v, plan, o, do, lse, *g, ws=B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD))
    return [o, lse.T.contiguous(), *g]


@gpu
@pytest.mark.parametrize("bad", [NAN, float("inf"), 3e38])
@pytest.mark.parametrize("d,causal", [(64, True), (128, False)])
def test_nothing_of_a_document_reaches_another(d, causal, bad):
    T, desc = 500, B.make_attn_desc(500, 4, 2, d, 3, causal=causal)
    x = inputs(T, 4, 2, d)
    offsets = offsets_of(150, 331, 480)
    want = run(desc, offsets, *x)
    for t in x:
        t[150:331] = bad
        t[480:] = bad
    got = run(desc, offsets, *x)
    for a, b in zip(got, want):
        assert torch.equal(a[:150], b[:150]) and torch.equal(a[331:480], b[331:480])
        assert torch.equal(a[480:], b[480:])
    assert B.acx_last_device_status() == B.ACX_OK


@gpu
def test_infinite_keys_that_the_mask_hides():
    """Scores that the mask takes out may be anything, and those of minus the largest number are weights of zero.  A value that is not a
    number, times such a weight, is none (as in the plain form): it ends at the tile of 128 tokens that it is in."""
    T, d = 300, 64
    desc, offsets = B.make_attn_desc(T, 2, 1, d), offsets_of(T)
    q, k, v, do = inputs(T, 2, 1, d)
    want = run(desc, offsets, q, k, v, do)
    k[200:], v[200:] = float("inf"), NAN
    got = run(desc, offsets, q, k, v, do)
    assert torch.equal(got[0][:128], want[0][:128]) and torch.equal(got[1][:200], want[1][:200])
    v = inputs(T, 2, 1, d)[2]
    got = run(desc, offsets, q, k, v, do)
    assert torch.equal(got[0][:200], want[0][:200]) and torch.equal(got[1][:200], want[1][:200])
    q, k, v, do = inputs(T, 2, 1, d)
    q[:], k[:100] = 1.0, -1e30
    o = run(desc, offsets, q, k, v, do)[0]
    w = torch.softmax((q.double()[:, 0] @ k.double()[:, 0].T * d ** -0.5).masked_fill(torch.triu(torch.ones(T, T, device="cuda"), 1).bool(), -1e300), -1)
    assert torch.isfinite(o).all()
    # p rounded once and o once: 2^-8 of sum p |v| and of o
    assert ((o[:, 0].double() - w @ v.double()[:, 0]).abs() <= 2.0 ** -8 * 2.1 * (w @ v.double()[:, 0].abs()) + 1e-6).all()


@gpu
def test_a_query_with_one_key_has_no_gradient_through_its_scores():
    T, d = 260, 64
    q, k, v, do = inputs(T, 2, 2, d)
    desc, offsets = B.make_attn_desc(T, 2, 2, d, 130), offsets_of(*range(2, 262, 2))      # documents of two tokens
    o, lse, dq, dk, dv = run(desc, offsets, q, k, v, do)
    assert not dq[::2].any() and torch.equal(o[::2], v[::2])
    desc = B.make_attn_desc(T, 2, 2, d, T)
    o, lse, dq, dk, dv = run(desc, offsets_of(*range(1, T + 1)), q, k, v, do)             # of one
    assert not dq.any() and not dk.any() and torch.equal(o, v) and torch.equal(dv, do)


@gpu
@pytest.mark.parametrize("ends", [(300, 100, 250, 120), (-5, 90, 1 << 30, 7), (-(1 << 31), (1 << 31) - 1, 0, (1 << 31) - 1), (999, 999, 999, 999)])
def test_offsets_that_are_wrong_reach_nothing_outside(ends):
    """Documents may not decrease or leave the batch; what is computed then is open, but only there, and the next call is right."""
    T, room = 400, 64
    desc = B.make_attn_desc(T, 4, 2, 64, 4)
    q, k, v, do = inputs(T, 4, 2, 64)
    wide = [torch.full((T + 2 * room, *t.shape[1:]), 7.0, dtype=BF, device="cuda") for t in (q, q, k, v)]
    o, dq, dk, dv = (w[room:room + T] for w in wide)
    lse = torch.full((4 * T + 2 * room,), 7.0, device="cuda")
    plan, ws = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN), B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD)
    B.acx_attn_plan(desc, offsets_of(*ends), plan, prefix=torch.tensor([5, -3, 1 << 30, 1], dtype=torch.int32, device="cuda"))
    B.acx_attn_fwd(desc, q, k, v, plan, o, lse[room:-room].view(4, T))
    B.acx_attn_bwd(desc, q, k, v, plan, o, do, lse[room:-room].view(4, T), dq, dk, dv, ws=ws)
    assert B.acx_last_device_status() == B.ACX_OK
    for w in (*wide, lse):
        assert (w[:room] == 7).all() and (w[-room:] == 7).all()
    good = offsets_of(100, 100, 333, T)
    a = run(desc, good, q, k, v, do)
    assert all(torch.isfinite(t).all() for t in a)


@gpu
def test_a_plan_of_another_batch_is_refused():
    q, k, v, do = inputs(300, 2, 1, 64)
    desc = B.make_attn_desc(300, 2, 1, 64, 2)
    other = B.make_attn_desc(900, 2, 1, 64, 2)
    plan = B.alloc_attn_workspace(other, B.ACX_OP_ATTN_PLAN)
    for make in (lambda: plan.zero_(), lambda: B.acx_attn_plan(other, offsets_of(400, 900), plan),
                 lambda: B.acx_attn_plan(B.make_attn_desc(300, 2, 1, 64, 2, causal=False), offsets_of(100, 300), plan),
                 lambda: B.acx_attn_plan(B.make_attn_desc(300, 2, 1, 64, 1), offsets_of(300), plan)):
        make()
        assert B.acx_last_device_status() == B.ACX_OK
        got = run(desc, None, q, k, v, do, plan=plan)
        assert B.acx_last_device_status() == B.ACX_ERR_INVALID_ARG
        assert all(torch.isnan(t).all() for t in got)
    B.acx_attn_plan(desc, offsets_of(100, 300), plan)
    assert all(torch.isfinite(t).all() for t in run(desc, None, q, k, v, do, plan=plan))
    assert B.acx_last_device_status() == B.ACX_OK


@gpu
def test_no_tokens_no_lse_and_no_neighbour_columns():
    empty = [t[:0] for t in inputs(1, 2, 1, 64)]
    run(B.make_attn_desc(0, 2, 1, 64), offsets_of(0), *empty[:3], empty[3])
    T = 200
    q, k, v, do = inputs(T, 3, 1, 40)
    desc, offsets = B.make_attn_desc(T, 3, 1, 40), offsets_of(T)
    want = run(desc, offsets, q, k, v, do)
    # every matrix a slice of a wider one, at an address that 16 divides and 32 does not
    def within(t):
        w = torch.full((T, t.shape[1] * 40 + 24), 7.0, dtype=BF, device="cuda")
        w[:, 8:-16] = t.flatten(1)
        return w, w[:, 8:-16].unflatten(1, (-1, 40))
    wide, views = zip(*(within(t) for t in (q, k, v, do, q, q, k, v)))
    plan = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN)
    B.acx_attn_plan(desc, offsets, plan)
    q2, k2, v2, do2, o2, dq2, dk2, dv2 = views
    B.acx_attn_fwd(desc, q2, k2, v2, plan, o2)
    assert torch.equal(o2, want[0])
    lse = torch.empty(3, T, device="cuda")
    B.acx_attn_fwd(desc, q2, k2, v2, plan, o2, lse)
    B.acx_attn_bwd(desc, q2, k2, v2, plan, o2, do2, lse, dq2, dk2, dv2, ws=B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD))
    assert all(torch.equal(a, b) for a, b in zip((dq2, dk2, dv2), want[2:]))
    assert all((w[:, :8] == 7).all() and (w[:, -16:] == 7).all() for w in wide)


@gpu
def test_on_a_stream_of_its_own():
    T, desc = 600, B.make_attn_desc(600, 2, 1, 128, 2)
    x, offsets = inputs(T, 2, 1, 128), offsets_of(100, 600)
    want = run(desc, offsets, *x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    plan, ws = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN), B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD)
    q, k, v, do = x
    o, lse, g = torch.empty_like(q), torch.empty(2, T, device="cuda"), [torch.empty_like(t) for t in (q, k, v)]
    side.wait_stream(torch.cuda.current_stream())
    B.acx_attn_plan(desc, offsets, plan, stream=side)
    B.acx_attn_fwd(desc, q, k, v, plan, o, lse, stream=side)
    B.acx_attn_bwd(desc, q, k, v, plan, o, do, lse, *g, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(o, want[0]) and all(torch.equal(a, b) for a, b in zip(g, want[2:]))


# --------------------------------------------------------------------------------------------------- beyond 32 bits
@gpu
def test_attention_in_a_matrix_of_more_than_2_31_elements():
    T, ld, docs = 70_000, 32_768, 280
    x = torch.zeros(T, ld, dtype=BF, device="cuda")
    out = torch.full((T, ld), 7.0, dtype=BF, device="cuda")
    cols = [slice(ld - 40, ld - 24), slice(0, 8), slice(ld - 8, ld), slice(1024, 1040)]     # q, k, v, dO
    q, k, v, do = inputs(T, 2, 1, 8)
    views = []
    for c, t in zip(cols, (q, k, v, do)):
        x[:, c] = t.flatten(1)
        views.append(x[:, c].unflatten(1, (-1, 8)))
    ends = [T * (i + 1) // docs for i in range(docs)]
    desc = B.make_attn_desc(T, 2, 1, 8, docs)
    plan = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN)
    B.acx_attn_plan(desc, offsets_of(*ends), plan)
    o, dq, dk, dv = (out[:, c].unflatten(1, (-1, 8)) for c in (slice(ld - 16, ld), slice(64, 80), slice(0, 8), slice(ld - 64, ld - 56)))
    lse = torch.empty(2, T, device="cuda")
    B.acx_attn_fwd(desc, *views[:3], plan, o, lse)
    B.acx_attn_bwd(desc, *views[:3], plan, o, views[3], lse, dq, dk, dv, ws=B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD))
    assert B.acx_last_device_status() == B.ACX_OK
    n0 = ends[-11]          # the last ten documents, whose rows lie behind 2^31 elements
    cpu = lambda t: t[n0:].double().cpu().numpy()  # noqa: E731
    want = oa.attention(*(cpu(t) for t in (q, k, v)), [0, *(e - n0 for e in ends[-10:])], do=cpu(do))
    for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert (np.abs(cpu(t) - want[name]) <= want[name + "_bound"] + 2.0 ** -22 * (1 + np.abs(want[name]).max())).all(), name
    assert (out[:, 100:ld - 100] == 7).all()


@gpu
def test_a_table_of_more_than_2_31_elements():
    vocab, d, T = 40_000, 65_536, 40
    E = torch.zeros(vocab, d, dtype=BF, device="cuda")
    ids = torch.tensor([vocab - 1, 0, vocab - 1, vocab // 2, vocab - 2] * 8, device="cuda")
    E[ids] = torch.randn(T, d, device="cuda").to(BF)
    desc = B.make_embed_desc(T, d, vocab, BF)
    Y = torch.empty(T, d, dtype=BF, device="cuda")
    B.acx_embed_fwd(desc, ids, E, Y)
    assert torch.equal(Y, E[ids])
    E.fill_(7.0)
    g = torch.randint(-4, 5, (T, d), device="cuda").to(BF)      # sums without a rounding
    B.acx_embed_bwd(desc, ids, g, E, ws=B.alloc_embed_workspace(desc, B.ACX_OP_EMBED_BWD))
    for w in (vocab - 1, 0, vocab // 2, vocab - 2):
        assert torch.equal(E[w], g[ids == w].float().sum(0).to(BF))
        E[w] = 0
    assert not E.any()


@gpu
def test_clipping_a_tensor_of_more_than_2_31_elements():
    n = (1 << 31) + 12_345
    x = torch.ones(n, dtype=BF, device="cuda")
    lst = B.make_grad_list([x])
    total = torch.empty(2, device="cuda")
    B.acx_grad_clip(lst, 0.25 * n ** 0.5, total, ws=B.alloc_grad_workspace(lst))
    assert abs(float(total[0]) - n ** 0.5) <= 2.0 ** -23 * n ** 0.5 and abs(float(total[1]) - 0.25) <= 2.0 ** -24
    assert (x == 0.25).all()
