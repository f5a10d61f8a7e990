"""Attention, clipping and the training step where numbers end: scores of minus infinity and far beyond 2^24, saturated caps, values that
are none where the mask hides them, short documents in long batches, steps whose norm is no number."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import mlp_lm as M
from test_gpu_step import reference, rel

pytestmark = pytest.mark.gpu
BF, NAN, INF = torch.bfloat16, float("nan"), float("inf")


def offsets_of(*ends):
    return torch.tensor([0, *ends], dtype=torch.int32, device="cuda")


def inputs(T, H, K, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, h, d, generator=g).to(BF).cuda() for h in (H, K, K, H)]


def run(desc, offsets, q, k, v, do, prefix=None, slopes=None):
    """o, lse (tokens first), dq, dk, dv; outputs start as NaN."""
    plan = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN)
    B.acx_attn_plan(desc, offsets, plan, prefix=prefix)
    o, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, device="cuda")
    B.acx_attn_fwd(desc, q, k, v, plan, o, lse, slopes=slopes)
    g = [torch.full_like(t, NAN) for t in (q, k, v)]
    B.acx_attn_bwd(desc, q, k, v, plan, o, do, lse, *g, slopes=slopes, ws=B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_BWD))
    assert B.acx_last_device_status() == B.ACX_OK
    return [o, lse.T.contiguous(), *g]


# ------------------------------------------------------------------------------------------ scores at the ends of the range
@pytest.mark.parametrize("T,hidden", [(300, (100, 300)), (300, (128, 256)), (1000, (0, 990)), (700, (384, 700))])
@pytest.mark.parametrize("d,slopes", [(64, False), (128, False), (64, True)])
def test_keys_whose_scores_are_minus_infinity_have_no_weight(T, hidden, d, slopes):
    """A mask written into a channel: the lowest bfloat16 times a query's 2 is beyond fp32.  Whole tiles of keys are such, the first that
    is taken among them; what is left has the weights, the gradients and the sums it has without them."""
    H, (n0, n1) = 2, hidden
    q, k, v, do = inputs(T, H, 1, d)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[n0:n1] = False
    q[:, :, 0] = 2.0
    k[:, :, 0] = torch.where(keep, 0.0, torch.finfo(BF).min)[:, None].to(BF)
    slope = torch.tensor([0.25, 0.01], device="cuda") if slopes else None
    o, lse, dq, dk, dv = run(B.make_attn_desc(T, H, 1, d, causal=False), offsets_of(T), q, k, v, do, slopes=slope)
    assert all(torch.isfinite(t).all() for t in (o, lse, dq, dk, dv))
    assert not dk[~keep].any() and not dv[~keep].any()
    pos = torch.arange(T, device="cuda").double()
    for h in range(H):
        Q, K, V, G = q[:, h].double(), k[keep, 0].double(), v[keep, 0].double(), do[:, h].double()
        z = Q @ K.T * d ** -0.5
        if slopes:
            z = z - slope[h].double() * (pos[:, None] - pos[keep][None, :]).abs()
        p = torch.softmax(z, 1)
        # p rounded once and o once: 2^-8 of sum p |v| and of o; fp32 in between
        assert ((o[:, h].double() - p @ V).abs() <= 2.0 ** -8 * 2.1 * (p @ V.abs()) + 1e-5).all()
        assert ((lse[:, h].double() - torch.logsumexp(z, 1)).abs() <= 1e-4).all()
        ds = p * (G @ V.T - ((G @ V.T) * p).sum(1, keepdim=True)) * d ** -0.5
        # dS once, the output once, and delta off by what rounding o leaves of it: 2^-8 |dO| |o| of every p
        lost = 2.0 ** -8 * 2 * (G.abs() * (p @ V.abs())).sum(1, keepdim=True)
        err = 2.0 ** -8 * 1.1 * ds.abs() + p * lost * d ** -0.5
        assert ((dq[:, h].double() - ds @ K).abs() <= 2.0 ** -8 * (ds @ K).abs() + err @ K.abs() + 1e-5).all()


@pytest.mark.parametrize("size", [1e5, 1e8, 1e30])
@pytest.mark.parametrize("d,cap,slopes,causal", [(64, 0.0, False, True), (128, 0.0, False, False), (64, 0.0, True, True), (64, 1e31, False, True)])
def test_gradients_beside_scores_that_fp32_cannot_tell_apart(size, d, cap, slopes, causal):
    """Queries whose scores are far beyond 2^24 have probabilities of no use in the backward pass, but of no more than 1: all gradients
    are numbers, and where such queries have no gradient of their own, those of the keys are what the other queries make of them."""
    T, H, n = 300, 2, 100
    desc, offsets = B.make_attn_desc(T, H, 1, d, causal=causal, softcap=cap), offsets_of(T)
    slope = torch.tensor([0.25, 0.01], device="cuda") if slopes else None
    q, k, v, do = inputs(T, H, 1, d)
    want = run(desc, offsets, q, k, v, torch.cat([torch.zeros_like(do[:n]), do[n:]]), slopes=slope)
    g = torch.Generator().manual_seed(9)
    q[:n] = (size * torch.randn(n, H, d, generator=g)).to(BF).cuda()
    got = run(desc, offsets, q, k, v, do, slopes=slope)
    assert all(torch.isfinite(t).all() for t in got)
    do[:n] = 0
    got = run(desc, offsets, q, k, v, do, slopes=slope)
    assert all(torch.isfinite(t).all() for t in got) and not got[2][:n].any()
    # the same sums: products of zero beside them
    for a, b in zip(got[2:], want[2:]):
        assert torch.equal(a[n:] if a is got[2] else a, b[n:] if b is want[2] else b)


def test_keys_of_minus_1e30_have_finite_gradients():
    T, H, d, n = 300, 2, 64, 100
    desc, offsets = B.make_attn_desc(T, H, 1, d), offsets_of(T)
    q, k, v, do = inputs(T, H, 1, d)
    q[:], k[:n] = 1.0, -1e30
    o, lse, dq, dk, dv = run(desc, offsets, q, k, v, do)
    assert all(torch.isfinite(t).all() for t in (o, lse, dq, dk, dv))
    do[:n] = 0                       # the queries that see nothing else
    o, lse, dq, dk, dv = run(desc, offsets, q, k, v, do)
    assert all(torch.isfinite(t).all() for t in (o, lse, dq, dk, dv))
    assert not dq[:n].any() and not dk[:n].any() and not dv[:n].any()


# ------------------------------------------------------------------------------------------------------- saturated caps
@pytest.mark.parametrize("d,alibi,causal", [(64, False, False), (128, False, True), (64, True, True)])
@pytest.mark.parametrize("T", [200, 700])
def test_gradients_through_a_saturated_cap(d, alibi, causal, T):
    """Scores of 6.5 to 9.5 times the cap, either way: the cap's slope is 4 e^-2|u|, 1e-5 to 2e-8, and the gradients have its digits."""
    H, cap, g = 2, 10.0, torch.Generator().manual_seed(T)
    u = (6.5 + 3 * torch.rand(T, 1, 1, generator=g)) * torch.where(torch.rand(T, 1, 1, generator=g) < 0.5, 1.0, -1.0)
    rnd = lambda h: torch.randn(T, h, d, generator=g)  # noqa: E731
    q, k = (1 + 0.1 * rnd(H)).to(BF).cuda(), (cap * u * d ** -0.5 * (1 + 0.1 * rnd(1))).to(BF).cuda()
    v, do = rnd(1).to(BF).cuda(), rnd(H).to(BF).cuda()
    slopes = torch.tensor([0.05, 0.01], device="cuda") if alibi else None
    got = dict(zip(("o", "lse", "dq", "dk", "dv"), run(B.make_attn_desc(T, H, 1, d, causal=causal, softcap=cap), offsets_of(T), q, k, v, do, slopes=slopes)))
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    # the slope's own error: half a step of fp16, 2^-11, and as much for fp32 scores, exponential and reciprocal (a score of 95 in
    # fp32 sums is off by 2^-21 of that, twice as much over the cap in the slope: 2^-16.7); absolutely half a step of fp16 below its range, 2^-39
    want = oa.attention(n(q), n(k), n(v), [0, T], causal=causal, softcap=cap, slopes=None if slopes is None else n(slopes), do=n(do),
                        slope_error=(2.0 ** -10, 2.0 ** -39))
    for name in ("o", "dq", "dk", "dv"):
        off = np.abs(n(got[name]) - want[name]) - want[name + "_bound"]
        assert off.max() <= 2.0 ** -22 * np.abs(want[name]).max(), (name, off.max(), np.abs(want[name]).max())
        assert np.median(want[name + "_bound"]) <= 0.1 * np.abs(want[name]).max(), name      # a bound that says something


# ----------------------------------------------------------------------------------- how far what is not a number reaches
def test_values_that_are_no_numbers_reach_the_tiles_that_take_them():
    """Tiles of 128 tokens count from the document's start.  A query takes those up to the prefix's end or its own, whichever is later; a
    key takes queries from its own tile on, or from the document's start if its tile begins inside the prefix."""
    T, H, d, s = 700, 2, 64, 37
    end = s + 600
    x = inputs(T, H, 1, d)
    desc = B.make_attn_desc(T, H, 1, d, 2)
    for prefix, bad in ((0, s + 132), (130, s + 260)):
        args, kw = (desc, offsets_of(s, end)), dict(prefix=torch.tensor([0, prefix], dtype=torch.int32, device="cuda"))
        want = run(*args, *x, **kw)
        tile = s + (bad - s) // 128 * 128            # queries before this one take no tile with the bad key
        for i in (1, 2):
            y = [t.clone() for t in x]
            y[i][bad] = NAN
            got = run(*args, *y, **kw)
            for a, b in zip(got[:3], want):
                assert torch.equal(a[:tile], b[:tile]), (prefix, i)
            assert torch.equal(got[3][:s], want[3][:s]) and torch.equal(got[3][end:], want[3][end:])
        later = s + 256                              # tiles of keys that begin behind the bad query's and behind the prefix
        for i in (0, 3):
            y = [t.clone() for t in x]
            y[i][s + 140] = INF
            got = run(*args, *y, **kw)
            assert torch.equal(got[3][later:], want[3][later:]) and torch.equal(got[4][later:], want[4][later:]), (prefix, i)
    # what the text says of a prefix: a query takes the whole tile that the prefix ends in
    y = [t.clone() for t in x]
    y[2][s + 250] = NAN
    o = run(*args, *y, **kw)[0]
    assert torch.isnan(o[s:end]).all()


# ------------------------------------------------------------------------------------------- short documents, long batches
def test_dk_of_a_document_does_not_depend_on_the_batch():
    """One query head per key head (no parts to join): the same bits in a batch of 500 tokens, of 513 and of 4000."""
    d, H, n = 64, 2, 100
    x = inputs(4000, H, H, d)
    want = None
    for T in (500, 513, 4000):
        y = [t[:T].contiguous() for t in x]
        ends = list(range(n, T, n)) + [T]
        got = run(B.make_attn_desc(T, H, H, d, len(ends)), offsets_of(*ends), *y)
        got = [t[:5 * n - n] for t in got]
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(got, want)), T


@pytest.mark.parametrize("T,docs", [(4096, 64), (2000, 5)])
def test_dk_of_short_documents_is_rounded_once(T, docs):
    """dS of a document of up to 512 tokens enters dK in two parts: what is left is dK's own rounding.  That is off by up to half a step,
    uniformly: 2^-9 to 2^-8 / sqrt(3) of a value, 0.00166 over all sizes of a mantissa; with dS rounded too it is 0.0024."""
    H, d = 2, 64
    q, k, v, do = inputs(T, H, 1, d)
    ends = [T * (i + 1) // docs for i in range(docs)]
    got = run(B.make_attn_desc(T, H, 1, d, docs), offsets_of(*ends), q, k, v, do)[3].double().cpu().numpy()
    want = oa.attention(*(t.double().cpu().numpy() for t in (q, k, v)), [0, *ends], do=do.double().cpu().numpy())["dk"]
    assert np.linalg.norm(got - want) <= 0.0020 * np.linalg.norm(want)


# --------------------------------------------------------------------------------------------------------------- status
def test_a_refused_plan_does_not_hide_a_wait_that_ran_out():
    q, k, v, do = inputs(300, 2, 1, 64)
    desc = B.make_attn_desc(300, 2, 1, 64, 2)
    plan = B.alloc_attn_workspace(desc, B.ACX_OP_ATTN_PLAN)
    o = torch.empty_like(q)
    refused = lambda: B.acx_attn_fwd(desc, q, k, v, plan.zero_(), o)  # noqa: E731
    assert B.acx_last_device_status() == B.ACX_OK
    for calls in ((refused, 0), (0, refused), (refused, 0, refused)):
        for call in calls:
            call() if call else B.acx_debug_expired_wait(1_000_000)      # 1 ms on a barrier nobody signals
        assert B.acx_last_device_status() == B.ACX_ERR_TIMEOUT
        assert B.acx_last_device_status() == B.ACX_OK
    refused()
    assert B.acx_last_device_status() == B.ACX_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------------ the training step
def test_step_against_autograd_with_the_weight_of_the_factors():
    """The whole step, its gradients and what its clipping bounds; tolerances as for the step in test_gpu_step.py."""
    s = M.Sizes(tokens=333, d=136, inter=264, vocab=1003, layers=2, r=32, alpha=0.8, max_norm=0.25, heads=6, kv_heads=2, head_dim=24, docs=4, tied=True)
    model = M.MlpLm(s)
    ids, y = M.synthetic_batch(s)
    offsets = offsets_of(1, 130, 130, 300)      # one token, 129, none, 170; the last 33 tokens are padding
    total = model.forward(ids, y, offsets=offsets)
    dh0 = model.backward()
    assert B.acx_last_device_status() == B.ACX_OK
    loss, p = reference(model, ids, y, offsets)
    norm, f = model.norm.double().tolist()
    assert abs(float(total[0] / total[1]) - float(loss.detach())) <= 1e-2 * float(loss.detach())
    tol = 6e-2
    assert rel(dh0, p["h0"].grad) <= tol
    assert 0 < f < 1 and abs(norm * f - s.max_norm) <= 1e-6 * s.max_norm
    assert rel(model.grads["head"][0] / f, p["head"].grad) <= tol
    for k in ("w_pre", "w_post", "gate"):
        for a, b in zip(model.grads[k], p[k]):
            assert rel(a / f, b.grad) <= tol, k
    # the norm is that of what was clipped, a factor counted as A S^T is on average: every bf16 element off by 2^-8 at most, of its own size
    square = lambda t: float(t.double().square().sum())  # noqa: E731
    clipped = sum(square(t) for ts in model.grads.values() for t in ts)
    clipped += sum((model.w[l][k].shape[1] + s.r + 1) / s.r * square(a) for l in range(s.layers) for k, a in model.factors[l].items())
    assert abs(clipped ** 0.5 - s.max_norm) <= 2.0 ** -8 * s.max_norm
    # |A|^2 is |dW|^2 on average.  One sketch: a standard deviation of sqrt(2 / r) = 25 % at most (dW of rank one), three of them.
    for l, lw in enumerate(p["w"]):
        for k, w in lw.items():
            got = square(model.factors[l][k].double() / f) / square(w.grad)
            assert 0.25 < got < 1.75, (l, k, got)


SIZES = dict(tokens=256, d=128, inter=256, vocab=301, layers=2, r=32, heads=4, kv_heads=1, head_dim=32, docs=3, tied=True)


def test_a_step_whose_norm_is_no_number_is_left_out():
    s = M.Sizes(max_norm=1.0, **SIZES)
    model = M.MlpLm(s)
    ids, y = M.synthetic_batch(s)
    keep = lambda: [t.clone() for l in range(s.layers) for k in model.w[l] for t in (model.w[l][k], model.master[l][k], *model.moments[l][k])]  # noqa: E731
    before, good = keep(), float(model.head[0, 0])
    model.head[ids[0], 0] = INF
    model.forward(ids, y)
    model.backward(lr=1e-3)
    assert not np.isfinite(float(model.norm[0])) and float(model.norm[1]) == 1.0
    assert model.step_no == 0 and all(torch.equal(a, b) for a, b in zip(keep(), before))
    model.head[ids[0], 0] = good
    model.forward(ids, y)
    model.backward(lr=1e-3)
    assert model.step_no == 1 and all(torch.isfinite(t).all() for t in keep())
    assert not any(torch.equal(a, b) for a, b in zip(keep(), before))


def test_a_clipped_step_can_be_captured():
    s = M.Sizes(max_norm=1.0, **SIZES)
    model = M.MlpLm(s)
    ids, y = M.synthetic_batch(s)

    def step():
        model.forward(ids, y)
        model.backward(lr=1e-3)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    state = [t for lw, mw, mo in zip(model.w, model.master, model.moments) for k in lw for t in (lw[k], mw[k], *mo[k])]
    keep = [t.clone() for t in state]
    step()
    want = [t.clone() for t in state]
    for t, k in zip(state, keep):
        t.copy_(k)
    model.step_no = 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(state, want))
    assert B.acx_last_device_status() == B.ACX_OK


@pytest.mark.parametrize("scale,cap,size", [(2.0 ** 104, 0.0, 2.0 ** -104), (0.125, 2.0 ** 104, 1.0), (1.0, 2.0 ** -104, 1.0)])
def test_scales_and_caps_at_their_limits(scale, cap, size):
    """The largest scale on queries as small (so that scores are ordinary ones), a cap that does nothing, one that leaves no score: the
    results are those of ordinary scales, and of a mean."""
    T, H, d = 200, 2, 64
    q, k, v, do = inputs(T, H, 1, d)
    offsets = offsets_of(T)
    got = run(B.make_attn_desc(T, H, 1, d, scale=scale, softcap=cap), offsets, q * size, k, v, do)
    assert all(torch.isfinite(t).all() for t in got)
    want = run(B.make_attn_desc(T, H, 1, d, scale=scale * size), offsets, torch.zeros_like(q) if cap == 2.0 ** -104 else q, k, v, do)
    # a rounding more or less of the scores (2^-24 of some tens) turns a bf16 result over: one step, 2^-7, of few
    for a, b in zip(got[:2], want[:2]):
        assert ((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-4).all()


def test_a_list_made_on_another_stream_waits_for_the_memory_it_gets():
    """The plan's memory comes from the current stream, where a kernel may still have to write what was there before."""
    grads = [torch.ones(n, device="cuda") for n in (100, 70_000, 5)]
    want = B.make_grad_list(grads).plan.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        old = torch.empty(want.numel(), dtype=torch.uint8, device="cuda")
        torch.cuda._sleep(20_000_000)                # some 10 ms of nothing, then the write
        old.fill_(255)
        del old
        lst = B.make_grad_list(grads, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(lst.plan, want)           # (before any call reads it)
        del lst
