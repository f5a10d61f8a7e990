"""GPU parity of the vocabulary cross entropy against the oracle in 64 bits: odd vocabularies and token counts, several
pieces, split sums, tokens that are not trained on, weights, extreme logits, empty inputs, streams and graphs."""
import numpy as np
import pytest
import torch

from oracle import cross_entropy as C
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import inputs as I

from _harness import TOL_DERIVED, raw_bits, to_device, to_host

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Head:
    """Device buffers of one call, full of NaN canaries."""

    def __init__(self, X, W, y, weight=None, logit_scale=1.0):
        (self.t, self.d), self.v = X.shape, W.shape[0]
        self.desc = B.make_ce_desc(self.t, self.d, self.v, logit_scale)
        self.X, self.W, self.y = to_device(X, "bf16"), to_device(W, "bf16"), torch.from_numpy(y.astype(np.int64)).cuda()
        self.w = None if weight is None else to_device(weight, "f32")
        full = lambda *s, dt=torch.float32: torch.full(s, NAN, dtype=dt, device="cuda")  # noqa: E731
        self.loss, self.lse, self.total = full(self.t), full(self.t), full(2)
        self.dX, self.dW = full(self.t, self.d, dt=torch.bfloat16), full(self.v, self.d, dt=torch.bfloat16)
        self.ws = B.alloc_ce_workspace(self.desc, B.ACX_OP_CE_BWD)
        self.ws.view(torch.uint8).fill_(255)      # NaN everywhere

    def fwd(self, stream=None):
        B.acx_linear_ce_fwd(self.desc, self.X, self.W, self.y, self.loss, self.lse, self.total, self.w, self.ws, stream=stream)

    def bwd(self, stream=None, scale=1.0, dx=True, dw=True):
        B.acx_linear_ce_bwd(self.desc, self.X, self.W, self.y, self.lse, self.dX if dx else None, self.dW if dw else None, weight=self.w,
                            denom=self.total[1:], scale=scale, ws=self.ws, stream=stream)

    def check(self):
        assert B.acx_last_device_status() == B.ACX_OK


def make(t, d, v, seed, weighted=False, boost=8.0):
    g = np.random.Generator(np.random.Philox(seed))
    W = I.gaussian((v, d), seed + 1, d ** -0.5, "bf16")
    y = (g.random(t) ** 3 * v).astype(np.int64)
    X = I.round_to_dtype(I.gaussian((t, d), seed + 2) + boost * g.random((t, 1)).astype(np.float32) * W[y], "bf16")
    y[np.arange(t) % 5 == 1] = -100
    y[t // 2] = v - 1
    return X, W, y, (g.random(t) * 2).astype(np.float32) if weighted else None


def logit_error(X, W, scale, lse):
    """Bound on a row's logits: the tensor core adds 16 products at a time, each sum off by at most 2^-23 of the magnitudes
    summed; and 2^-21 of the result's own size for exponentials, logarithm and their sums."""
    d = X.shape[1]
    mag = abs(scale) * (np.abs(X).astype(np.float64) @ np.abs(W).astype(np.float64).T).max(1)
    return 2.0 ** -23 * (d / 16 + 8) * mag + 2.0 ** -21 * (1 + np.abs(lse))


# a word, a partly filled tile, odd everything, several token tiles, a d of several tiles, split sums; up to 64 tokens (exchanged
# operands) and just above; the last three in pieces, with few tokens, with and without what is put back into dW
SHAPES = [(1, 64, 1000), (7, 8, 1), (5, 72, 37), (130, 136, 257), (300, 904, 3203), (1000, 264, 20000), (257, 2056, 1111), (700, 520, 513),
          (64, 1024, 50001), (33, 264, 5000), (65, 264, 5000), (513, 136, 777),
          (64, 8, 1100001),
          (500, 64, 140001), (4096, 72, 17001)]


@pytest.mark.parametrize("t,d,v", SHAPES)
@pytest.mark.parametrize("weighted,logit_scale", [(False, 1.0), (True, 0.5)])
def test_against_the_oracle(t, d, v, weighted, logit_scale):
    X, W, y, w = make(t, d, v, t + d + v, weighted)
    h = Head(X, W, y, w, logit_scale)
    h.fwd()
    h.bwd(scale=3.0)
    h.check()
    loss, lse, total = C.ce_fwd(X, W, y, w, logit_scale)
    e = logit_error(X, W, logit_scale, lse)
    assert np.all(np.abs(to_host(h.lse) - lse) <= e)
    assert np.all(np.abs(to_host(h.loss) - loss) <= 2 * e)
    wt = np.where((y >= 0) & (y < v), 1.0 if w is None else w, 0.0)
    assert abs(to_host(h.total)[0] - total[0]) <= np.sum(wt * 2 * e) + 2.0 ** -20 * np.sum(wt * loss)
    assert abs(to_host(h.total)[1] - total[1]) <= 2.0 ** -20 * total[1]
    dX, dW = C.ce_bwd(X, W, y, w, logit_scale, total[1], 3.0)
    # D is rounded to bfloat16 once (half a unit: 2^-8 of it), its probabilities are off by the logits' error; then sums over
    # the vocabulary or the tokens on the tensor core, and one rounding of the result
    D = np.abs(C.ce_dlogits(X, W, y, w, logit_scale))
    f = 3.0 * abs(logit_scale) / total[1]
    per_d = 2.0 ** -8 * D + 4 * e[:, None] * np.minimum(D + wt[:, None], D * 4 + 1e-30)
    for name, got, want, mag in (("dX", h.dX, dX, f * ((per_d + 2.0 ** -23 * (v / 16 + 40) * D) @ np.abs(W.astype(np.float64)))),
                                 ("dW", h.dW, dW, f * ((per_d + 2.0 ** -23 * (t / 16 + 40) * D).T @ np.abs(X.astype(np.float64))))):
        got = to_host(got)
        assert np.all(np.abs(got - want) <= 1.05 * mag + 2.0 ** -8 * np.abs(want) + 1e-37), name
        norm = np.linalg.norm(want)
        if norm > 0 and v > 1:
            assert np.linalg.norm(got - want) <= TOL_DERIVED["bf16"] * norm, name
    # one of the gradients alone, and again: the same bits
    both = raw_bits(h.dX).copy(), raw_bits(h.dW).copy()
    h.dX.fill_(NAN)
    h.dW.fill_(NAN)
    h.bwd(scale=3.0, dw=False)
    assert torch.isnan(h.dW.float()).all()
    h.dW.fill_(NAN)
    h.bwd(scale=3.0, dx=False)
    h.check()
    assert np.array_equal(raw_bits(h.dX), both[0]) and np.array_equal(raw_bits(h.dW), both[1])


def test_tokens_that_are_not_trained_on():
    X, W, y, _ = make(300, 136, 1000, 5)
    y[:] = -1
    y[7], y[200] = 1000, 1 << 40
    h = Head(X, W, y)
    h.fwd()
    h.bwd()
    h.check()
    assert not h.loss.any() and not h.total.any() and not h.dX.any() and not h.dW.any()
    assert np.all(np.abs(to_host(h.lse) - C.ce_fwd(X, W, y)[1]) <= logit_error(X, W, 1.0, to_host(h.lse)))
    # a row that holds NaN and is not trained on: its lse is NaN, the others' loss and dX are what they were
    y[::2] = 3
    Xn = X.copy()
    Xn[1, 5] = np.nan
    a, b = Head(X, W, y), Head(Xn, W, y)
    for q in (a, b):
        q.fwd()
        q.bwd()
        q.check()
    assert torch.isnan(b.lse[1]) and b.loss[1] == 0 and torch.equal(a.loss, b.loss) and torch.equal(a.total, b.total)
    assert torch.equal(a.dX, b.dX) and not b.dX[1].any()
    # and one that is trained on carries it into its own loss and gradient
    Xn = X.copy()
    Xn[2, 0] = np.nan
    b = Head(Xn, W, y)
    b.fwd()
    b.bwd()
    b.check()
    assert torch.isnan(b.loss[2]) and torch.isnan(b.dX[2].float()).all() and torch.equal(a.loss[3:], b.loss[3:])
    assert torch.isfinite(b.dX[3:].float()).all() and torch.isnan(b.total[0])


def test_extreme_logits():
    t, d, v = 64, 64, 600
    X, W, y, _ = make(t, d, v, 9)
    big = I.round_to_dtype(X * 3000, "bf16")               # logits of some 10^4: one word has all the probability
    h = Head(big, W, y)
    h.fwd()
    h.bwd()
    h.check()
    loss, lse, total = C.ce_fwd(big, W, y)
    e = logit_error(big, W, 1.0, lse)
    assert np.all(np.abs(to_host(h.loss) - loss) <= 2 * e) and np.all(np.abs(to_host(h.lse) - lse) <= e)
    assert torch.isfinite(h.dX.float()).all() and torch.isfinite(h.dW.float()).all()
    h = Head(0 * X, W, y)                                  # all words alike
    h.fwd()
    h.bwd()
    h.check()
    want = C.ce_bwd(0 * X, W, y, denom=(y >= 0).sum())[0]
    # every element of D but the target's is the same power-of-ten fraction: its one rounding (2^-9 of it) repeats v times
    assert np.all(np.abs(to_host(h.dX) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -8 / (y >= 0).sum() * np.abs(W).mean(0) * 1.01)
    assert not h.dW.any()


def test_gradients_against_differences():
    t, d, v, eps = 40, 32, 300, 2.0 ** -4
    g = np.random.Generator(np.random.Philox(4))
    X = (np.round(g.standard_normal((t, d)) * 16).clip(-40, 40) / 16).astype(np.float32)      # exact after +- eps too
    W = (np.round(g.standard_normal((v, d)) * 8).clip(-30, 30) / 64).astype(np.float32)
    y = g.integers(0, v, t)
    y[::3] = -1
    h = Head(X, W, y)
    h.fwd()
    h.bwd()
    h.check()
    n = float((y >= 0).sum())

    def value(a):
        q = Head(a.astype(np.float32), W, y)
        q.fwd()
        return float(q.total[0].double().cpu()) / n

    for seed in range(3):
        p = np.sign(g.standard_normal((t, d)))
        s = p @ W.T.astype(np.float64)                        # change of the logits per unit
        # third derivative of log-sum-exp: a third central moment, at most 2 max |s|^3; roundings of the loss 2^-21 * 8 over eps
        tol = eps * eps / 6 * 2 * np.abs(s).max() ** 3 * 0.25 + 8 * 2.0 ** -21 / eps
        # and the gradient's own: 2^-8 of D and of dX, random over the sum
        tol += 2.0 ** -8 * np.abs(to_host(h.dX)).sum()
        quot = (value(X + eps * p) - value(X - eps * p)) / (2 * eps)
        assert abs(np.sum(to_host(h.dX) * p) - quot) <= tol, (seed, quot, tol)


def test_empty_streams_and_graph():
    d0 = B.make_ce_desc(0, 64, 100)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    W = torch.randn(100, 64, device="cuda").bfloat16()
    total, dW = torch.full((2,), 5.0, device="cuda"), torch.full((100, 64), 5.0, device="cuda").bfloat16()
    r, y0 = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    B.acx_linear_ce_fwd(d0, e, W, y0, r, r, total)
    B.acx_linear_ce_bwd(d0, e, W, y0, r, e, dW)
    assert not total.any() and not dW.any()
    X, Wh, y, w = make(900, 264, 9001, 3, True)
    ref = Head(X, Wh, y, w)
    ref.fwd()
    ref.bwd()
    torch.cuda.synchronize()
    streams, heads = [torch.cuda.Stream(), torch.cuda.Stream()], [Head(X, Wh, y, w) for _ in range(3)]
    torch.cuda.synchronize()
    for s, h in zip(streams, heads):
        h.fwd(s)
        h.bwd(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        heads[2].fwd()
        heads[2].bwd()
    g.replay()
    torch.cuda.synchronize()
    ref.check()
    for h in heads:
        for k in ("loss", "lse", "total", "dX", "dW"):
            assert torch.equal(getattr(h, k), getattr(ref, k)), k
