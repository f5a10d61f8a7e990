"""The vocabulary cross entropy beyond the sizes of the parity tests: backward passes of many pieces, whose launches overlap and use
the buffers of D again; wide hidden states; logits' scales below and at zero."""
import numpy as np
import pytest
import torch

from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Call:
    """Inputs and outputs of one call; inputs as a half-trained model has them, every seventh token not trained on."""

    def __init__(self, t, d, v, logit_scale=1.0, weighted=False):
        g = torch.Generator(device="cuda").manual_seed(t + d + v)
        rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.t, self.d, self.v, self.c = t, d, v, logit_scale
        self.W = (rnd(v, d) * d ** -0.5).bfloat16()
        self.y = (rand(t) ** 3 * v).long().clamp_(max=v - 1)
        self.X = (rnd(t, d) + 8 * rand(t, 1) * self.W[self.y].float()).bfloat16()
        self.y[::7] = -100
        self.y[t - 1] = v - 1
        self.w = rand(t) * 2 if weighted else None
        full = lambda *s, dt=torch.float32: torch.full(s, NAN, dtype=dt, device="cuda")  # noqa: E731
        self.loss, self.lse, self.total = full(t), full(t), full(2)
        self.dX, self.dW = full(t, d, dt=torch.bfloat16), full(v, d, dt=torch.bfloat16)
        self.desc = B.make_ce_desc(t, d, v, logit_scale)
        self.ws = B.alloc_ce_workspace(self.desc, B.ACX_OP_CE_BWD)
        self.ws.fill_(255)

    def fwd(self, stream=None):
        B.acx_linear_ce_fwd(self.desc, self.X, self.W, self.y, self.loss, self.lse, self.total, self.w, self.ws, stream=stream)

    def bwd(self, stream=None, dx=True, dw=True):
        B.acx_linear_ce_bwd(self.desc, self.X, self.W, self.y, self.lse, self.dX if dx else None, self.dW if dw else None, loss=self.loss,
                            weight=self.w, denom=self.total[1:], ws=self.ws, stream=stream)

    def check(self):
        """Every output against 64 bits, element by element, in blocks of tokens."""
        assert B.acx_last_device_status() == B.ACX_OK
        t, d, v, c = self.t, self.d, self.v, self.c
        W = self.W.double()
        ok = (self.y >= 0) & (self.y < v)
        wt = torch.where(ok, torch.ones(t, device="cuda") if self.w is None else self.w, 0.0).double()
        f = abs(c) / float(wt.sum())
        dW, dW_mag = torch.zeros_like(W), torch.zeros_like(W)
        total = torch.zeros(2, dtype=torch.float64, device="cuda")
        slack = 0.0
        for r0 in range(0, t, 512):
            r = slice(r0, min(t, r0 + 512))
            X, y, w = self.X[r].double(), self.y[r], wt[r]
            L = c * (X @ W.T)
            lse = torch.logsumexp(L, 1)
            at = torch.nonzero(ok[r])[:, 0]
            hot = torch.zeros_like(L)
            hot[at, y[at]] = 1.0
            loss = torch.where(ok[r], lse - (L * hot).sum(1), 0.0)
            # a logit: every addition of 16 products off by at most 2^-23 of the magnitudes summed; exponentials and logarithms
            e = 2.0 ** -23 * (d / 16 + 8) * abs(c) * (X.abs() @ W.abs().T).amax(1) + 2.0 ** -21 * (1 + lse.abs())
            assert bool(((self.lse[r] - lse).abs() <= e).all()) and bool(((self.loss[r] - loss).abs() <= 2 * e).all())
            D = (torch.softmax(L, 1) - hot) * w[:, None]
            total += torch.stack([(w * loss).sum(), w.sum()])
            slack += float((w * 2 * e).sum() + 2.0 ** -20 * (w * loss).sum())
            # D: its rounding to bfloat16 (2^-8 of it), the exponents' errors, sums on the tensor core; then one rounding
            A = D.abs()
            per_d = (2.0 ** -8 + 4 * e[:, None]) * A
            mag = 1.05 * f * ((per_d + 2.0 ** -23 * (v / 16 + 40) * A) @ W.abs())
            want = f * np.sign(c) * (D @ W)
            assert bool(((self.dX[r].double() - want).abs() <= mag + 2.0 ** -8 * want.abs() + 1e-37).all()), r0
            dW += f * np.sign(c) * (D.T @ X)
            dW_mag += 1.05 * f * ((per_d + 2.0 ** -23 * (t / 16 + 40) * A).T @ X.abs())
        assert bool(((self.dW.double() - dW).abs() <= dW_mag + 2.0 ** -8 * dW.abs() + 1e-37).all())
        assert abs(float(self.total[0] - total[0])) <= slack and abs(float(self.total[1] - total[1])) <= 2.0 ** -20 * float(total[1])


# pieces of at most 128 MB of D: five, five, seven (the last one short) and thirteen, of which three buffers hold three at a time
MANY = [(8192, 72, 40001), (4096, 136, 70000), (600, 64, 700001), (16384, 64, 50001)]


@pytest.mark.parametrize("t,d,v", MANY)
@pytest.mark.parametrize("weighted", [False, True])
def test_many_pieces(t, d, v, weighted):
    h = Call(t, d, v, 0.5 if weighted else 1.0, weighted)
    h.fwd()
    h.bwd()
    h.check()
    # one of the gradients alone, and again: the same bits
    both = h.dX.clone(), h.dW.clone()
    h.dX.fill_(NAN)
    h.dW.fill_(NAN)
    h.bwd(dw=False)
    h.bwd(dx=False)
    assert torch.equal(h.dX, both[0]) and torch.equal(h.dW, both[1])


def test_many_pieces_on_two_streams_in_a_graph_and_back_to_back():
    h = Call(8192, 72, 40001)
    h.fwd()
    h.bwd()
    torch.cuda.synchronize()
    want = h.dX.clone(), h.dW.clone()
    calls = [Call(8192, 72, 40001) for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, c in zip(streams, calls):
        for _ in range(3):                   # a forward lines up behind the backward of the call before
            c.fwd(s)
            c.bwd(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.fwd()
        h.bwd()
    for _ in range(3):
        h.dX.fill_(NAN)
        h.dW.fill_(NAN)
        graph.replay()
        for c in calls + [h]:
            assert torch.equal(c.dX, want[0]) and torch.equal(c.dW, want[1])
    assert B.acx_last_device_status() == B.ACX_OK


@pytest.mark.parametrize("t,d,v", [(70, 4104, 1500), (300, 8192, 700), (40, 16392, 600), (129, 65536, 300), (24, 65536, 300)])
def test_wide_hidden_states(t, d, v):
    h = Call(t, d, v)
    h.fwd()
    h.bwd()
    h.check()


@pytest.mark.parametrize("t", [33, 300])
@pytest.mark.parametrize("logit_scale", [-1.0, -0.37, 0.0])
@pytest.mark.parametrize("v", [65, 1111])
def test_scales_below_and_at_zero(t, logit_scale, v):
    h = Call(t, 136, v, logit_scale, True)
    h.fwd()
    h.bwd()
    h.check()
    if logit_scale == 0.0:
        n = np.float32(np.log(v))
        assert torch.allclose(h.lse, torch.full_like(h.lse, float(n)), rtol=1e-6) and not h.dX.any() and not h.dW.any()
