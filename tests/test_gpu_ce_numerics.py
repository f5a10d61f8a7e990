"""Accuracy of the vocabulary cross entropy where little is left of a difference: logits of minus infinity, tokens that are almost
certain, the systematic part of the tensor core's error, the roundings of D, weights of zero."""
import numpy as np
import pytest
import torch

from oracle import cross_entropy as C
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import inputs as I

from _harness import to_device, to_host

pytestmark = pytest.mark.gpu
NAN = float("nan")


def run(X, W, y, weight=None, logit_scale=1.0, backward=True, scale=1.0, with_loss=True):
    """Outputs of a forward and a backward call, by name; numpy float64."""
    (t, d), v = X.shape, W.shape[0]
    desc = B.make_ce_desc(t, d, v, logit_scale)
    Xd, Wd, yd = to_device(X, "bf16"), to_device(W, "bf16"), torch.from_numpy(np.asarray(y, np.int64)).cuda()
    wd = None if weight is None else to_device(np.asarray(weight, np.float32), "f32")
    o = {"loss": torch.full((t,), NAN, device="cuda"), "lse": torch.full((t,), NAN, device="cuda"), "total": torch.full((2,), NAN, device="cuda")}
    ws = B.alloc_ce_workspace(desc, B.ACX_OP_CE_BWD)
    ws.fill_(255)                  # NaN everywhere
    B.acx_linear_ce_fwd(desc, Xd, Wd, yd, o["loss"], o["lse"], o["total"], wd, ws)
    if backward:
        o["dX"], o["dW"] = torch.full_like(Xd, NAN), torch.full_like(Wd, NAN)
        B.acx_linear_ce_bwd(desc, Xd, Wd, yd, o["lse"], o["dX"], o["dW"], loss=o["loss"] if with_loss else None, weight=wd, scale=scale,
                            ws=ws)
    assert B.acx_last_device_status() == B.ACX_OK
    return {k: to_host(a) for k, a in o.items()}


# up to 64 tokens the words are the rows of a tile, above that the tokens
TOKENS = [7, 64, 65, 300]


@pytest.mark.parametrize("t", TOKENS)
@pytest.mark.parametrize("d,v", [(64, 700), (72, 65)])
def test_logits_of_minus_infinity(t, d, v):
    """Words whose products overflow to minus infinity count for nothing, whether they fill 64 columns, a lane's first word, the
    last words or all but one."""
    g = np.random.Generator(np.random.Philox(t + v))
    for some in range(3):
        gone = np.zeros(v, bool)
        if some == 0:
            gone[:min(v - 1, 128)] = True
            gone[-37:] = True
            gone[v // 2] = False
        elif some == 1:
            gone[g.random(v) < 0.5] = True
            gone[3] = False
        else:
            gone[:] = True
            gone[v - 1] = False
        X, W = I.gaussian((t, d), 1, 1.0, "bf16"), I.gaussian((v, d), 2, d ** -0.5, "bf16")
        X[:, 0] = 2.0 ** 120
        W[:, 0] = np.where(gone, -2.0 ** 20, 0.0)
        left = np.nonzero(~gone)[0]
        y = left[g.integers(0, len(left), t)]
        y[1] = -1
        o = run(X, W, y)
        loss, lse, total = C.ce_fwd(X, W, y)
        e = 2.0 ** -23 * (d / 16 + 8) * (np.abs(X[:, 1:]).astype(np.float64) @ np.abs(W[left, 1:]).astype(np.float64).T).max(1)
        e += 2.0 ** -21 * (1 + np.abs(lse))
        assert np.all(np.abs(o["lse"] - lse) <= e) and np.all(np.abs(o["loss"] - loss) <= 2 * e)
        assert abs(o["total"][0] - total[0]) <= np.sum(2 * e) + 2.0 ** -20 * np.sum(loss)
        assert not o["dW"][gone].any()
        dX, dW = C.ce_bwd(X, W, y)
        D = np.abs(C.ce_dlogits(X, W, y))
        per_d = 2.0 ** -8 * D + 4 * e[:, None] * np.minimum(D + 1, D * 4 + 1e-30)
        for got, want, mag in ((o["dX"], dX, (per_d + 2.0 ** -23 * (v / 16 + 40) * D) @ np.abs(W.astype(np.float64))),
                               (o["dW"], dW, (per_d + 2.0 ** -23 * (t / 16 + 40) * D).T @ np.abs(X.astype(np.float64)))):
            assert np.all(np.abs(got - want) <= 1.05 * mag + 2.0 ** -8 * np.abs(want) + 1e-37)
    # a target that is impossible: an infinite loss; its element of D is -1, everything else is what it was
    y2 = y.copy()
    y2[0] = np.nonzero(gone)[0][0]
    q = run(X, W, y2)
    assert q["loss"][0] == np.inf and q["total"][0] == np.inf and np.array_equal(q["lse"][1:], o["lse"][1:])
    assert np.array_equal(q["dX"][1:], o["dX"][1:]) and np.isfinite(q["dX"][0, 1:]).all()
    # and no possible word at all: nothing to be said
    W[:, 0] = -2.0 ** 20
    assert np.isnan(run(X, W, y, backward=False)["lse"]).all()


def _certain(t, v, d, shift, seed):
    """Tokens whose target's logit stands 8 to 26 above `shift`, the other words' around it."""
    g = np.random.Generator(np.random.Philox(seed))
    W = I.gaussian((v, d), seed + 1, d ** -0.5, "bf16")
    W[:, 0] = 1.0
    y = g.integers(0, v, t)
    rest = W[:, 1:].astype(np.float64)
    X = np.zeros((t, d))
    X[:, 0] = shift
    X[:, 1:] = 0.3 * I.gaussian((t, d - 1), seed + 2) + np.linspace(8, 26, t)[:, None] * rest[y] / (rest[y] ** 2).sum(1, keepdims=True)
    return I.round_to_dtype(X.astype(np.float32), "bf16"), W, y


@pytest.mark.parametrize("t", [40, 300])
@pytest.mark.parametrize("shift", [0.0, 24.0])
@pytest.mark.parametrize("v", [1, 2, 1000])
def test_loss_of_almost_certain_tokens(t, shift, v):
    """The loss is known relative to itself: log(1 + sum over the others / the target's), not a difference of two logits."""
    d = 64
    X, W, y = _certain(t, v, d, shift, 11 + v)
    loss, lse, _ = C.ce_fwd(X, W, y)
    L = C.logits(X, W)
    with np.errstate(divide="ignore"):
        others = np.exp(L - L[np.arange(t), y][:, None])
        others[np.arange(t), y] = 0
        loss = np.log1p(others.sum(1))               # (the oracle's difference in 64 bits has 1e-15 of the logits left)
    o = run(X, W, y, backward=False)
    # a logit's error, and the roundings of the two logarithms' difference and of the result
    e = 2.0 ** -23 * (d / 16 + 8) * (np.abs(X).astype(np.float64) @ np.abs(W).astype(np.float64).T).max(1) + 2.0 ** -21
    assert np.all(np.abs(o["loss"] - loss) <= 2 * e * loss)
    assert np.all(o["loss"] >= 0) and np.all(np.abs(o["lse"] - lse) <= e + 2.0 ** -22 * np.abs(lse))
    if v == 1000:
        assert loss.min() < 2e-6 and loss.max() > 0.1     # what the inputs are meant to cover


@pytest.mark.parametrize("t", [40, 300])
@pytest.mark.parametrize("shift", [0.0, 24.0])
@pytest.mark.parametrize("v", [1, 2, 1000])
def test_gradients_of_almost_certain_tokens(t, shift, v):
    """With the forward's losses a token's gradient is right relative to 1 - p, however small that is."""
    d = 64
    X, W, y = _certain(t, v, d, shift, 31 + v)
    w = (0.5 + np.random.Generator(np.random.Philox(5)).random(t)).astype(np.float32)
    at = np.arange(t)
    L = C.logits(X, W)
    D = np.exp(L - L.max(1, keepdims=True))
    D /= D.sum(1, keepdims=True)
    D[at, y] = 0.0
    rest = D.sum(1)
    D[at, y] = -rest                                  # p - 1 without the difference
    D *= w[:, None]
    o = run(X, W, y, w, scale=2.0)
    e = 2.0 ** -23 * (d / 16 + 8) * (np.abs(X).astype(np.float64) @ np.abs(W).astype(np.float64).T).max(1) + 2.0 ** -20
    e += 2.0 ** -22 * np.abs(C.ce_fwd(X, W, y)[1])   # the log-sum-exp is a 32-bit number
    A = np.abs(D)
    # bf16 elements of D (half a unit: 2^-8 of it; the target's is made good in fp32), their exponents, sums on the tensor core
    rel = np.full_like(A, 2.0 ** -8)
    rel_x = rel.copy()
    rel_x[at, y] = 0.0
    for name, want, mag in (("dX", 2 * (D @ W.astype(np.float64)), 2 * ((A * (rel_x + 2 * e[:, None] + 2.0 ** -23 * (v / 16 + 40))) @ np.abs(W.astype(np.float64)))),
                            ("dW", 2 * (D.T @ X.astype(np.float64)), 2 * ((A * (rel + 2 * e[:, None] + 2.0 ** -23 * (t / 16 + 40))).T @ np.abs(X.astype(np.float64))))):
        assert np.all(np.abs(o[name] - want) <= mag + 2.0 ** -8 * np.abs(want) + 1e-37), name
    if v == 1:
        assert not o["dX"].any() and not o["dW"].any()


def test_losses_of_another_type_or_shape_are_refused():
    X, W, y = _certain(9, 40, 64, 0.0, 3)
    d, Xd, Wd, yd = B.make_ce_desc(9, 64, 40), to_device(X, "bf16"), to_device(W, "bf16"), torch.from_numpy(y).cuda()
    lse, ws = torch.zeros(9, device="cuda"), B.alloc_ce_workspace(B.make_ce_desc(9, 64, 40), B.ACX_OP_CE_BWD)
    launches = B.acx_kernel_launches()
    for bad in (lse.double(), lse[:8].clone(), lse.cpu(), torch.zeros(18, device="cuda")[::2]):
        with pytest.raises(ValueError, match="loss must be"):
            B.acx_linear_ce_bwd(d, Xd, Wd, yd, lse, torch.empty_like(Xd), torch.empty_like(Wd), loss=bad, ws=ws)
    with pytest.raises(B.AcxError) as err:
        B.acx_linear_ce_bwd(d, Xd, Wd, yd, lse, torch.empty_like(Xd), torch.empty_like(Wd), loss=torch.zeros(16, device="cuda")[1:10], ws=ws)
    assert err.value.status == B.ACX_ERR_ALIGNMENT and B.acx_kernel_launches() == launches


@pytest.mark.parametrize("t", TOKENS)
def test_a_weight_of_zero_does_not_hide_a_nan(t):
    """A token that is trained on with weight zero adds 0 * softmax: nothing, or the NaN that its row holds, however many tokens
    there are."""
    X, W, y = _certain(t, 300, 64, 0.0, 7)
    w = np.ones(t, np.float32)
    w[3] = 0.0
    o = run(X, W, y, w)
    assert not o["dX"][3].any() and np.isfinite(o["dW"]).all() and o["dX"][2].any()
    X[3, 5] = np.nan
    n = run(X, W, y, w)
    assert np.isnan(n["loss"][3]) and np.isnan(n["dX"][3]).all() and np.isnan(n["dW"]).all()
    assert np.array_equal(n["dX"][4:], o["dX"][4:])
    y[3] = -100                     # not trained on: its D is zero (and zero times the NaN of X in D^T X)
    n = run(X, W, y, w)
    assert n["loss"][3] == 0 and not n["dX"][3].any() and np.isfinite(np.delete(n["dW"], 5, 1)).all()


@pytest.mark.parametrize("t", [1, 16, 100, 256, 257, 333, 512])
def test_error_of_dw_is_that_of_one_rounding(t):
    """Up to 512 tokens dW does not show that D is held in bfloat16: what rounding takes from the targets' elements, the large
    ones, is put back.  The other elements' roundings remain; both are random, so their squares add up."""
    d, v = 264, 3203
    g = np.random.Generator(np.random.Philox(t))
    X, W = I.gaussian((t, d), 1, 1.0, "bf16"), I.gaussian((v, d), 2, d ** -0.5, "bf16")
    y = (g.random(t) ** 3 * v).astype(np.int64)
    w = (g.random(t) * 2).astype(np.float32)
    o = run(X, W, y, w)
    want = C.ce_bwd(X, W, y, w)[1]
    one = np.linalg.norm(I.round_to_dtype(want.astype(np.float32), "bf16") - want)
    mag = (C.ce_dlogits(X, W, y, w) ** 2) * (X.astype(np.float64) ** 2).sum(1, keepdims=True)
    target = mag[np.arange(t), y].sum()
    assert np.linalg.norm(o["dW"] - want) <= 1.05 * one * np.sqrt(1 + (mag.sum() - target) / target)


def _raw_logits(X, W):
    """The logits of one word as the tensor core and the logits' scale give them: the log-sum-exp of tokens that are not trained on
    over a vocabulary of that word."""
    t, d = X.shape
    desc = B.make_ce_desc(t, d, 1)
    loss, lse = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    B.acx_linear_ce_fwd(desc, X, W, torch.full((t,), -100, device="cuda"), loss, lse, None, None, B.alloc_ce_workspace(desc, B.ACX_OP_CE_FWD))
    return lse.double()


@pytest.mark.parametrize("d", [256, 1024, 4096, 16384])
@pytest.mark.parametrize("kind", ["flat", "peaked", "outliers"])
@pytest.mark.parametrize("t", [64, 2048])
def test_dense_logits_have_no_systematic_error(d, kind, t):
    """What the tensor core's truncation takes from dense rows, some 0.135 * 2^-23 of a logit per 16 columns, is put back: at most half of
    it is left on average.  (Without the correction, or with its sign turned, the whole or twice of it would be.)"""
    g = torch.Generator(device="cuda").manual_seed(d)
    short, size = 0.0, 0.0
    for _ in range(2048 // t):
        W = torch.randn(1, d, generator=g, device="cuda") * d ** -0.5
        X = torch.randn(t, d, generator=g, device="cuda")
        if kind == "outliers":
            X[:, ::64] *= 8
        if kind != "flat":
            X += 12 * W / W.square().sum()
        X, W = X.bfloat16(), W.bfloat16()
        want = (X.double() @ W.double().T)[:, 0]
        short += float(((want - _raw_logits(X, W)) * want.sign()).sum())
        size += float(want.abs().sum())
    assert abs(short / size) <= 0.07 * 2.0 ** -23 * d / 16 + 2.0 ** -25      # (and the roundings to and from base 2)


@pytest.mark.parametrize("d", [1024, 4096, 16384])
@pytest.mark.parametrize("t", [48, 100])
def test_exact_sums(d, t):
    """Rows of +-1 lose nothing on the tensor core: there the correction is what the logits are off by, and no more; the target's own
    logit, summed apart, is exact."""
    g = np.random.Generator(np.random.Philox(d))
    v = 500
    X, W = (2.0 * g.integers(0, 2, s).astype(np.float32) - 1 for s in ((t, d), (v, d)))
    W *= 2.0 ** -np.round(np.log2(d ** 0.5 / 16))       # logits of size 16
    y = g.integers(0, v, t)
    o = run(X, W, y, backward=False)
    loss, lse, _ = C.ce_fwd(X, W, y)
    L = C.logits(X, W)
    rounding = 2.0 ** -22 * (1 + np.abs(L).max(1))
    assert np.all(np.abs(o["lse"] - lse) <= 0.14 * 2.0 ** -23 * d / 16 * np.abs(L).max(1) + rounding)
    assert np.all(np.abs(o["lse"] - o["loss"] - L[np.arange(t), y]) <= 2 * rounding)
