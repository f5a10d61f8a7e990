"""Pins of the cross entropy's oracle: closed forms, gradients against central differences, tokens that are not trained on;
and the C ABI's refusals, which need no GPU."""
import ctypes

import numpy as np
import pytest

from oracle import cross_entropy as C
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import build as acx_build


def _inputs(t, d, v, seed=1):
    g = np.random.Generator(np.random.Philox(seed))
    y = g.integers(0, v, t)
    y[::4] = -100
    return g.standard_normal((t, d)), 0.3 * g.standard_normal((v, d)), y, g.random(t) * 2


def test_closed_forms():
    X, W, y, _ = _inputs(6, 5, 9)
    loss, lse, total = C.ce_fwd(0 * X, W, y)
    assert np.allclose(lse, np.log(9)) and np.allclose(loss[y >= 0], np.log(9)) and not loss[y < 0].any()
    assert np.allclose(total, [np.log(9) * (y >= 0).sum(), (y >= 0).sum()])
    one, _, _ = C.ce_fwd(X, W[:1], np.zeros(6, int))                    # one word: certain
    assert np.allclose(one, 0)
    assert not C.ce_dlogits(X, W, y)[y < 0].any()
    assert np.allclose(C.ce_dlogits(X, W, y).sum(1), 0)                 # softmax and onehot both sum to one
    assert not np.any(C.ce_bwd(X, W, np.full(6, 9), denom=0.0)[1])


@pytest.mark.parametrize("weighted", [False, True])
def test_gradients_are_difference_quotients(weighted):
    X, W, y, w = _inputs(7, 6, 11, 2)
    w = w if weighted else None
    kw = dict(weight=w, logit_scale=0.5)
    den = C.ce_fwd(X, W, y, **kw)[2][1]
    dX, dW = C.ce_bwd(X, W, y, denom=den, scale=3.0, **kw)
    g = np.random.Generator(np.random.Philox(3))
    f = lambda a, b: 3.0 * C.ce_fwd(a, b, y, **kw)[2][0] / den  # noqa: E731
    e = 1e-5
    p, q = g.standard_normal(X.shape), g.standard_normal(W.shape)
    assert np.isclose(np.sum(dX * p), (f(X + e * p, W) - f(X - e * p, W)) / (2 * e), rtol=1e-7)
    assert np.isclose(np.sum(dW * q), (f(X, W + e * q) - f(X, W - e * q)) / (2 * e), rtol=1e-7)


def test_refusals_happen_on_the_host():
    acx_build.build()
    L = B.lib()
    good = dict(tokens=64, d=64, vocab=1000)
    fwd = lambda d, x=0x1000, ws=0x9000, n=1 << 30: L.acx_linear_ce_fwd(d, x, 0x2000, 0x3000, None, 0x4000, 0x5000, None, ws, n, None)  # noqa: E731
    bwd = lambda d, dx=0x5000, dw=0x6000, s=1.0, n=1 << 30: L.acx_linear_ce_bwd(d, 0x1000, 0x2000, 0x3000, None, 0x4000, None, s, dx, dw, 0x9000, n, None)  # noqa: E731
    for bad in (dict(tokens=-1), dict(d=60), dict(d=0), dict(d=65544), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(tokens=(1 << 24) + 1)):
        d = B.make_ce_desc(**{**good, **bad})
        assert fwd(d) == B.ACX_ERR_UNSUPPORTED_SHAPE and bwd(d) == B.ACX_ERR_UNSUPPORTED_SHAPE, bad
        assert B.acx_ce_workspace_bytes(d, B.ACX_OP_CE_BWD) == 0
    d = B.make_ce_desc(**good)
    d.struct_size = 8
    assert fwd(d) == B.ACX_ERR_INVALID_ARG
    d = B.make_ce_desc(**good)
    d.io_dtype = B.ACX_F32
    assert fwd(d) == B.ACX_ERR_INVALID_ARG
    assert fwd(B.make_ce_desc(**good, logit_scale=float("nan"))) == B.ACX_ERR_INVALID_ARG
    d = B.make_ce_desc(**good)
    assert fwd(d, x=None) == B.ACX_ERR_INVALID_ARG and fwd(d, x=0x1008) == B.ACX_ERR_ALIGNMENT
    need_f, need_b = (B.acx_ce_workspace_bytes(d, op) for op in (B.ACX_OP_CE_FWD, B.ACX_OP_CE_BWD))
    assert 0 < need_f <= need_b and B.acx_ce_workspace_bytes(d, B.ACX_OP_FWD) == 0
    assert fwd(d, n=need_f - 1) == B.ACX_ERR_WORKSPACE and fwd(d, ws=None) == B.ACX_ERR_WORKSPACE
    assert bwd(d, n=need_b - 1) == B.ACX_ERR_WORKSPACE
    assert bwd(d, dx=None, dw=None) == B.ACX_ERR_INVALID_ARG and bwd(d, s=float("inf")) == B.ACX_ERR_INVALID_ARG
    assert ctypes.sizeof(B.acx_ce_desc) == 40
