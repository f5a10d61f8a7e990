"""Pins of the row operators' oracle: the 8-bit format's error bound and corner values, gradients against central
differences of the forward formulas."""
import numpy as np
import pytest

from oracle import rows as R

RNG = lambda s: np.random.Generator(np.random.Philox(s))  # noqa: E731


@pytest.mark.parametrize("cols", [8, 120, 128, 136, 1000])
def test_q8_values_are_within_half_a_step(cols):
    x = (RNG(cols).standard_normal((17, cols)) * np.exp(RNG(1).standard_normal((17, 1)) * 3)).astype(np.float32)
    codes, scales = R.q8_encode(x)
    v = R.q8_decode(codes, scales)
    step = np.repeat(scales.astype(np.float64), 128, axis=1)[:, :cols]
    # half a step, and the roundings of 127 / a, of the product and of a / 127: 127 * 3 * 2^-24 of a step
    assert np.all(np.abs(v - x) <= step * (0.5 + 127 * 3 * 2.0 ** -24))
    assert np.abs(codes).max() == 127 and np.abs(codes).min() >= 0
    for g in range(scales.shape[1]):   # the largest element of a group has a code of +-127
        assert np.all(np.abs(codes[:, g * 128:(g + 1) * 128].astype(int)).max(1) == 127)


def test_q8_corner_values():
    x = np.zeros((6, 256), np.float32)
    x[1, 3], x[1, 200] = 2.0 ** -101, 2.0 ** -100
    x[2, 0], x[3, 130], x[4, 255] = np.inf, np.nan, -np.inf
    x[5] = 127.0 * 2.0 ** -3
    codes, scales = R.q8_encode(x)
    v = R.q8_decode(codes, scales)
    assert not v[0].any() and not v[1, :128].any()
    assert abs(v[1, 200] / 2.0 ** -100 - 1) < 1e-6
    assert np.isnan(v[2, :128]).all() and not v[2, 128:].any()
    assert np.isnan(v[3, 128:]).all() and np.isnan(v[4, 128:]).all() and not v[4, :128].any()
    assert np.array_equal(v[5], x[5].astype(np.float64))      # a power-of-two scale is exact
    half = np.zeros((1, 128), np.float32)
    half[0, :4] = (127, 0.5, 1.5, -2.5)                       # ties go to the even code
    assert R.q8_encode(half)[0][0, :4].tolist() == [127, 0, 2, -2]


def _central(f, x, d, eps=1e-5):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


def test_swiglu_gradient_is_the_difference_quotient():
    g = RNG(3)
    G, U, dH, d = (g.standard_normal((5, 24)) for _ in range(4))
    dG, dU = R.swiglu_bwd(dH, G, U)
    assert np.isclose(np.sum(dG * d), _central(lambda a: np.sum(dH * R.swiglu_fwd(a, U)), G, d), rtol=1e-7)
    assert np.isclose(np.sum(dU * d), _central(lambda a: np.sum(dH * R.swiglu_fwd(G, a)), U, d), rtol=1e-7)
    assert np.isfinite(R.swiglu_fwd(np.array([[-1000.0, 1000.0]]), np.ones((1, 2)))).all()


@pytest.mark.parametrize("join,post,gate", [(False, False, False), (True, False, False), (True, True, False), (True, False, True), (True, True, True)])
def test_norm_join_gradients_are_difference_quotients(join, post, gate):
    g = RNG(7)
    m, n, alpha, eps = 4, 16, 0.7, 1e-5
    a = {"h": g.standard_normal((m, n)), "b": g.standard_normal((m, n)) if join else None,
         "w_post": 1 + 0.3 * g.standard_normal(n) if post else None, "gate": g.standard_normal(n) if gate else None,
         "w_pre": 1 + 0.3 * g.standard_normal(n)}
    dy, dn = g.standard_normal((m, n)), g.standard_normal((m, n))

    def value(**kw):
        q = {**a, **kw}
        t, y, _, _ = R.norm_join_fwd(q["h"], q["b"], q["w_post"], q["gate"], q["w_pre"], alpha, eps)
        return np.sum(dy * y) + np.sum(dn * t)

    _, _, r_b, r_t = R.norm_join_fwd(a["h"], a["b"], a["w_post"], a["gate"], a["w_pre"], alpha, eps)
    got = R.norm_join_bwd(dy, dn, a["h"], a["b"], a["w_post"], a["gate"], a["w_pre"], r_b, r_t, alpha)
    names = {"dh": "h", "db": "b", "dw_post": "w_post", "dgate": "gate", "dw_pre": "w_pre"}
    assert set(got) == {k for k, v in names.items() if a[v] is not None}
    for k, grad in got.items():
        d = g.standard_normal(grad.shape)
        assert np.isclose(np.sum(grad * d), _central(lambda x: value(**{names[k]: x}), a[names[k]], d), rtol=1e-6, atol=1e-8), k
