"""The fp64 oracles of attention, the embedding table and the clipping against plain loops and differences."""
import math

import numpy as np
import pytest

from oracle import attention as oa
from oracle import embedding as oe


def _loops(q, k, v, offsets, causal, prefix, scale, softcap, slopes):
    """One query and one head at a time."""
    T, H, d = q.shape
    o, lse = np.zeros((T, H, d)), np.full((H, T), -np.inf)
    group = H // k.shape[1]
    for n, (s, e) in enumerate(zip(offsets[:-1], offsets[1:])):
        for i in range(s, e):
            for h in range(H):
                js = [j for j in range(s, e) if not causal or j <= i or (prefix is not None and j < s + prefix[n])]
                z = []
                for j in js:
                    x = scale * float(q[i, h] @ k[j, h // group])
                    x = softcap * math.tanh(x / softcap) if softcap else x
                    z.append(x - (slopes[h] * abs(i - j) if slopes is not None else 0.0))
                top = max(z)
                w = [math.exp(x - top) for x in z]
                lse[h, i] = top + math.log(sum(w))
                o[i, h] = sum(a * v[j, h // group] for a, j in zip(w, js)) / sum(w)
    return o, lse


CASES = {
    "causal": dict(),
    "all": dict(causal=False),
    "prefix": dict(prefix=[2, 0, 9]),
    "cap": dict(softcap=0.7),
    "distance": dict(slopes=[0.5, 0.1]),
    "everything": dict(prefix=[3, 1, 0], softcap=1.5, slopes=[0.25, 0.0], scale=0.9),
}


def _inputs(seed=0):
    rng = np.random.default_rng(seed)
    T, H, K, d = 14, 2, 1, 3
    return rng.normal(size=(T, H, d)), rng.normal(size=(T, K, d)), rng.normal(size=(T, K, d)), rng.normal(size=(T, H, d)), [1, 6, 7, 12]


@pytest.mark.parametrize("name", CASES)
def test_attention_is_the_loops(name):
    q, k, v, _, offsets = _inputs()
    kw = CASES[name]
    got = oa.attention(q, k, v, offsets, **kw)
    o, lse = _loops(q, k, v, offsets, kw.get("causal", True), kw.get("prefix"), kw.get("scale", 3 ** -0.5), kw.get("softcap", 0.0), kw.get("slopes"))
    assert np.allclose(got["o"], o, rtol=1e-12, atol=1e-13)
    assert np.array_equal(np.isneginf(got["lse"]), np.isneginf(lse))
    assert np.allclose(got["lse"][:, 1:12], lse[:, 1:12], rtol=1e-12)


@pytest.mark.parametrize("name", CASES)
def test_gradients_are_the_differences(name):
    q, k, v, do, offsets = _inputs(1)
    kw = CASES[name]
    got = oa.attention(q, k, v, offsets, do=do, **kw)
    f = lambda: float((oa.attention(q, k, v, offsets, **kw)["o"] * do).sum())  # noqa: E731
    step = 1e-5
    for x, g in ((q, got["dq"]), (k, got["dk"]), (v, got["dv"])):
        for at in np.ndindex(*x.shape):
            keep = x[at]
            x[at] = keep + step
            up = f()
            x[at] = keep - step
            down = f()
            x[at] = keep
            assert abs((up - down) / (2 * step) - g[at]) < 1e-7, (name, at)      # step^2 / 6 times a third derivative, and 1e-16 / step


def test_bounds_hold_for_rounded_probabilities():
    """What the bounds are for: o from probabilities rounded to bf16, in fp64 otherwise, is within them, and they are not wide."""
    q, k, v, _, offsets = _inputs(2)
    got = oa.attention(q, k, v, offsets, causal=False)
    worst = 0.0
    for s, e in zip(offsets[:-1], offsets[1:]):
        for h in range(2):
            x = q[s:e, h] @ k[s:e, 0].T / math.sqrt(3)
            p = np.exp(x - x.max(1, keepdims=True))
            total = p.sum(1, keepdims=True)
            bits = p.astype(np.float32).view(np.uint32)
            p16 = ((bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)
            off = np.abs(p16 @ v[s:e, 0] / total - got["o"][s:e, h])
            assert (off <= got["o_bound"][s:e, h]).all()
            worst = max(worst, float(got["o_bound"][s:e, h].max()))
    assert worst < 2.0 ** -5


def test_table_gradient_is_the_derivative():
    rng = np.random.default_rng(3)
    E, dY, ids = rng.normal(size=(5, 4)), rng.normal(size=(7, 4)), [0, 3, 3, -1, 5, 4, 3]
    g, size = oe.table_gradient(ids, dY, 5, 0.5, rng.normal(size=(5, 4)), 0.0)
    for at in np.ndindex(5, 4):
        more = E.copy()
        more[at] += 1.0
        assert abs(((oe.lookup(ids, more, 0.5) - oe.lookup(ids, E, 0.5)) * dY).sum() - g[at]) < 1e-12
    assert (size >= np.abs(g)).all() and not oe.lookup(ids, E)[[3, 4]].any()
    old = rng.normal(size=(5, 4))
    assert np.allclose(oe.table_gradient(ids, dY, 5, 0.5, old, -2.0)[0], g - 2.0 * old)


def test_clip():
    norm, f, out = oe.clip([[3.0], [4.0, 0.0]], 1.0)
    assert (norm, f) == (5.0, 0.2) and np.allclose(out[1], [0.8, 0.0])
    assert oe.clip([[3.0], [4.0]], 5.0)[1] == 1.0
    assert oe.clip([[3.0], [4.0]], 1.0, weights=[0.0, 4.0])[0] == 8.0
    assert oe.clip([[np.inf]], 1.0)[1] == 1.0
