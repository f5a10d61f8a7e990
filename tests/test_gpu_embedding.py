"""Embedding rows and the table's gradient against the fp64 oracle, and the clipping of gradients."""
import math

import numpy as np
import pytest
import torch

from oracle import embedding as oe
from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN = float("nan")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def numbers(t):
    return t.double().cpu().numpy()


# T, d, vocab, dtype, grad dtype, scale, kind of ids
CASES = [
    (1, 8, 1, "bf16", "bf16", 1.0, "random"),
    (1, 64, 5, "f32", "f32", 2.0, "all outside"),
    (7, 1024, 3, "bf16", "f32", 1.0, "random"),
    (32, 40, 1000, "f32", "bf16", 0.5, "all different"),
    (33, 1032, 17, "bf16", "bf16", 1.0, "random"),
    (64, 64, 40, "f32", "f32", 1.0, "one word"),
    (65, 2048, 300, "bf16", "f32", 22.6, "skewed"),
    (1000, 136, 513, "f32", "f32", 31.6, "skewed"),
    (1024, 72, 1 << 22, "bf16", "bf16", 1.0, "far apart"),
    (3001, 24, 511, "f32", "f32", 1.0, "runs"),
    (3001, 24, 512, "f32", "bf16", 1.0, "one word"),
    (5000, 3000, 257, "bf16", "f32", 1.0, "skewed"),
    (8192, 64, 100000, "f32", "f32", 1.0, "all different"),
    (8193, 64, 2, "bf16", "f32", 1.0, "random"),
    (40000, 16, 70000, "f32", "f32", 1.0, "skewed"),
    (70001, 8, 9, "f32", "f32", 1.0, "runs"),
    # behind the sizes at which the sort changes: one block up to 8192, one item per thread up to 148 blocks, then eight
    (16384, 520, 130000, "bf16", "f32", 1.0, "skewed"),
    (151_552, 8, 600, "bf16", "bf16", 1.0, "skewed"),
    (151_553, 8, 600, "f32", "f32", 1.0, "random"),
    (300_001, 16, 300_000, "bf16", "f32", 1.0, "skewed"),
]


def make_ids(kind, T, vocab, rng):
    if kind == "all outside":
        return rng.choice([-1, -100, vocab, vocab + 7, 2 ** 40, -2 ** 63], T)
    if kind == "one word":
        return np.full(T, vocab - 1)
    if kind == "all different":
        return rng.permutation(max(vocab, T))[:T]
    if kind == "far apart":
        return rng.choice([0, 1, vocab - 1, vocab - 2, vocab // 2, 255, 256, 65535, 65536], T)
    if kind == "runs":
        return (np.arange(T) // 97 * 5) % (vocab + 2) - 1
    ids = (rng.random(T) ** (4 if kind == "skewed" else 1) * vocab).astype(np.int64)
    ids[rng.random(T) < 0.1] = -100
    if kind == "skewed":
        ids[rng.random(T) < 0.2] = vocab // 2
    return ids


class Table:
    def __init__(self, T, d, vocab, dtype, grad, scale, kind, seed=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.ids = make_ids(kind, T, vocab, rng).astype(np.int64)
        self.E = torch.randn(vocab, d, generator=g).to(TYPES[dtype])
        self.dY = torch.randn(T, d, generator=g).to(TYPES[dtype])
        self.dE = torch.randn(vocab, d, generator=g).to(TYPES[grad])
        self.shape, self.dtype, self.grad, self.scale = (T, d, vocab), dtype, grad, scale
        self.desc = B.make_embed_desc(T, d, vocab, dtype, grad, scale=scale)
        self.ws = B.alloc_embed_workspace(self.desc, B.ACX_OP_EMBED_BWD)
        self.dev_ids = torch.from_numpy(self.ids).cuda()

    def gradient(self, beta, dE, **kw):
        B.acx_embed_bwd(self.desc, self.dev_ids, self.dY.cuda(), dE, beta=beta, ws=self.ws, **kw)
        return dE


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rows(case):
    t = Table(*case)
    T, d, vocab = t.shape
    Y = torch.full((T, d), NAN, dtype=TYPES[t.dtype], device="cuda")
    B.acx_embed_fwd(t.desc, t.dev_ids, t.E.cuda(), Y)
    want = oe.lookup(t.ids, numbers(t.E), np.float32(t.scale).item())
    # one fp32 product, one rounding
    assert (np.abs(numbers(Y) - want) <= (HALF_STEP[t.dtype] + 2.0 ** -24) * np.abs(want)).all()


@pytest.mark.parametrize("beta", [0.0, 1.0, -0.5])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_table_gradient(case, beta):
    t = Table(*case)
    T, d, vocab = t.shape
    dE = torch.full((vocab, d), NAN, dtype=TYPES[t.grad], device="cuda") if beta == 0.0 else t.dE.cuda()
    t.gradient(beta, dE)
    want, size = oe.table_gradient(t.ids, numbers(t.dY), vocab, np.float32(t.scale).item(), numbers(t.dE), beta)
    got = numbers(dE)
    # a sum of n terms level by level makes at most 32 additions per level, each half a step of the partial sum: 32 * levels + 2 of them
    levels = 1 + max(0, math.ceil(math.log(max(T / 32, 1), 16)))
    bound = HALF_STEP[t.grad] * np.abs(want) + (32 * levels + 4) * 2.0 ** -24 * size
    assert (np.abs(got - want) <= bound).all()
    absent = np.setdiff1d(np.arange(vocab), t.ids)
    if beta == 1.0 and len(absent):
        assert torch.equal(dE[torch.from_numpy(absent).cuda()].cpu(), t.dE[torch.from_numpy(absent)])
    if beta == 0.0:
        assert not got[absent].any()
        again = t.gradient(beta, torch.full_like(dE, NAN))
        assert torch.equal(again, dE)          # fixed order: the same bits


@pytest.mark.parametrize("beta", [0.0, 1.0, 0.25])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_no_tokens(beta, grad):
    desc = B.make_embed_desc(0, 24, 7, "bf16", grad)
    dE = torch.randn(7, 24, device="cuda").to(TYPES[grad])
    want = (beta * dE.double()).to(TYPES[grad])
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    B.acx_embed_bwd(desc, none, torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), dE, beta=beta)
    B.acx_embed_fwd(desc, none, torch.zeros(7, 24, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(dE, want)


def test_rows_that_are_not_read_may_be_anything():
    """Words that no token names, and gradients of tokens that stand for no word, reach nothing."""
    t = Table(300, 64, 50, "f32", "f32", 1.0, "random")
    E, dY = t.E.cuda(), t.dY.clone()
    absent = torch.from_numpy(np.setdiff1d(np.arange(50), t.ids[:100])).cuda()
    E[absent] = NAN
    desc = B.make_embed_desc(100, 64, 50, "f32")
    Y = torch.empty(100, 64, device="cuda")
    B.acx_embed_fwd(desc, t.dev_ids[:100], E, Y)
    assert torch.isfinite(Y).all()
    dY[torch.from_numpy((t.ids < 0) | (t.ids >= 50))] = NAN
    t.dY = dY
    assert torch.isfinite(t.gradient(0.0, torch.full((50, 64), NAN, device="cuda"))).all()


def test_gradient_is_the_derivative_of_the_rows():
    """<dE, V> = d/de <Y(E + e V), G>: both sides linear, so the difference quotient is exact up to rounding."""
    t = Table(500, 40, 31, "f32", "f32", 3.0, "skewed")
    g = torch.Generator().manual_seed(5)
    V = torch.randn(31, 40, generator=g).cuda()
    rows = []
    for E in (t.E.cuda() + V, t.E.cuda() - V):
        Y = torch.empty(500, 40, device="cuda")
        B.acx_embed_fwd(t.desc, t.dev_ids, E, Y)
        rows.append(Y.double())
    dE = t.gradient(0.0, torch.empty(31, 40, device="cuda"))
    left, right = (dE.double() * V.double()).sum(), ((rows[0] - rows[1]) / 2 * t.dY.cuda().double()).sum()
    assert abs(float(left - right)) <= 2.0 ** -20 * float((rows[0].abs() * t.dY.cuda().double().abs()).sum())


# ------------------------------------------------------------------------------------------------------------ clipping
def gradients(sizes, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g) * 2.0 ** (i % 5 - 2)).to(TYPES[t]) for i, (n, t) in enumerate(sizes)]


def check_clip(grads, max_norm, weights=None, out_types=None):
    want_norm, want_f, want = oe.clip([numbers(g) for g in grads], max_norm, weights)
    dev = [g.cuda() for g in grads]
    out = None if out_types is None else [torch.full(g.shape, NAN, dtype=TYPES[t], device="cuda") for g, t in zip(grads, out_types)]
    lst = B.make_grad_list(dev, weights, out)
    total, ws = torch.full((2,), NAN, device="cuda"), B.alloc_grad_workspace(lst)
    B.acx_grad_clip(lst, max_norm, total, ws=ws)
    norm, f = total.tolist()
    # squares of eight in fp32, then 64 bits; the root halves the relative error
    assert abs(norm - want_norm) <= 8 * 2.0 ** -24 * want_norm
    assert abs(f - want_f) <= 8 * 2.0 ** -24 * want_f
    for i, (x, w) in enumerate(zip(dev if out is None else out, want)):
        half = HALF_STEP["bf16" if x.dtype == torch.bfloat16 else "f32"]
        assert (np.abs(numbers(x) - w) <= (half + 12 * 2.0 ** -24) * np.abs(w)).all(), i
    if out is not None:
        assert all(torch.equal(a.cpu(), b) for a, b in zip(dev, grads))
    return total


SIZES = {
    "one": [(1, "f32")],
    "empty among others": [(0, "f32"), (5, "bf16"), (0, "bf16"), (9, "f32")],
    "odd": [(n, t) for n in (1, 7, 8, 9, 255, 2047, 2049, 8191, 8192, 8193, 16385) for t in ("f32", "bf16")],
    "many small": [(1 + 13 * i % 97, "bf16" if i % 3 else "f32") for i in range(700)],
    "large": [(5_000_011, "bf16"), (3_000_000, "f32"), (17, "f32")],
}


@pytest.mark.parametrize("name", SIZES)
@pytest.mark.parametrize("fraction", [0.5, 2.0])
def test_clip(name, fraction):
    grads = gradients(SIZES[name])
    norm = oe.clip([numbers(g) for g in grads], 1.0)[0]
    check_clip(grads, fraction * norm)
    check_clip(grads, fraction * norm, weights=[0.5 + i % 3 for i in range(len(grads))])
    check_clip(grads, fraction * norm, out_types=["f32" if i % 2 else "bf16" for i in range(len(grads))])


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e15, 1e19])
def test_squares_outside_the_range_of_fp32(scale):
    """(1e19: the squares overflow fp32; 1e-22 and below: they are its smallest numbers or none.)"""
    grads = gradients([(1000, "f32"), (77, "f32")], scale=scale)
    norm = oe.clip([numbers(g) for g in grads], 1.0)[0]
    check_clip(grads, float(np.float32(0.25 * norm)))


def test_zero_gradients_and_weights():
    check_clip([torch.zeros(100), torch.zeros(3, dtype=torch.bfloat16)], 1.0)
    check_clip(gradients([(100, "f32"), (50, "f32")]), 1.0, weights=[0.0, 1.0])
    check_clip(gradients([(100, "f32"), (50, "bf16")]), float("inf"), out_types=["f32", "f32"])


@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    grads = gradients([(100, "f32"), (5000, "bf16")])
    grads[1][4321] = bad
    dev = [g.cuda() for g in grads]
    lst = B.make_grad_list(dev)
    total = torch.zeros(2, device="cuda")
    B.acx_grad_clip(lst, 0.1, total, ws=B.alloc_grad_workspace(lst))
    assert not math.isfinite(total[0]) and float(total[1]) == 1.0
    assert all(torch.equal(a.cpu().view(torch.uint8), b.view(torch.uint8)) for a, b in zip(dev, grads))


def test_a_list_without_elements():
    total = check_clip([torch.zeros(0), torch.zeros(0, dtype=torch.bfloat16)], 1.0)
    assert total.tolist() == [0.0, 1.0]


def test_clip_again_and_same_bits():
    grads = gradients([(100_003, "f32"), (40_000, "bf16")], scale=3.0)
    results = []
    for _ in range(2):
        dev = [g.cuda() for g in grads]
        lst = B.make_grad_list(dev)
        total, ws = torch.zeros(2, device="cuda"), B.alloc_grad_workspace(lst)
        B.acx_grad_clip(lst, 10.0, total, ws=ws)
        first = total.clone()
        B.acx_grad_clip(lst, 10.5, total, ws=ws)      # now below it
        assert float(first[1]) < 1.0 and float(total[1]) == 1.0 and abs(float(total[0]) - 10.0) < 0.02
        results.append((first, *dev))
    assert all(torch.equal(a, b) for a, b in zip(*results))
