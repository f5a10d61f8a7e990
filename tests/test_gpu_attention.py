"""Attention over packed documents against the fp64 oracle: element-wise, within what the roundings of bf16 may do (the oracle's
bounds, derived there).  Outputs start as NaN, so that what a call leaves out shows; what lies beside them has to stay."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu
BF, NAN = torch.bfloat16, float("nan")


class Attn:
    """One batch: its inputs on the GPU, the calls, and what the oracle says."""

    def __init__(self, lengths, heads, kv_heads, d, *, before=0, behind=0, causal=True, prefix=None, cap=0.0, alibi=False, stacked=True, seed=0,
                 size=1.5, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.T = T = before + sum(lengths) + behind
        self.H, self.K, self.d = heads, kv_heads, d
        rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        x = size * rnd(T, (heads + 2 * kv_heads) * d)
        x[:, heads * d:(heads + kv_heads) * d:8] += 1.0
        self.offsets = before + np.concatenate([[0], np.cumsum(lengths)])
        self.prefix, self.cap, self.causal, self.scale = prefix, cap, causal, scale
        self.slopes = [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)] if alibi else None
        self.x, self.do = x.to(BF), (0.3 * rnd(T, heads, d)).to(BF)
        pad = np.ones(T, bool)
        pad[self.offsets[0]:self.offsets[-1]] = False
        self.pad = pad
        self.desc = B.make_attn_desc(T, heads, kv_heads, d, docs=len(lengths), causal=causal, softcap=cap, scale=scale)
        dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t).cuda()  # noqa: E731
        self.dev_offsets = dev(self.offsets, torch.int32)
        self.dev_prefix = None if prefix is None else dev(prefix, torch.int32)
        self.dev_slopes = None if not alibi else dev(self.slopes, torch.float32)
        xg, self.dog = self.x.cuda(), self.do.cuda()
        if pad.any():     # padding may hold anything
            xg[torch.from_numpy(pad).cuda()] = NAN
            self.dog[torch.from_numpy(pad).cuda()] = float("inf")
        self.stacked = stacked
        self.q, self.k, self.v = self.split(xg)
        self.plan = B.alloc_attn_workspace(self.desc, B.ACX_OP_ATTN_PLAN)
        self.ws = B.alloc_attn_workspace(self.desc, B.ACX_OP_ATTN_BWD)

    def split(self, x):
        parts = [p.unflatten(1, (-1, self.d)) for p in x.split([self.H * self.d, self.K * self.d, self.K * self.d], 1)]
        return parts if self.stacked else [p.contiguous() for p in parts]

    def forward(self, want_lse=True, stream=None):
        o, lse = torch.full((self.T, self.H, self.d), NAN, dtype=BF, device="cuda"), torch.full((self.H, self.T), NAN, device="cuda")
        B.acx_attn_plan(self.desc, self.dev_offsets, self.plan, prefix=self.dev_prefix, stream=stream)
        B.acx_attn_fwd(self.desc, self.q, self.k, self.v, self.plan, o, lse if want_lse else None, slopes=self.dev_slopes, stream=stream)
        return o, lse

    def backward(self, o, lse, stream=None):
        g = self.split(torch.full((self.T, (self.H + 2 * self.K) * self.d), NAN, dtype=BF, device="cuda"))
        B.acx_attn_bwd(self.desc, self.q, self.k, self.v, self.plan, o, self.dog, lse, *g, slopes=self.dev_slopes, ws=self.ws, stream=stream)
        return g

    def check(self, backward=True):
        o, lse = self.forward()
        got = {"o": o, "lse": lse}
        if backward:
            got.update(zip(("dq", "dk", "dv"), self.backward(o, lse)))
        assert B.acx_last_device_status() == B.ACX_OK
        self.compare(got)
        return got

    def compare(self, got):
        n = [self.H * self.d, self.K * self.d, self.K * self.d]
        q, k, v = (p.unflatten(1, (-1, self.d)).double().numpy() for p in self.x.split(n, 1))
        want = oa.attention(q, k, v, self.offsets, causal=self.causal, prefix=self.prefix, softcap=self.cap, slopes=self.slopes,
                            scale=self.scale, do=self.do.double().numpy() if "dq" in got else None)
        for name, t in got.items():
            x = t.double().cpu().numpy()
            if name == "lse":
                assert np.array_equal(np.isneginf(x), np.isneginf(want["lse"])), name
                x, w, b = (np.where(self.pad[None], 0.0, a) for a in (x, want["lse"], want["lse_bound"]))
            else:
                w, b = want[name], want[name + "_bound"]
                assert not x[self.pad].any() and np.isfinite(x).all(), (name, "padding")
            # fp32 sums leave an absolute rest of the tensor's size where everything cancels
            worst = np.max(np.abs(x - w) - b) if x.size else 0.0
            assert worst <= 2.0 ** -22 * (1 + np.abs(w).max(initial=0.0)), (name, worst, np.unravel_index(np.argmax(np.abs(x - w) - b), x.shape))


CASES = {
    "one token": dict(lengths=[1], heads=1, kv_heads=1, d=64),
    "two": dict(lengths=[2], heads=2, kv_heads=1, d=64),
    "one tile": dict(lengths=[128], heads=2, kv_heads=2, d=128),
    "a row more": dict(lengths=[129], heads=3, kv_heads=1, d=128),
    "two halves": dict(lengths=[256], heads=2, kv_heads=1, d=64),
    "behind two halves": dict(lengths=[257], heads=2, kv_heads=1, d=64),
    "long": dict(lengths=[1111], heads=4, kv_heads=2, d=128),
    "long 64": dict(lengths=[1500], heads=7, kv_heads=1, d=64),
    "narrow": dict(lengths=[300], heads=2, kv_heads=1, d=8),
    "d 40": dict(lengths=[200, 77], heads=2, kv_heads=1, d=40),
    "d 72": dict(lengths=[333, 130], heads=6, kv_heads=2, d=72),
    "d 120": dict(lengths=[260], heads=2, kv_heads=2, d=120),
    "all see all": dict(lengths=[77, 300, 1, 128], heads=2, kv_heads=1, d=64, causal=False),
    "all see all 128": dict(lengths=[700], heads=2, kv_heads=1, d=128, causal=False),
    "many documents": dict(lengths=[1, 1, 2, 31, 127, 128, 129, 1, 255, 256, 257, 3, 400], heads=2, kv_heads=1, d=64),
    "empty documents": dict(lengths=[0, 50, 0, 0, 131, 0], heads=2, kv_heads=1, d=64),
    "padding": dict(lengths=[100, 200], before=37, behind=91, heads=2, kv_heads=1, d=64),
    "padding 128": dict(lengths=[130, 5], before=3, behind=300, heads=2, kv_heads=2, d=128, causal=False),
    "prefix": dict(lengths=[300, 200, 129, 64], prefix=[100, 0, 129, 1], heads=2, kv_heads=1, d=64),
    "long prefixes": dict(lengths=[700, 500], prefix=[300, 1000], heads=2, kv_heads=1, d=128, behind=9),
    "cap": dict(lengths=[300, 200], cap=20.0, heads=2, kv_heads=1, d=64, size=2.5),
    "small cap": dict(lengths=[300], cap=0.5, heads=2, kv_heads=1, d=128),
    "large cap": dict(lengths=[300], cap=1e5, heads=2, kv_heads=1, d=64),
    "distance": dict(lengths=[600, 33], alibi=True, heads=4, kv_heads=2, d=64),
    "distance both ways": dict(lengths=[400], alibi=True, causal=False, heads=4, kv_heads=2, d=128),
    "everything": dict(lengths=[500, 130, 7], before=5, behind=70, prefix=[200, 0, 7], cap=10.0, alibi=True, heads=6, kv_heads=2, d=72, stacked=False),
    "separate tensors": dict(lengths=[300], heads=3, kv_heads=3, d=64, stacked=False),
    "own scale": dict(lengths=[300], heads=2, kv_heads=1, d=64, scale=0.02),
    "sharp scores": dict(lengths=[400], heads=2, kv_heads=1, d=64, size=5.0),
    "flat scores": dict(lengths=[900], heads=2, kv_heads=1, d=64, size=0.05),
    # more documents and more tiles than the plan's block has threads and registers for
    "1500 documents": dict(lengths=[i % 3 for i in range(1500)], heads=2, kv_heads=1, d=16, behind=3),
    "4500 documents": dict(lengths=[1 + i % 3 for i in range(4500)], heads=2, kv_heads=2, d=8, causal=False, before=2),
    # enough heads for work items of 256 queries, and for a key tile's heads to be dealt in twos
    "many heads": dict(lengths=[700, 1000, 257], heads=28, kv_heads=4, d=64, before=11),
    "many heads 128": dict(lengths=[513, 900], heads=40, kv_heads=8, d=128, behind=5),
    "many heads, all": dict(lengths=[650, 700], heads=32, kv_heads=32, d=40, causal=False),
    "many heads, everything": dict(lengths=[900, 640, 1], prefix=[400, 0, 1], cap=15.0, alibi=True, heads=27, kv_heads=9, d=72, before=2, behind=3),
    "many heads, distance": dict(lengths=[1100, 300], alibi=True, heads=32, kv_heads=8, d=64),
    "many heads, cap": dict(lengths=[1100, 300], cap=5.0, heads=32, kv_heads=8, d=64),
    "heads in twos": dict(lengths=[256] * 12 + [200] * 5 + [131], heads=28, kv_heads=4, d=16),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name):
    Attn(**CASES[name]).check()
