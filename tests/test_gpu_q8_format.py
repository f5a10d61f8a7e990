"""The 8-bit format, bit for bit, where its roundings show: values half way between two codes, of which bfloat16 has many, and scales
in every binade.  Two further statements of it beside the oracle's: the plain form that the operator is measured against, as torch
evaluates it on the GPU, and the header's formulas one operation at a time."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2605_01255_b200 import binding as B

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("operators", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py"))
operators = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(operators)


def _inputs(dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(4096, 256, generator=g, device="cuda")
    x[1024:2048] *= torch.exp2(torch.randint(-90, 100, (1024, 1), generator=g, device="cuda").float())
    # a and a * (k + 1/2) / 127 for every code, in as many rows as there are magnitudes of a
    a = 1 + torch.rand(2048, 1, generator=g, device="cuda")
    k = torch.arange(127, device="cuda").float()
    x[2048:, :128] = torch.cat([a, a * (k + 0.5) / 127 * torch.where(k % 3 == 0, -1.0, 1.0)], 1)
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[3000:, 1] = x[3000:, 0] / 2          # 63.5 steps exactly
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_and_scales(dtype):
    x = _inputs(dtype)
    d = B.make_rows_desc(*x.shape, dtype)
    codes, scales = B.q8_empty(*x.shape)
    B.acx_q8_store(d, x, codes, scales)
    wide = x.float().view(x.shape[0], 2, 128)
    a = wide.abs().amax(-1)
    reciprocal = torch.reciprocal(a)
    inv = reciprocal * 127.0
    assert torch.equal(scales, a * torch.tensor(1.0 / 127.0, dtype=torch.float32, device="cuda"))
    want = torch.round(wide * inv[..., None]).view(x.shape)
    assert torch.equal(codes.float(), want)
    c, s = R.q8_encode(x.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scales.cpu().numpy(), s)
    # the values the plain form gives are those that are read back
    back = torch.empty(x.shape, device="cuda")
    B.acx_q8_load(B.make_rows_desc(*x.shape, "f32"), codes, scales, back)
    assert torch.equal(back, operators._q8(x.float()))
    # a code is one of the two next to the quotient in real numbers, half a step of it away at most
    exact = wide.double() * (127.0 / a.double())[..., None]
    assert bool(((codes.view(wide.shape).double() - exact).abs() <= 0.5 + 127 * 2.0 ** -22).all())
