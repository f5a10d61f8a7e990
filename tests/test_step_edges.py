"""What a training step around its linears is told: the weight of a factor in a norm, descriptors that no list or batch has, and steps that
are left out.  No GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import sketch as sk
from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import build as acx_build
from paper_2605_01255_b200 import mlp_lm as M

P = 1 << 20      # an aligned address that no refused call reads


@pytest.fixture(scope="module", autouse=True)
def built():
    acx_build.build()


def test_clipping_without_tensors_has_no_chunks():
    """A descriptor that no list has: its chunks would be read from a plan that nothing asked for."""
    d = B.acx_grad_desc(ctypes.sizeof(B.acx_grad_desc), 0, 0, 5)
    L, p = B.lib(), ctypes.c_void_p
    need = L.acx_grad_workspace_bytes(ctypes.byref(B.acx_grad_desc(ctypes.sizeof(B.acx_grad_desc), 0, 0, 0)), B.ACX_OP_GRAD_CLIP)
    assert need > 0
    for plan, room in ((None, 0), (P, 0), (P, 1 << 30)):
        assert L.acx_grad_clip(ctypes.byref(d), p(plan), room, 1.0, p(P), p(P), need, None) == B.ACX_ERR_INVALID_ARG
    assert L.acx_grad_plan(ctypes.byref(d), None, p(P), 1 << 30, None) == B.ACX_ERR_INVALID_ARG
    for op in (B.ACX_OP_GRAD_PLAN, B.ACX_OP_GRAD_CLIP):
        assert L.acx_grad_workspace_bytes(ctypes.byref(d), op) == 0
