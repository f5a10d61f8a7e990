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


@pytest.mark.parametrize("d_in,r", [(136, 32), (264, 32), (896, 64)])
def test_weight_of_a_factor_is_what_its_gradient_has_on_average(d_in, r):
    """A = dW S: ||A S^T||^2 over ||A||^2, over forty sketches.  For one row of dW and y = S^T x it is |y|^2 + chi^2 (d_in - 1 degrees) / r:
    relative deviation sqrt(2 (d_in + r - 1)) / (d_in + r + 1), about sqrt(2 / (d_in + r)); four of them over sqrt(40)."""
    dW = np.random.default_rng(0).normal(size=(5, d_in))
    whole = factors = 0.0
    for seed in range(40):
        S = sk.sketch_for_dtype(seed, d_in, r, "bf16")
        A = dW @ S
        whole, factors = whole + ((A @ S.T) ** 2).sum(), factors + (A ** 2).sum()
    assert abs(whole / factors / B.grad_factor_weight(d_in, r) - 1) <= 4 * (2 / (d_in + r) / 40) ** 0.5


def test_the_step_counts_its_factors_so(monkeypatch):
    lists = []
    monkeypatch.setattr(B, "make_grad_list", lambda tensors, weights: lists.append((tensors, weights)))
    monkeypatch.setattr(B, "alloc_grad_workspace", lambda grads: None)
    s = M.Sizes(tokens=32, d=64, inter=128, vocab=100, layers=2, r=16, heads=2, kv_heads=1, head_dim=24, max_norm=1.0)
    model = M.MlpLm(s, device="cpu")
    (tensors, weights), = lists
    of = {t.data_ptr(): w for t, w in zip(tensors, weights)}
    for l in range(s.layers):
        for k, d_in in (("gu", 64), ("dn", 128), ("qkv", 64), ("o", 48)):
            assert of.pop(model.factors[l][k].data_ptr()) == (d_in + 17) / 16
    assert set(of.values()) == {1.0} and len(of) == sum(len(t) for t in model.grads.values())


@pytest.mark.parametrize("norm,f,steps", [(0.5, 1.0, 1), (4.0, 0.25, 1), (float("inf"), 1e-40, 1), (float("inf"), 1.0, 0), (float("nan"), 1.0, 0)])
def test_a_step_whose_norm_is_no_number_is_left_out(monkeypatch, norm, f, steps):
    """(a norm beyond fp32 reads as infinity, but has a factor: those gradients are clipped like others)"""
    monkeypatch.setattr(B, "make_grad_list", lambda tensors, weights: None)
    monkeypatch.setattr(B, "alloc_grad_workspace", lambda grads: None)
    model = M.MlpLm(M.Sizes(tokens=32, d=64, inter=128, vocab=100, layers=2, r=16, max_norm=1.0), device="cpu")
    for name in ("acx_norm_join_fwd", "acx_linear_fwd", "acx_swiglu_fwd", "acx_linear_ce_fwd", "acx_linear_ce_bwd", "acx_norm_join_bwd",
                 "acx_linear_bwd", "acx_swiglu_bwd"):
        monkeypatch.setattr(B, name, lambda *a, **k: None)
    monkeypatch.setattr(B, "acx_grad_clip", lambda grads, max_norm, total, ws: total.copy_(torch.tensor([norm, f])))
    updates = []
    monkeypatch.setattr(B, "acx_reconstruct_adamw", lambda *a, step, **k: updates.append(step))
    model.forward(*M.synthetic_batch(model.s, device="cpu"))
    model.backward()
    assert not updates and model.step_no == 0
    model.backward(lr=1e-3)
    assert updates == steps * 4 * [1] and model.step_no == steps


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


@pytest.mark.parametrize("scale,cap,ok", [(0.125, 50.0, True), (0.125, 1e5, True), (2.0 ** 104, 0.0, True), (2.0 ** 105, 0.0, False), (2.0 ** 127, 0.0, False),
                                          (3e38, 0.0, False), (0.125, 2.0 ** 104, True), (0.125, 2.0 ** 105, False), (0.125, 2.4e38, False),
                                          (1.0, 2.0 ** -104, True), (1.0, 2.0 ** -105, False), (1e3, 1e-36, False), (1.0, 1e-45, False)])
def test_scales_and_caps_beyond_what_fp32_holds(scale, cap, ok):
    """The kernels take scale log2(e), cap log2(e) and 2^7 scale / cap, and scale times gradients: each has to be a number."""
    d = B.make_attn_desc(256, 4, 2, 64, scale=scale, softcap=cap)
    assert (B.acx_attn_workspace_bytes(d, B.ACX_OP_ATTN_PLAN) > 0) == ok
    if not ok:
        p = ctypes.c_void_p
        assert B.lib().acx_attn_plan(ctypes.byref(d), p(P), None, p(P), 1 << 30, None) == B.ACX_ERR_INVALID_ARG
