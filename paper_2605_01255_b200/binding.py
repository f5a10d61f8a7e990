"""ctypes binding to libacx.so: same names as the C ABI (include/acx.h), argument marshalling only.

torch supplies device memory and streams; every arithmetic step runs in the library's kernels.  The row operators and the
cross entropy check and convert their arguments in a compiled module (csrc/host_calls.cpp), the linears here.  If
the library has not been built the import of a symbol raises: there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libacx.so")

ACX_OK = 0
ACX_ERR_INVALID_ARG, ACX_ERR_UNSUPPORTED_SHAPE, ACX_ERR_ALIGNMENT = 1, 2, 3
ACX_ERR_WORKSPACE, ACX_ERR_CUDA, ACX_ERR_TIMEOUT = 4, 5, 6
ACX_ERR_SCRATCH_LIMIT = 7
ACX_BUILTIN_SCRATCH_BYTES = 16 << 20
ACX_F32, ACX_BF16 = 0, 1
ACX_OP_FWD, ACX_OP_BWD, ACX_OP_RECONSTRUCT, ACX_OP_BWD_BUILTIN_SCRATCH, ACX_OP_RSVD, ACX_OP_BIAS_GRAD = 0, 1, 2, 3, 4, 5
ACX_OP_BWD_BIAS = 6
ACX_OP_NORM_BWD, ACX_OP_CE_FWD, ACX_OP_CE_BWD = 7, 8, 9
ACX_Q8_GROUP = 128

EXPORTS = (
    "acx_workspace_bytes", "acx_linear_fwd", "acx_linear_bwd", "acx_reconstruct",
    "acx_sketch_materialize", "acx_last_device_status", "acx_kernel_launches", "acx_status_string", "acx_version",
    "acx_linear_bwd_factor_builtin_scratch", "acx_reconstruct_adamw", "acx_debug_expired_wait",
    "acx_debug_force_gemm_mode", "acx_linear_fwd_v", "acx_reconstruct_v", "acx_lowrank_adamw", "acx_rsvd_factor", "acx_linear_fwd_bias", "acx_bias_grad", "acx_linear_bwd_bias",
    "acx_rows_workspace_bytes", "acx_q8_store", "acx_q8_load", "acx_swiglu_fwd", "acx_swiglu_bwd", "acx_norm_join_fwd", "acx_norm_join_bwd",
    "acx_ce_workspace_bytes", "acx_linear_ce_fwd", "acx_linear_ce_bwd", "acx_linear_ce_bwd_loss",
)


class AcxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s" % (where, status_string(status)))


class acx_adamw_params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("step", ctypes.c_int32), ("lr", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float)]


class acx_desc(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("sketch_kind", ctypes.c_uint32),
        ("tokens", ctypes.c_int64), ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
        ("r", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("seed", ctypes.c_uint64),
    ]


class acx_rows_desc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("io_dtype", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class acx_ce_desc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("io_dtype", ctypes.c_int32), ("tokens", ctypes.c_int64), ("d", ctypes.c_int64),
                ("vocab", ctypes.c_int64), ("logit_scale", ctypes.c_float), ("reserved", ctypes.c_uint32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if libacx.so is missing (build it with paper_2605_01255_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libacx.so is not built (%s); run `python -m paper_2605_01255_b200.build`. "
                               "There is no CPU or PyTorch fallback." % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, dp = ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(acx_desc)
        L.acx_workspace_bytes.restype, L.acx_workspace_bytes.argtypes = sz, [dp, ctypes.c_int]
        L.acx_linear_fwd.restype, L.acx_linear_fwd.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, vp, sz, vp]
        L.acx_linear_bwd.restype, L.acx_linear_bwd.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.acx_linear_bwd_factor_builtin_scratch.restype = ctypes.c_int
        L.acx_linear_bwd_factor_builtin_scratch.argtypes = [dp, vp, vp, vp, vp]
        L.acx_reconstruct.restype, L.acx_reconstruct.argtypes = ctypes.c_int, [dp, vp, vp, ctypes.c_float, vp, sz, vp]
        L.acx_linear_fwd_v.restype, L.acx_linear_fwd_v.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.acx_reconstruct_v.restype, L.acx_reconstruct_v.argtypes = ctypes.c_int, [dp, vp, vp, vp, ctypes.c_float, vp, sz, vp]
        L.acx_reconstruct_adamw.restype = ctypes.c_int
        L.acx_reconstruct_adamw.argtypes = [dp, vp, vp, vp, vp, vp, ctypes.POINTER(acx_adamw_params), vp, sz, vp]
        L.acx_lowrank_adamw.restype = ctypes.c_int
        L.acx_lowrank_adamw.argtypes = [dp, vp, vp, vp, vp, vp, ctypes.POINTER(acx_adamw_params), vp, sz, vp]
        L.acx_rsvd_factor.restype, L.acx_rsvd_factor.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, sz, vp]
        L.acx_linear_fwd_bias.restype, L.acx_linear_fwd_bias.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.acx_bias_grad.restype, L.acx_bias_grad.argtypes = ctypes.c_int, [dp, vp, vp, vp, sz, vp]
        L.acx_linear_bwd_bias.restype, L.acx_linear_bwd_bias.argtypes = ctypes.c_int, [dp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        rp, i64, f32 = ctypes.POINTER(acx_rows_desc), ctypes.c_int64, ctypes.c_float
        L.acx_rows_workspace_bytes.restype, L.acx_rows_workspace_bytes.argtypes = sz, [rp, ctypes.c_int]
        L.acx_q8_store.restype, L.acx_q8_store.argtypes = ctypes.c_int, [rp, vp, i64, vp, vp, vp]
        L.acx_q8_load.restype, L.acx_q8_load.argtypes = ctypes.c_int, [rp, vp, vp, vp, i64, vp]
        L.acx_swiglu_fwd.restype, L.acx_swiglu_fwd.argtypes = ctypes.c_int, [rp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp]
        L.acx_swiglu_bwd.restype, L.acx_swiglu_bwd.argtypes = ctypes.c_int, [rp, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp]
        L.acx_norm_join_fwd.restype, L.acx_norm_join_fwd.argtypes = ctypes.c_int, [rp] + [vp] * 13 + [f32, f32, vp]
        L.acx_norm_join_bwd.restype, L.acx_norm_join_bwd.argtypes = ctypes.c_int, [rp] + [vp] * 16 + [f32, vp, sz, vp]
        cp = ctypes.POINTER(acx_ce_desc)
        L.acx_ce_workspace_bytes.restype, L.acx_ce_workspace_bytes.argtypes = sz, [cp, ctypes.c_int]
        L.acx_linear_ce_fwd.restype, L.acx_linear_ce_fwd.argtypes = ctypes.c_int, [cp] + [vp] * 8 + [sz, vp]
        L.acx_linear_ce_bwd.restype, L.acx_linear_ce_bwd.argtypes = ctypes.c_int, [cp] + [vp] * 6 + [f32, vp, vp, vp, sz, vp]
        L.acx_linear_ce_bwd_loss.restype, L.acx_linear_ce_bwd_loss.argtypes = ctypes.c_int, [cp] + [vp] * 7 + [f32, vp, vp, vp, sz, vp]
        L.acx_sketch_materialize.restype, L.acx_sketch_materialize.argtypes = ctypes.c_int, [dp, vp, vp]
        L.acx_last_device_status.restype, L.acx_last_device_status.argtypes = ctypes.c_int, [vp]
        L.acx_debug_expired_wait.restype, L.acx_debug_expired_wait.argtypes = ctypes.c_int, [ctypes.c_uint64, vp]
        L.acx_debug_force_gemm_mode.restype, L.acx_debug_force_gemm_mode.argtypes = ctypes.c_int, [ctypes.c_int]
        L.acx_status_string.restype, L.acx_status_string.argtypes = ctypes.c_char_p, [ctypes.c_int]
        L.acx_version.restype, L.acx_version.argtypes = ctypes.c_int, []
        L.acx_kernel_launches.restype, L.acx_kernel_launches.argtypes = ctypes.c_ulonglong, []
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().acx_status_string(int(status)).decode()


def acx_version() -> int:
    return lib().acx_version()


def acx_kernel_launches() -> int:
    return int(lib().acx_kernel_launches())


def make_desc(tokens: int, d_in: int, d_out: int, r: int, seed: int, dtype) -> acx_desc:
    """dtype: torch.float32 / torch.bfloat16 or "f32" / "bf16"."""
    code = {torch.float32: ACX_F32, torch.bfloat16: ACX_BF16, "f32": ACX_F32, "bf16": ACX_BF16}[dtype]
    return acx_desc(ctypes.sizeof(acx_desc), 0, tokens, d_in, d_out, r, code, seed & 0xFFFFFFFFFFFFFFFF)


def io_torch_dtype(desc: acx_desc):
    return torch.bfloat16 if desc.io_dtype == ACX_BF16 else torch.float32


def _ptr(t: Optional[torch.Tensor], shape: Tuple[int, ...], dtype, name: str):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous() or t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be a contiguous CUDA tensor of shape %s and dtype %s (got %s %s on %s)"
                         % (name, tuple(shape), dtype, tuple(t.shape), t.dtype, t.device))
    return ctypes.c_void_p(t.data_ptr())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # the handle without building a Stream object


def _stream(stream) -> ctypes.c_void_p:
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if _raw_stream is not None:
        return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(status: int, where: str):
    if status != ACX_OK:
        raise AcxError(status, where)


def acx_workspace_bytes(desc: acx_desc, op: int) -> int:
    return int(lib().acx_workspace_bytes(ctypes.byref(desc), op))


def alloc_workspace(desc: acx_desc, op: int, device="cuda") -> Optional[torch.Tensor]:
    n = acx_workspace_bytes(desc, op)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _ws(ws: Optional[torch.Tensor]):
    if ws is None:
        return None, 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor")
    return ctypes.c_void_p(ws.data_ptr()), ws.numel() * ws.element_size()


def acx_linear_fwd(desc: acx_desc, X, W, Y, XS, ws=None, stream=None) -> None:
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_linear_fwd(ctypes.byref(desc), _ptr(X, (desc.tokens, desc.d_in), dt, "X"),
                                _ptr(W, (desc.d_out, desc.d_in), dt, "W"),
                                _ptr(Y, (desc.tokens, desc.d_out), dt, "Y"),
                                _ptr(XS, (desc.tokens, desc.r), dt, "XS"), wp, wn, _stream(stream)), "acx_linear_fwd")


def acx_linear_fwd_v(desc: acx_desc, X, W, Vt, Y, XV, ws=None, stream=None) -> None:
    """Y = X W^T and XV = X V for a second factor given in memory as Vt (r x d_in)."""
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_linear_fwd_v(ctypes.byref(desc), _ptr(X, (desc.tokens, desc.d_in), dt, "X"),
                                  _ptr(W, (desc.d_out, desc.d_in), dt, "W"),
                                  _ptr(Vt, (desc.r, desc.d_in), dt, "Vt"),
                                  _ptr(Y, (desc.tokens, desc.d_out), dt, "Y"),
                                  _ptr(XV, (desc.tokens, desc.r), dt, "XV"), wp, wn, _stream(stream)), "acx_linear_fwd_v")


def acx_linear_bwd(desc: acx_desc, G_out, W, XS, dX, dW_A, ws=None, stream=None) -> None:
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_linear_bwd(ctypes.byref(desc), _ptr(G_out, (desc.tokens, desc.d_out), dt, "G_out"),
                                _ptr(W, (desc.d_out, desc.d_in), dt, "W"),
                                _ptr(XS, (desc.tokens, desc.r), dt, "XS"),
                                _ptr(dX, (desc.tokens, desc.d_in), dt, "dX"),
                                _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"), wp, wn, _stream(stream)),
           "acx_linear_bwd")


def acx_linear_bwd_factor_builtin_scratch(desc: acx_desc, G_out, XS, dW_A, stream=None) -> None:
    """dW_A = G_out^T XS (bf16 inputs) with the split-K partial sums kept in the scratch array that is
    built into the library, for callers that cannot allocate a workspace.  Calls on one device share that
    array: keep them ordered on the GPU.  Raises AcxError(ACX_ERR_SCRATCH_LIMIT) if the shape needs more
    than ACX_BUILTIN_SCRATCH_BYTES."""
    _check(lib().acx_linear_bwd_factor_builtin_scratch(
        ctypes.byref(desc), _ptr(G_out, (desc.tokens, desc.d_out), torch.bfloat16, "G_out"),
        _ptr(XS, (desc.tokens, desc.r), torch.bfloat16, "XS"),
        _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"), _stream(stream)),
        "acx_linear_bwd_factor_builtin_scratch")


def acx_reconstruct(desc: acx_desc, dW_A, dW, beta: float = 0.0, ws=None, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(lib().acx_reconstruct(ctypes.byref(desc), _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"),
                                 _ptr(dW, (desc.d_out, desc.d_in), torch.float32, "dW"),
                                 ctypes.c_float(beta), wp, wn, _stream(stream)), "acx_reconstruct")


def acx_reconstruct_v(desc: acx_desc, dW_A, Vt, dW, beta: float = 0.0, ws=None, stream=None) -> None:
    """dW = beta * dW + dW_A Vt for a second factor given in memory as Vt (r x d_in)."""
    wp, wn = _ws(ws)
    _check(lib().acx_reconstruct_v(ctypes.byref(desc), _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"),
                                   _ptr(Vt, (desc.r, desc.d_in), io_torch_dtype(desc), "Vt"),
                                   _ptr(dW, (desc.d_out, desc.d_in), torch.float32, "dW"),
                                   ctypes.c_float(beta), wp, wn, _stream(stream)), "acx_reconstruct_v")


def acx_reconstruct_adamw(desc: acx_desc, dW_A, W, m, v, W_lp=None, *, step: int, lr: float, beta1: float = 0.9,
                          beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0, ws=None, stream=None) -> None:
    """One AdamW step on fp32 master weights W (moments m, v) with the gradient dW_A S^T, which is never written out.
    W_lp (bfloat16, optional) receives the updated weights rounded for the next forward pass."""
    hp = acx_adamw_params(ctypes.sizeof(acx_adamw_params), step, lr, beta1, beta2, eps, weight_decay)
    shape = (desc.d_out, desc.d_in)
    wp, wn = _ws(ws)
    _check(lib().acx_reconstruct_adamw(ctypes.byref(desc), _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"),
                                       _ptr(W, shape, torch.float32, "W"), _ptr(m, shape, torch.float32, "m"),
                                       _ptr(v, shape, torch.float32, "v"), _ptr(W_lp, shape, torch.bfloat16, "W_lp"),
                                       ctypes.byref(hp), wp, wn, _stream(stream)), "acx_reconstruct_adamw")


def acx_lowrank_adamw(desc: acx_desc, dW_A, m_A, v_A, W, Vt=None, *, step: int, lr: float, beta1: float = 0.9,
                      beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0, ws=None, stream=None) -> None:
    """One GaLore-style step: Adam moments m_A, v_A kept for the gradient factor dW_A (d_out x r), the normalised step
    projected back through V^T (Vt, or the seeded sketch when Vt is None) into the fp32 weights W."""
    hp = acx_adamw_params(ctypes.sizeof(acx_adamw_params), step, lr, beta1, beta2, eps, weight_decay)
    fshape = (desc.d_out, desc.r)
    wp, wn = _ws(ws)
    _check(lib().acx_lowrank_adamw(ctypes.byref(desc), _ptr(dW_A, fshape, torch.float32, "dW_A"),
                                   _ptr(m_A, fshape, torch.float32, "m_A"), _ptr(v_A, fshape, torch.float32, "v_A"),
                                   _ptr(Vt, (desc.r, desc.d_in), torch.bfloat16, "Vt"),
                                   _ptr(W, (desc.d_out, desc.d_in), torch.float32, "W"),
                                   ctypes.byref(hp), wp, wn, _stream(stream)), "acx_lowrank_adamw")


def acx_linear_fwd_bias(desc: acx_desc, X, W, bias, Y, XS, ws=None, stream=None) -> None:
    """Y = X W^T + bias (one bias vector of length d_out, bf16) and XS = X S."""
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_linear_fwd_bias(ctypes.byref(desc), _ptr(X, (desc.tokens, desc.d_in), dt, "X"),
                                     _ptr(W, (desc.d_out, desc.d_in), dt, "W"), _ptr(bias, (desc.d_out,), dt, "bias"),
                                     _ptr(Y, (desc.tokens, desc.d_out), dt, "Y"),
                                     _ptr(XS, (desc.tokens, desc.r), dt, "XS"), wp, wn, _stream(stream)), "acx_linear_fwd_bias")


def acx_bias_grad(desc: acx_desc, G_out, db, ws=None, stream=None) -> None:
    """db = column sums of G_out over the tokens (fp32)."""
    wp, wn = _ws(ws)
    _check(lib().acx_bias_grad(ctypes.byref(desc), _ptr(G_out, (desc.tokens, desc.d_out), io_torch_dtype(desc), "G_out"),
                               _ptr(db, (desc.d_out,), torch.float32, "db"), wp, wn, _stream(stream)), "acx_bias_grad")


def acx_linear_bwd_bias(desc: acx_desc, G_out, W, XS, dX, dW_A, db, ws=None, stream=None) -> None:
    """acx_linear_bwd plus the bias gradient db (column sums of G_out), summed inside the gradient-factor kernel."""
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_linear_bwd_bias(ctypes.byref(desc), _ptr(G_out, (desc.tokens, desc.d_out), dt, "G_out"),
                                     _ptr(W, (desc.d_out, desc.d_in), dt, "W"), _ptr(XS, (desc.tokens, desc.r), dt, "XS"),
                                     _ptr(dX, (desc.tokens, desc.d_in), dt, "dX"),
                                     _ptr(dW_A, (desc.d_out, desc.r), torch.float32, "dW_A"),
                                     _ptr(db, (desc.d_out,), torch.float32, "db"), wp, wn, _stream(stream)), "acx_linear_bwd_bias")


def acx_rsvd_factor(desc: acx_desc, X, U, Vt, ws=None, stream=None) -> None:
    """Vt = (U^T U)^-1 U^T X (r x d_in): the second factor of the randomized-SVD compressor for the stored sketch U = X S."""
    dt = io_torch_dtype(desc)
    wp, wn = _ws(ws)
    _check(lib().acx_rsvd_factor(ctypes.byref(desc), _ptr(X, (desc.tokens, desc.d_in), dt, "X"),
                                 _ptr(U, (desc.tokens, desc.r), dt, "U"), _ptr(Vt, (desc.r, desc.d_in), dt, "Vt"),
                                 wp, wn, _stream(stream)), "acx_rsvd_factor")


def acx_sketch_materialize(desc: acx_desc, S_out, stream=None) -> None:
    _check(lib().acx_sketch_materialize(ctypes.byref(desc), _ptr(S_out, (desc.d_in, desc.r), io_torch_dtype(desc), "S_out"),
                                        _stream(stream)), "acx_sketch_materialize")


def acx_debug_expired_wait(limit_ns: int, stream=None) -> None:
    """Launches a warp whose bounded wait runs out after limit_ns (test of the time-out reporting path)."""
    _check(lib().acx_debug_expired_wait(int(limit_ns), _stream(stream)), "acx_debug_expired_wait")


def acx_debug_force_gemm_mode(mode: int) -> None:
    """Test/debug: 0 = the cost models pick the tile shape of the forward and dX, 1..4 = force a GEMM mode."""
    _check(lib().acx_debug_force_gemm_mode(int(mode)), "acx_debug_force_gemm_mode")


def acx_last_device_status(stream=None) -> int:
    return int(lib().acx_last_device_status(_stream(stream)))


# ---- what stands between the linears: 8-bit checkpoints, gated activation, residual join -------------------------------
def make_rows_desc(rows: int, cols: int, dtype) -> acx_rows_desc:
    """dtype: torch.float32 / torch.bfloat16 or "f32" / "bf16"."""
    code = {torch.float32: ACX_F32, torch.bfloat16: ACX_BF16, "f32": ACX_F32, "bf16": ACX_BF16}[dtype]
    return acx_rows_desc(ctypes.sizeof(acx_rows_desc), code, rows, cols)


def acx_rows_workspace_bytes(desc: acx_rows_desc, op: int) -> int:
    return int(lib().acx_rows_workspace_bytes(ctypes.byref(desc), op))


def alloc_rows_workspace(desc: acx_rows_desc, op: int, device="cuda") -> Optional[torch.Tensor]:
    n = acx_rows_workspace_bytes(desc, op)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def q8_empty(rows: int, cols: int, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """Room for the 8-bit checkpoint of a rows x cols matrix: codes (int8) and scales (fp32)."""
    return (torch.empty(rows, cols, dtype=torch.int8, device=device),
            torch.empty(rows, -(-cols // ACX_Q8_GROUP), dtype=torch.float32, device=device))


_host = None


def _calls():
    """The compiled argument checks of the operators below (csrc/host_calls.cpp), bound to the library's entry points: a small call
    costs its launch and little more.  Raises if the module has not been built."""
    global _host
    if _host is None:
        L = lib()
        try:
            from . import _acx_host
        except ImportError as e:
            raise RuntimeError("_acx_host.so is not built for this torch; run `python -m paper_2605_01255_b200.build`") from e
        _acx_host.bind(tuple(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in (
            "acx_q8_store", "acx_q8_load", "acx_swiglu_fwd", "acx_swiglu_bwd", "acx_norm_join_fwd", "acx_norm_join_bwd",
            "acx_linear_ce_fwd", "acx_linear_ce_bwd_loss")))
        _host = _acx_host
    return _host


def acx_q8_store(desc: acx_rows_desc, X, codes, scales, stream=None) -> None:
    """Codes and scales of X (rows x cols; its rows may be strided)."""
    _check((_host or _calls()).q8_store(desc, X, codes, scales, stream), "acx_q8_store")


def acx_q8_load(desc: acx_rows_desc, codes, scales, X, stream=None) -> None:
    """The values of an 8-bit checkpoint into X (rows x cols; its rows may be strided)."""
    _check((_host or _calls()).q8_load(desc, codes, scales, X, stream), "acx_q8_load")


def acx_swiglu_fwd(desc: acx_rows_desc, G, U, H, Gq=None, Gs=None, Uq=None, Us=None, stream=None) -> None:
    """H = silu(G) * U; with Gq, Gs, Uq, Us also the 8-bit checkpoints of G and U."""
    _check((_host or _calls()).swiglu_fwd(desc, G, U, H, Gq, Gs, Uq, Us, stream), "acx_swiglu_fwd")


def acx_swiglu_bwd(desc: acx_rows_desc, dH, Gq, Gs, Uq, Us, dG, dU, stream=None) -> None:
    """dG, dU of H = silu(G) * U at the checkpointed G and U."""
    _check((_host or _calls()).swiglu_bwd(desc, dH, Gq, Gs, Uq, Us, dG, dU, stream), "acx_swiglu_bwd")


def acx_norm_join_fwd(desc: acx_rows_desc, h, b, w_post, gate, w_pre, h_out, y, Hq=None, Hs=None, Bq=None, Bs=None, rstd_post=None,
                      rstd_pre=None, *, eps: float = 1e-5, alpha: float = 1.0, stream=None) -> None:
    """h_out = h + alpha * gate * RMSNorm(b) * w_post and y = RMSNorm(h_out) * w_pre; b, w_post, gate may be None (see acx.h)."""
    _check((_host or _calls()).norm_join_fwd(desc, h, b, w_post, gate, w_pre, h_out, y, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, eps, alpha,
                                             stream), "acx_norm_join_fwd")


def acx_norm_join_bwd(desc: acx_rows_desc, dy, dh_next, w_post, gate, w_pre, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, dh, db, dw_post, dgate,
                      dw_pre, *, alpha: float = 1.0, ws=None, stream=None) -> None:
    """Gradients of acx_norm_join_fwd at its checkpoints; ws: alloc_rows_workspace(desc, ACX_OP_NORM_BWD)."""
    _check((_host or _calls()).norm_join_bwd(desc, dy, dh_next, w_post, gate, w_pre, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, dh, db, dw_post,
                                             dgate, dw_pre, alpha, ws, stream), "acx_norm_join_bwd")


# ---- softmax cross entropy over a vocabulary ----------------------------------------------------------------------------
def make_ce_desc(tokens: int, d: int, vocab: int, logit_scale: float = 1.0) -> acx_ce_desc:
    return acx_ce_desc(ctypes.sizeof(acx_ce_desc), ACX_BF16, tokens, d, vocab, logit_scale, 0)


def acx_ce_workspace_bytes(desc: acx_ce_desc, op: int) -> int:
    return int(lib().acx_ce_workspace_bytes(ctypes.byref(desc), op))


def alloc_ce_workspace(desc: acx_ce_desc, op: int, device="cuda") -> Optional[torch.Tensor]:
    n = acx_ce_workspace_bytes(desc, op)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def acx_linear_ce_fwd(desc: acx_ce_desc, X, W, targets, loss, lse, total=None, weight=None, ws=None, stream=None) -> None:
    """Per-token cross entropy of logit_scale * X W^T at `targets` (int64; outside [0, vocab): not trained on), its log-sum-exp,
    and total = (sum of weight * loss, sum of weight); ws: alloc_ce_workspace(desc, ACX_OP_CE_FWD)."""
    _check((_host or _calls()).linear_ce_fwd(desc, X, W, targets, weight, loss, lse, total, ws, stream), "acx_linear_ce_fwd")


def acx_linear_ce_bwd(desc: acx_ce_desc, X, W, targets, lse, dX, dW, *, loss=None, weight=None, denom=None, scale: float = 1.0, ws=None,
                      stream=None) -> None:
    """Gradients of scale * sum(weight * loss) / denom (denom: one fp32 number on the device, such as total[1:]); dX or dW may be
    None; loss: the forward's, so that the gradients of almost certain tokens keep their digits (see acx.h); ws:
    alloc_ce_workspace(desc, ACX_OP_CE_BWD)."""
    _check((_host or _calls()).linear_ce_bwd(desc, X, W, targets, weight, lse, loss, denom, scale, dX, dW, ws, stream), "acx_linear_ce_bwd")
