"""Run one call of the library a few times on random inputs: the command to profile a single kernel.

    python -m paper_2605_01255_b200.run_op {fwd,fwd_nows,fwd_plain,fwd_v,dx,factor,reconstruct,reconstruct_v,adamw,lowrank_adamw,rsvd,factor_bias,q8,swiglu,norm_join,linear_ce} tokens,d_in,d_out,r [launches] [f32|bf16]

`fwd_nows` is the forward without a workspace (the sketch generated inside the GEMM), `fwd_plain` the forward of a linear
whose input's factor another linear stores (XS = NULL); `dx` and `factor` are acx_linear_bwd with the other output left out.
`q8` (store, then load) and `norm_join` work on tokens x d_in, `swiglu` on tokens x d_out, `linear_ce` takes d = d_in and a
vocabulary of d_out (any number); those four run forward and backward and do not read r.  Prints "ok" after checking the
device status word.  Inputs come from torch.randn on the device (values do not matter for a profile).
"""
from __future__ import annotations

import sys

import torch

from . import binding as B


def _q8(m, d_in, d_out, tdt):
    d, X, q = B.make_rows_desc(m, d_in, tdt), torch.randn(m, d_in, device="cuda").to(tdt), B.q8_empty(m, d_in)
    Y = torch.empty_like(X)

    def run():
        B.acx_q8_store(d, X, *q)
        B.acx_q8_load(d, *q, Y)
    return run


def _swiglu(m, d_in, d_out, tdt):
    d = B.make_rows_desc(m, d_out, tdt)
    G, U, dH = (torch.randn(m, d_out, device="cuda").to(tdt) for _ in range(3))
    H, dG, dU = (torch.empty_like(G) for _ in range(3))
    q = B.q8_empty(m, d_out) + B.q8_empty(m, d_out)

    def run():
        B.acx_swiglu_fwd(d, G, U, H, *q)
        B.acx_swiglu_bwd(d, dH, *q, dG, dU)
    return run


def _norm_join(m, d_in, d_out, tdt):
    d = B.make_rows_desc(m, d_in, tdt)
    h, b, dy, dn = (torch.randn(m, d_in, device="cuda").to(tdt) for _ in range(4))
    w = torch.ones(d_in, device="cuda").to(tdt)
    h_out, y, dh, db = (torch.empty_like(h) for _ in range(4))
    q = B.q8_empty(m, d_in) + B.q8_empty(m, d_in)
    rstd = [torch.empty(m, device="cuda") for _ in range(2)]
    dw = [torch.empty(d_in, device="cuda") for _ in range(3)]
    ws = B.alloc_rows_workspace(d, B.ACX_OP_NORM_BWD)

    def run():
        B.acx_norm_join_fwd(d, h, b, w, w, w, h_out, y, *q, *rstd)
        B.acx_norm_join_bwd(d, dy, dn, w, w, w, *q, *rstd, dh, db, *dw, ws=ws)
    return run


def _linear_ce(m, d_in, d_out, tdt):
    d = B.make_ce_desc(m, d_in, d_out)
    X, W = torch.randn(m, d_in, device="cuda").bfloat16(), (torch.randn(d_out, d_in, device="cuda") * d_in ** -0.5).bfloat16()
    y = torch.randint(0, d_out, (m,), device="cuda")
    loss, lse, total, dX, dW = (torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty(2, device="cuda"),
                                torch.empty_like(X), torch.empty_like(W))
    ws = B.alloc_ce_workspace(d, B.ACX_OP_CE_BWD)

    def run():
        B.acx_linear_ce_fwd(d, X, W, y, loss, lse, total, ws=ws)
        B.acx_linear_ce_bwd(d, X, W, y, lse, dX, dW, loss=loss, denom=total[1:], ws=ws)
    return run


BETWEEN = {"q8": _q8, "swiglu": _swiglu, "norm_join": _norm_join, "linear_ce": _linear_ce}


def finish(run=None, launches: int = 0) -> int:
    for _ in range(launches):
        run()
    torch.cuda.synchronize()
    st = B.acx_last_device_status()
    if st != B.ACX_OK:
        raise SystemExit(B.status_string(st))
    print("ok")
    return 0


def main(argv) -> int:
    if len(argv) < 2:
        print(__doc__)
        return 2
    op = argv[0]
    m, d_in, d_out, r = (int(x) for x in argv[1].split(","))
    launches = int(argv[2]) if len(argv) > 2 else 3
    dtype = argv[3] if len(argv) > 3 else "bf16"
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dev = "cuda"
    if op in BETWEEN:
        return finish(BETWEEN[op](m, d_in, d_out, tdt), launches)
    d = B.make_desc(m, d_in, d_out, r, 0, dtype)
    X = torch.randn(m, d_in, device=dev).to(tdt)
    W = (torch.randn(d_out, d_in, device=dev) * 0.02).to(tdt)
    G = torch.randn(m, d_out, device=dev).to(tdt)
    XS = torch.randn(m, r, device=dev).to(tdt)
    Y = torch.empty(m, d_out, device=dev, dtype=tdt)
    dX = torch.empty(m, d_in, device=dev, dtype=tdt)
    A = torch.randn(d_out, r, device=dev)
    Vt = (torch.randn(r, d_in, device=dev) * d_in ** -0.5).to(tdt) if op.endswith("_v") or op == "rsvd" else None
    ws_v = B.alloc_workspace(d, B.ACX_OP_RSVD) if op == "rsvd" else None
    dW = torch.empty(d_out, d_in, device=dev)
    mom = torch.zeros(d_out, d_in, device=dev) if op == "adamw" else None
    var = torch.zeros(d_out, d_in, device=dev) if op == "adamw" else None
    W_lp = torch.empty(d_out, d_in, device=dev, dtype=torch.bfloat16) if op == "adamw" else None
    mA, vA = torch.zeros(d_out, r, device=dev), torch.zeros(d_out, r, device=dev)
    db = torch.empty(d_out, device=dev) if op == "factor_bias" else None
    ws_bb = B.alloc_workspace(d, B.ACX_OP_BWD_BIAS) if op == "factor_bias" else None
    ws_f = B.alloc_workspace(d, B.ACX_OP_FWD)
    ws_b = B.alloc_workspace(d, B.ACX_OP_BWD)
    ws_r = B.alloc_workspace(d, B.ACX_OP_RECONSTRUCT)
    for _ in range(launches):
        if op == "fwd":
            B.acx_linear_fwd(d, X, W, Y, XS, ws_f)
        elif op == "fwd_nows":
            B.acx_linear_fwd(d, X, W, Y, XS)
        elif op == "fwd_plain":
            B.acx_linear_fwd(d, X, W, Y, None)
        elif op == "fwd_v":
            B.acx_linear_fwd_v(d, X, W, Vt, Y, XS)
        elif op == "reconstruct_v":
            B.acx_reconstruct_v(d, A, Vt, dW, 0.0, ws_r)
        elif op == "dx":
            B.acx_linear_bwd(d, G, W, XS, dX, None, ws_b)
        elif op == "factor":
            B.acx_linear_bwd(d, G, W, XS, None, A, ws_b)
        elif op == "reconstruct":
            B.acx_reconstruct(d, A, dW, 0.0, ws_r)
        elif op == "factor_bias":
            B.acx_linear_bwd_bias(d, G, None, XS, None, A, db, ws_bb)
        elif op == "rsvd":
            B.acx_rsvd_factor(d, X, XS, Vt, ws_v)
        elif op == "lowrank_adamw":
            B.acx_lowrank_adamw(d, A, mA, vA, dW, step=2, lr=1e-3, weight_decay=0.01, ws=ws_r)
        elif op == "adamw":
            B.acx_reconstruct_adamw(d, A, dW, mom, var, W_lp, step=2, lr=1e-3, weight_decay=0.01, ws=ws_r)
        else:
            raise SystemExit("unknown op %r" % op)
    return finish()


if __name__ == "__main__":
    sys.exit(main(sys.argv[1:]))
