"""Oracle for the row operators, numpy.  TEST INFRASTRUCTURE.

8-bit checkpoint: per row, groups of 128 columns; a = max |x|, scale = a * (1 / 127), code = rint(x * (127 * (1 / a))), each step one
binary32 operation, the scale at most MAX_SCALE (these are whole decisions of the format, so they are made in binary32 here too); everything after
the codes is float64.  A group with a < 2^-100 is zeros; one with an infinity or a NaN reads back as NaN.

Gated activation:   H = silu(G) U;  dU = dH G s,  dG = dH U s (1 + G (1 - s)),  s = 1 / (1 + exp(-G)).

Residual join:      t = h + alpha gate w_post b r_b,  y = w_pre t r_t,  r_x = (mean(x^2) + eps)^(-1/2);
its gradients are written out per row from the derivative of x r(x): d(x_i r)/dx_j = r (delta_ij - x_i x_j r^2 / n).
"""
from __future__ import annotations

import numpy as np

GROUP = 128
MAX_SCALE = np.nextafter(np.finfo(np.float32).max / np.float32(127), np.float32(0))   # the largest float whose 127-fold is finite


def q8_encode(x):
    """(codes int8, scales float32) of a float32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    ng = -(-cols // GROUP)
    codes, scales = np.zeros((rows, cols), np.int8), np.zeros((rows, ng), np.float32)
    with np.errstate(all="ignore"):
        for g in range(ng):
            part = x[:, g * GROUP:(g + 1) * GROUP]
            a = np.max(np.abs(part), axis=1)            # NaN if there is one
            bad = ~np.isfinite(a)
            live = ~bad & (a >= np.float32(2.0 ** -100))
            safe = np.where(live, a, np.float32(1))
            inv = np.float32(127) * (np.float32(1) / safe)
            k = np.rint(part * inv[:, None])
            codes[:, g * GROUP:(g + 1) * GROUP] = np.where(live[:, None], k, 0).astype(np.int8)
            scales[:, g] = np.where(bad, np.float32(np.nan), np.where(live, np.minimum(a * (np.float32(1) / np.float32(127)), MAX_SCALE), np.float32(0)))
    return codes, scales


def q8_decode(codes, scales):
    """float64 values of a checkpoint."""
    cols = codes.shape[1]
    return codes.astype(np.float64) * np.repeat(np.asarray(scales, np.float64), GROUP, axis=1)[:, :cols]


def q8_values(x):
    return q8_decode(*q8_encode(x))


def _sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def swiglu_fwd(G, U):
    G, U = np.asarray(G, np.float64), np.asarray(U, np.float64)
    return G * _sigmoid(G) * U


def swiglu_bwd(dH, G, U):
    dH, G, U = (np.asarray(a, np.float64) for a in (dH, G, U))
    s = _sigmoid(G)
    return dH * U * s * (1.0 + G * (1.0 - s)), dH * G * s


def _rstd(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)


def norm_join_fwd(h, b, w_post, gate, w_pre, alpha, eps):
    """(h_out, y, r_b, r_t); b None: the norm alone; w_post, gate may be None."""
    t = np.asarray(h, np.float64)
    r_b = None
    if b is not None:
        j = np.asarray(b, np.float64)
        if w_post is not None:
            r_b = _rstd(j, eps)
            j = j * r_b * np.asarray(w_post, np.float64)
        if gate is not None:
            j = j * np.asarray(gate, np.float64)
        t = t + alpha * j
    r_t = _rstd(t, eps)
    return t, t * r_t * np.asarray(w_pre, np.float64), r_b, r_t


def norm_join_bwd(dy, dh_next, h, b, w_post, gate, w_pre, r_b, r_t, alpha):
    """Gradients at the given (checkpointed) h and b with the given r_b, r_t:
    dict of dh, db, dw_post, dgate, dw_pre (those that apply)."""
    dy, h, w_pre = (np.asarray(a, np.float64) for a in (dy, h, w_pre))
    n = h.shape[1]
    k = np.full(n, float(alpha))
    t = h
    if b is not None:
        bh = np.asarray(b, np.float64) * (r_b if r_b is not None else 1.0)
        if w_post is not None:
            k = k * np.asarray(w_post, np.float64)
        if gate is not None:
            k = k * np.asarray(gate, np.float64)
        t = h + k * bh
    th = t * r_t
    v = dy * w_pre
    d = r_t * (v - th * (np.sum(v * th, axis=1, keepdims=True) / n))
    if dh_next is not None:
        d = d + np.asarray(dh_next, np.float64)
    out = {"dh": d, "dw_pre": np.sum(dy * th, axis=0)}
    if b is not None:
        p = k * d
        out["db"] = r_b * (p - bh * (np.sum(p * bh, axis=1, keepdims=True) / n)) if w_post is not None else p
        c = alpha * np.sum(d * bh, axis=0)
        if w_post is not None:
            out["dw_post"] = c * (np.asarray(gate, np.float64) if gate is not None else 1.0)
        if gate is not None:
            out["dgate"] = c * (np.asarray(w_post, np.float64) if w_post is not None else 1.0)
    return out
