"""Softmax attention over packed documents in fp64, document by document and head by head, with bounds on what roundings may do.

    z_ij = cap(scale q_i k_j) - slope_h |i - j|,  cap(s) = c tanh(s / c) or s;   p_i = softmax over the keys that i sees
    o_i = sum_j p_ij v_j,   lse_i = log sum_j exp(z_ij)

Keys that i sees: those of its document; causal: only j <= i and the document's prefix.  Tokens of no document: o = 0 and no gradient."""
import numpy as np


def documents(offsets, prefix=None):
    """(start, end, end of the prefix) of every document that holds a token."""
    out = []
    for i, (s, e) in enumerate(zip(offsets[:-1], offsets[1:])):
        if e > s:
            out.append((int(s), int(e), int(s) + min(int(prefix[i]), int(e) - int(s)) if prefix is not None else int(s)))
    return out


def seen(start, end, prefix_end, causal):
    i = np.arange(start, end)
    if not causal:
        return np.ones((len(i), len(i)), dtype=bool)
    return (i[None, :] <= i[:, None]) | (i[None, :] < prefix_end)


def attention(q, k, v, offsets, *, causal=True, prefix=None, scale=None, softcap=0.0, slopes=None, do=None,
              slope_error=(0.0, 2.0 ** -18)):
    """q [tokens, heads, d], k, v [tokens, kv_heads, d].  A dict of o, lse and, with do, dq, dk, dv; each with the largest error that
    the roundings of a bf16 implementation may make (`*_bound`): every stored value once, the probabilities and their gradients once
    before they are multiplied (2^-8 of the value each), fp32 in between.  slope_error: what the cap's slope may be off by, relatively
    and absolutely."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    T, H, d = q.shape
    group = H // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    r, eps = 2.0 ** -8, 2.0 ** -12          # one rounding to bf16; what fp32 exponentials and sums may add, relatively
    out = {n: np.zeros_like(q) for n in ("o", "o_bound")}
    out["lse"], out["lse_bound"] = np.full((H, T), -np.inf), np.zeros((H, T))
    if do is not None:
        do = np.asarray(do, dtype=np.float64)
        out.update({n: np.zeros_like(q) for n in ("dq", "dq_bound")})
        out.update({n: np.zeros_like(k) for n in ("dk", "dv", "dk_bound", "dv_bound")})
    for s, e, pe in documents(offsets, prefix):
        mask, pos = seen(s, e, pe, causal), np.arange(s, e)
        for h in range(H):
            g, t = h // group, slice(s, e)
            Q, K, V = q[t, h], k[t, g], v[t, g]
            raw = scale * (Q @ K.T)
            size = scale * (np.abs(Q) @ np.abs(K).T)
            th = np.tanh(raw / softcap) if softcap else None
            z = softcap * th if softcap else raw
            if slopes is not None:
                z = z - slopes[h] * np.abs(pos[:, None] - pos[None, :])
            z = np.where(mask, z, -np.inf)
            top = z.max(1, keepdims=True)
            p = np.exp(z - top)
            total = p.sum(1, keepdims=True)
            p /= total
            lse = top[:, 0] + np.log(total[:, 0])
            o = p @ V
            spread = p @ np.abs(V)
            out["o"][t, h], out["lse"][h, t] = o, lse
            # a score's fp32 error, absolutely, is that relative error of its exponential
            zerr = (2.0 ** -21 * np.where(mask, size, 0)).max(1) + 2.0 ** -20 * (1 + np.abs(np.where(mask, z, 0)).max(1))
            out["lse_bound"][h, t] = zerr + 2.0 ** -20 * np.abs(lse)
            rel = eps + 2 * zerr[:, None]
            out["o_bound"][t, h] = ob = r * np.abs(o) + (r + rel) * spread
            if do is None:
                continue
            G = do[t, h]
            dp = G @ V.T
            delta = (G * o).sum(1, keepdims=True)
            slope = scale * (1 - th * th if softcap else 1.0)
            ds = p * (dp - delta) * slope
            lost = (np.abs(G) * ob).sum(1, keepdims=True) + 2.0 ** -18 * (np.abs(G) @ np.abs(V).T + np.abs(delta))
            lost = p * lost * slope
            if softcap:
                lost = lost + p * np.abs(dp - delta) * (slope_error[0] * slope + slope_error[1] * scale)
            ds_err = (r + rel) * np.abs(ds) + lost
            single = mask.sum(1) == 1
            ds_err[single] = 0.0                          # the gradient of a softmax over one key is zero, exactly
            out["dq"][t, h] = ds @ K
            out["dq_bound"][t, h] = r * np.abs(ds @ K) + ds_err @ np.abs(K)
            out["dk"][t, g] += ds.T @ Q
            out["dk_bound"][t, g] += ds_err.T @ np.abs(Q)
            out["dv"][t, g] += p.T @ G
            out["dv_bound"][t, g] += ((r + rel) * p).T @ np.abs(G)
    if do is not None:
        for n in ("dk", "dv"):
            out[n + "_bound"] += r * np.abs(out[n])
    return out
