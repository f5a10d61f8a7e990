"""Oracle for the softmax cross entropy over a vocabulary, float64 numpy.  TEST INFRASTRUCTURE.

    L = c X W^T (c: the logits' scale),   lse_t = log sum_v exp(L_tv),   loss_t = lse_t - L_ty  (0 for a token whose target
    is outside the vocabulary),   total = (sum of w loss, sum of w) over the other tokens,
    D = w (softmax(L) - onehot),   dX = f D W,   dW = f D^T X,   f = scale c / denom  (0 where denom <= 0).
"""
from __future__ import annotations

import numpy as np


def logits(X, W, logit_scale=1.0):
    return logit_scale * (np.asarray(X, np.float64) @ np.asarray(W, np.float64).T)


def ce_fwd(X, W, targets, weight=None, logit_scale=1.0):
    """(loss, lse, total)."""
    L = logits(X, W, logit_scale)
    V = L.shape[1]
    y = np.asarray(targets)
    trained = (y >= 0) & (y < V)
    top = L.max(1)
    lse = top + np.log(np.exp(L - top[:, None]).sum(1))
    loss = np.where(trained, lse - L[np.arange(len(y)), np.where(trained, y, 0)], 0.0)
    w = np.where(trained, 1.0 if weight is None else np.asarray(weight, np.float64), 0.0)
    return loss, lse, np.array([np.sum(w * loss), np.sum(w)])


def ce_dlogits(X, W, targets, weight=None, logit_scale=1.0):
    """D, the gradient of sum w loss with respect to the logits."""
    L = logits(X, W, logit_scale)
    V = L.shape[1]
    y = np.asarray(targets)
    trained = (y >= 0) & (y < V)
    P = np.exp(L - L.max(1, keepdims=True))
    P /= P.sum(1, keepdims=True)
    P[np.nonzero(trained)[0], y[trained]] -= 1.0
    w = np.where(trained, 1.0 if weight is None else np.asarray(weight, np.float64), 0.0)
    return P * w[:, None]


def ce_bwd(X, W, targets, weight=None, logit_scale=1.0, denom=None, scale=1.0):
    """(dX, dW) of scale * sum(w loss) / denom."""
    D = ce_dlogits(X, W, targets, weight, logit_scale)
    den = 1.0 if denom is None else float(denom)
    f = scale * logit_scale / den if den > 0 else 0.0
    return f * (D @ np.asarray(W, np.float64)), f * (D.T @ np.asarray(X, np.float64))
