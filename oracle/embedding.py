"""Embedding rows, the table's gradient and the clipping of gradients in fp64."""
import numpy as np


def lookup(ids, E, scale=1.0):
    ids, E = np.asarray(ids), np.asarray(E, dtype=np.float64)
    Y = np.zeros((len(ids), E.shape[1]))
    inside = (ids >= 0) & (ids < len(E))
    Y[inside] = scale * E[ids[inside]]
    return Y


def table_gradient(ids, dY, vocab, scale=1.0, dE=None, beta=0.0):
    """beta * dE + scale * sum of dY over each word's tokens, and the sum of the magnitudes that went into every element."""
    ids, dY = np.asarray(ids), np.asarray(dY, dtype=np.float64)
    out = np.zeros((vocab, dY.shape[1])) if dE is None or beta == 0.0 else beta * np.asarray(dE, dtype=np.float64)
    size = np.abs(out)
    inside = (ids >= 0) & (ids < vocab)
    np.add.at(out, ids[inside], scale * dY[inside])
    np.add.at(size, ids[inside], np.abs(scale * dY[inside]))
    return out, size


def clip(grads, max_norm, weights=None):
    """(norm, factor, clipped gradients)."""
    grads = [np.asarray(g, dtype=np.float64) for g in grads]
    weights = [1.0] * len(grads) if weights is None else weights
    norm = float(np.sqrt(sum(w * np.square(g).sum() for g, w in zip(grads, weights))))
    f = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, f, [g * f for g in grads]
