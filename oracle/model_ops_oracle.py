"""CPU oracle for the operators between the attention layers and the loss head: the normalisation and the token embedding,
forward and backward.

TEST INFRASTRUCTURE ONLY.  Plain fp64 statements, row by row and token by token; they share no code with the CUDA path and
must never be imported by it.
"""
from __future__ import annotations

import numpy as np


def norm_stats(h, rms=False, eps=0.0):
    """Row means (zero with rms) and reciprocal standard deviations of h [T, D]."""
    h = np.asarray(h, dtype=np.float64)
    mean = np.zeros(h.shape[0]) if rms else h.sum(axis=1) / h.shape[1]
    var = ((h - mean[:, None]) ** 2).sum(axis=1) / h.shape[1]
    return mean, 1.0 / np.sqrt(var + eps)


def norm_forward(h, weight=None, bias=None, rms=False, eps=0.0):
    mean, rstd = norm_stats(h, rms, eps)
    n = (np.asarray(h, dtype=np.float64) - mean[:, None]) * rstd[:, None]
    y = n if weight is None else n * weight
    return (y if bias is None else y + bias), mean, rstd


def norm_backward(dy, h, weight, mean, rstd, dh=None, rms=False):
    """Gradients with the statistics as given: dx, dweight, dbias."""
    dy, h = np.asarray(dy, dtype=np.float64), np.asarray(h, dtype=np.float64)
    n = (h - (0.0 if rms else mean[:, None])) * rstd[:, None]
    g = dy if weight is None else dy * weight
    D = h.shape[1]
    dx = g - n * ((g * n).sum(axis=1) / D)[:, None]
    if not rms:
        dx = dx - (g.sum(axis=1) / D)[:, None]
    dx = dx * rstd[:, None]
    return (dx if dh is None else dx + dh), (dy * n).sum(axis=0), dy.sum(axis=0)


def embed_forward(table, ids, scale=1.0):
    """Row t is scale * table[ids[t]], zero where ids[t] is no row of the table."""
    V, D = table.shape
    out = np.zeros((len(ids), D))
    for t, v in enumerate(ids):
        if 0 <= v < V:
            out[t] = np.asarray(table[v], dtype=np.float64) * scale
    return out


def embed_backward(dout, ids, V, scale=1.0, start=None):
    """Row v is scale times the sum of dout over the tokens whose id is v, added to `start` if given."""
    grad = np.zeros((V, dout.shape[1])) if start is None else np.array(start, dtype=np.float64)
    for t, v in enumerate(ids):
        if 0 <= v < V:
            grad[v] += np.asarray(dout[t], dtype=np.float64) * scale
    return grad
