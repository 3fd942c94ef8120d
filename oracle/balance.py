"""Oracle of a router's counts, balance loss and its gradient over packed sequences, in fp64.

Pinned by loops over tokens and by differences."""
from __future__ import annotations

import numpy as np

from .gate import scores

__all__ = ["shares", "loss", "backward"]


def shares(logits, kind):
    s = scores(logits, kind)
    total = s.sum(1, keepdims=True)
    return s / np.where(total == 0, 1.0, total)


def loss(logits, idx, starts, kind, alpha):
    """counts [n][E], mean shares [n][E], loss [n]; slots outside [0, E) are absent."""
    p, E, k = shares(logits, kind), np.shape(logits)[1], np.shape(idx)[1]
    n = len(starts) - 1
    counts, mean, out = np.zeros((n, E), dtype=np.int64), np.zeros((n, E)), np.zeros(n)
    for s in range(n):
        a, b = starts[s], starts[s + 1]
        if b <= a:
            continue
        e = np.asarray(idx[a:b]).ravel()
        counts[s] = np.bincount(e[(e >= 0) & (e < E)], minlength=E)
        mean[s] = p[a:b].mean(0)
        out[s] = alpha * E * (counts[s] / (k * (b - a)) * mean[s]).sum()
    return counts, mean, out


def backward(logits, counts, k, starts, kind, alpha, d_loss):
    """(gradient [T][E], magnitude of its terms); rows outside every sequence are NaN."""
    l = np.asarray(logits, dtype=np.float64)
    p, rest = shares(l, kind), scores(-l, "sigmoid")
    E = l.shape[1]
    grad, mag = np.full(l.shape, np.nan), np.full(l.shape, np.nan)
    for s in range(len(starts) - 1):
        a, b = starts[s], starts[s + 1]
        if b <= a:
            continue
        c = alpha * E * counts[s] / (k * (b - a)) * d_loss[s] / (b - a)
        P = p[a:b]
        grad[a:b] = P * (c - (P * c).sum(1, keepdims=True))
        mag[a:b] = P * (np.abs(c) + (P * np.abs(c)).sum(1, keepdims=True))
        if kind == "sigmoid":
            grad[a:b] *= rest[a:b]
            mag[a:b] *= rest[a:b]
    return grad, mag
