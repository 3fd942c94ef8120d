"""Oracle of the routing gates (softmax or sigmoid scores, balance bias, groups, top-k, renormalized
and scaled weights) and of the weights' gradient in the logits, in fp64, token by token.

Pinned by brute force over all selections and by differences of the weights."""
from __future__ import annotations

import numpy as np

__all__ = ["scores", "select", "weights", "route", "backward"]


def scores(logits, kind):
    """fp64 scores [T][E]; a masked expert (-inf) has 0."""
    l = np.asarray(logits, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "sigmoid":
            s = 1.0 / (1.0 + np.exp(-l))
        else:
            m = np.max(np.where(np.isnan(l), -np.inf, l), axis=1, keepdims=True)
            e = np.exp(l - np.where(np.isfinite(m), m, 0.0))
            total = e.sum(1, keepdims=True)
            s = e / np.where(total == 0, 1.0, total)
    return np.where(l == -np.inf, 0.0, s)


def select(logits, k, kind, n_group=1, topk_group=1, top2=False, bias=None):
    """Indices [T][k]: ordered by (not masked, biased score) within the kept groups, ties to the lower."""
    l = np.asarray(logits, dtype=np.float64)
    T, E = l.shape
    s = scores(l, kind)
    by_logit = bias is None and (n_group == 1 or not top2)
    key = l.copy() if by_logit else s + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
    masked = (l == -np.inf) | np.isnan(key)
    out = np.zeros((T, k), dtype=np.int32)
    size = E // n_group
    for t in range(T):
        order = sorted(range(E), key=lambda e: (masked[t, e], 0.0 if masked[t, e] else -key[t, e], e))
        ranked = []
        for g in range(n_group):
            live = [key[t, e] for e in order if e // size == g and not masked[t, e]]
            total = sum(live[:2]) if top2 else (live[0] if live else 0.0)
            ranked.append((not live, -total if live else 0.0, g))
        kept = {g for _, _, g in sorted(ranked)[:topk_group]}
        out[t] = [e for e in order if e // size in kept][:k]
    return out


def weights(logits, idx, kind, renorm=False, scale=1.0):
    s = np.take_along_axis(scores(logits, kind), np.asarray(idx, dtype=np.int64), 1)
    if renorm:
        total = s.sum(1, keepdims=True)
        s = np.where(total == 0, 0.0, s / np.where(total == 0, 1.0, total))
    return s * scale


def route(logits, k, kind, n_group=1, topk_group=1, top2=False, bias=None, renorm=False, scale=1.0):
    idx = select(logits, k, kind, n_group, topk_group, top2, bias)
    return idx, weights(logits, idx, kind, renorm, scale)


def backward(logits, idx, d_w, kind, renorm=False, scale=1.0):
    """(gradient, magnitude): dL/dlogits for dL/dw = d_w, and the sum of the magnitudes of the terms that
    each element is made of (what rounding errors are relative to). Slots with an index outside [0, E)
    count as absent."""
    l = np.asarray(logits, dtype=np.float64)
    T, E = l.shape
    s, rest = scores(l, kind), scores(-l, "sigmoid")     # rest: 1 - sigmoid, near 1 too
    grad, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        slots = [(int(e), float(g) * scale) for e, g in zip(idx[t], d_w[t]) if 0 <= e < E]
        S = sum(s[t, e] for e, _ in slots)
        dot = sum(g * s[t, e] for e, g in slots)
        adot = sum(abs(g) * s[t, e] for e, g in slots)
        terms = []
        for e, g in slots:
            if renorm:
                terms.append((e, 0.0, 0.0) if S == 0 else (e, (g - dot / S) / S, (abs(g) + adot / S) / S))
            else:
                terms.append((e, g, abs(g)))
        if kind == "sigmoid":
            for e, d, a in terms:
                grad[t, e] += d * s[t, e] * rest[t, e]
                mag[t, e] += a * s[t, e] * rest[t, e]
        else:
            shared = 0.0 if renorm else sum(d * s[t, e] for e, d, _ in terms)
            grad[t] -= s[t] * shared
            mag[t] += s[t] * (0.0 if renorm else sum(a * s[t, e] for e, _, a in terms))
            for e, d, a in terms:
                grad[t, e] += s[t, e] * d
                mag[t, e] += s[t, e] * a
    return grad, mag
