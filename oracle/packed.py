"""Oracle of attention over packed sequences with grouped heads, and of its gradients, in fp64, with bounds of
what bf16 results computed in fp32 may differ by, each element at worst and many in the 2-norm.

Pinned by explicit loops and by differences."""
from __future__ import annotations

import math

import numpy as np

__all__ = ["attention", "gradients", "deviations", "U"]

U = 2.0 ** -8                 # half a step of bf16, relative
E = 2.0 ** -24                # of fp32


def _visible(n, m, causal):
    i, j = np.arange(n)[:, None], np.arange(m)
    return j <= i + m - n if causal else np.ones((n, m), dtype=bool)


def _head(q, k, v, scale, causal):
    """One head of one sequence: P, o, lse, and the bound of a probability's relative error (a score's error, its
    rounding against the maximum, the exponential's, and the sum's, which has the same)."""
    n, m, D = len(q), len(k), q.shape[1]
    see = _visible(n, m, causal)
    s = np.where(see, scale * (q @ k.T), -np.inf)
    top = np.max(s, axis=1, initial=-np.inf, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    l = p.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(l))[:, 0] if m else np.full(n, -np.inf)
    P = p / np.where(l == 0, 1.0, l)
    mag = scale * (np.abs(q) @ np.abs(k).T)
    es = (D + 8) * E * (mag.max() if mag.size else 0.0) + 2.0 ** -18
    return P, P @ v, lse, es


def attention(q, k, v, spans, scale=None, causal=True):
    """q [Tq][H][D], k, v [Tk][Hkv][D] fp64; spans of (first query, queries, first key, keys). Returns o, its
    bound, lse [H][Tq] and its bound; rows outside every span are NaN."""
    H, D = q.shape[1:]
    G = H // k.shape[1]
    scale = scale or 1.0 / math.sqrt(D)
    o, bo = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, bl = np.full((H, len(q)), np.nan), np.full((H, len(q)), np.nan)
    for q0, n, k0, m in spans:
        for h in range(H):
            vv = v[k0:k0 + m, h // G]
            P, oo, ll, es = _head(q[q0:q0 + n, h], k[k0:k0 + m, h // G], vv, scale, causal)
            o[q0:q0 + n, h] = oo
            bo[q0:q0 + n, h] = U * np.abs(oo) + (1 + U) * (U + 2 * es + (m + 64) * E) * (P @ np.abs(vv))
            lse[h, q0:q0 + n] = ll
            bl[h, q0:q0 + n] = es + (m + 64) * E + 4 * E * np.abs(np.where(np.isfinite(ll), ll, 0.0))
    return o, bo, lse, bl


def gradients(q, k, v, d_o, spans, scale=None, causal=True):
    """dq, dk, dv and their bounds (dicts). The kernels take P from scores, dS from P, the product d_o v and
    d_o . o with o as it was rounded, and round P and dS to bf16 for the last products."""
    H, D = q.shape[1:]
    G = H // k.shape[1]
    scale = scale or 1.0 / math.sqrt(D)
    out = {x: np.full(t.shape, np.nan) for x, t in (("dq", q), ("dk", k), ("dv", v))}
    bound = {x: t.copy() for x, t in out.items()}
    for q0, n, k0, m in spans:
        for x in ("dk", "dv"):
            out[x][k0:k0 + m] = 0.0
            bound[x][k0:k0 + m] = 0.0
        for h in range(H):
            rows, keys, kv = slice(q0, q0 + n), slice(k0, k0 + m), h // G
            Q, K, V, dO = q[rows, h], k[keys, kv], v[keys, kv], d_o[rows, h]
            P, o, _, es = _head(Q, K, V, scale, causal)
            dP, delta = dO @ V.T, (dO * o).sum(1, keepdims=True)
            dS = P * (dP - delta)
            fine = (D + 8) * E
            b_delta = (np.abs(dO) * (U * np.abs(o) + (1 + U) * (U + 2 * es + (m + 64) * E) * (P @ np.abs(V)))).sum(1, keepdims=True)
            b_delta = b_delta + fine * (np.abs(dO) * np.abs(o)).sum(1, keepdims=True)
            bS = P * ((2 * es + 8 * E) * np.abs(dP - delta) + (1 + 2 * es) * (fine * (np.abs(dO) @ np.abs(V).T) + b_delta))
            bS = (1 + U) * bS + U * np.abs(dS)
            out["dq"][rows, h] = scale * dS @ K
            bound["dq"][rows, h] = scale * (bS + (m + 64) * E * np.abs(dS)) @ np.abs(K)
            out["dk"][keys, kv] += scale * dS.T @ Q
            bound["dk"][keys, kv] += scale * (bS + (n * G + 64) * E * np.abs(dS)).T @ np.abs(Q)
            out["dv"][keys, kv] += P.T @ dO
            bound["dv"][keys, kv] += (P * (U + 2 * es + (n * G + 64) * E)).T @ np.abs(dO)
    for x in out:
        bound[x] = (1 + U) * bound[x] + U * np.abs(out[x])
    return out, bound


def deviations(q, k, v, d_o, spans, scale=None, causal=True):
    """Mean squares that the elements of dq, dk and dv may differ by (a dict): the sum over many of them bounds the
    square of the 2-norm, which the bounds of gradients(), all roundings at their worst together, do not say anything
    about (a sum of N terms may lose some sqrt(N) of them there). Roundings to bf16 are independent of each other and of mean
    square U^2 / 3 relative to the power of two below at most; U^2 relative to the value is taken. A row's delta, d_o . o with o as it
    was rounded (each of its columns, and each probability that went into it), is common to all of the row's dS. A score's error
    es stands beside each rounding of P and dS."""
    H, D = q.shape[1:]
    G = H // k.shape[1]
    scale = scale or 1.0 / math.sqrt(D)
    mean = {x: np.full(t.shape, np.nan) for x, t in (("dq", q), ("dk", k), ("dv", v))}
    for q0, n, k0, m in spans:
        keys = slice(k0, k0 + m)
        sums = {x: np.zeros(t[keys].shape) for x, t in (("dk", k), ("dv", v))}
        mean["dk"][keys] = mean["dv"][keys] = 0.0
        for h in range(H):
            rows, kv = slice(q0, q0 + n), h // G
            Q, K, V, dO = q[rows, h], k[keys, kv], v[keys, kv], d_o[rows, h]
            P, o, _, es = _head(Q, K, V, scale, causal)
            dP = dO @ V.T
            dS = P * (dP - (dO * o).sum(1, keepdims=True))
            u2 = U ** 2 + (2 * es) ** 2
            m_delta = u2 * (((dO * o) ** 2).sum(1, keepdims=True) + ((P * dP) ** 2).sum(1, keepdims=True))
            m_S = u2 * dS ** 2 + (P * ((D + 8) * E * (np.abs(dO) @ np.abs(V).T))) ** 2
            mean["dq"][rows, h] = scale ** 2 * (m_S @ K ** 2 + m_delta * (P @ K) ** 2) + (U * scale * dS @ K) ** 2
            mean["dk"][keys, kv] += scale ** 2 * (m_S + m_delta * P ** 2).T @ Q ** 2
            mean["dv"][keys, kv] += u2 * (P ** 2).T @ dO ** 2
            sums["dk"][:, kv] += scale * dS.T @ Q
            sums["dv"][:, kv] += P.T @ dO
        for x in sums:
            mean[x][keys] += (U * sums[x]) ** 2
    return mean
