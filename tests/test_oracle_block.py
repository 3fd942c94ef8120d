"""Oracles of packed attention, the RMS norm and the balance loss against explicit loops and differences."""
import math

import numpy as np
import pytest

from oracle import balance, norm, packed


def _qkv(rng, Tq, Tk, H, Hkv, D):
    return rng.standard_normal((Tq, H, D)), rng.standard_normal((Tk, Hkv, D)), rng.standard_normal((Tk, Hkv, D))


SPANS = [(0, 3, 0, 3), (3, 0, 3, 2), (3, 1, 5, 4), (4, 4, 9, 2), (8, 2, 11, 0)]   # packed, no query, a cache, rows that see none


@pytest.mark.parametrize("causal", [True, False])
def test_attention_by_loops(causal):
    rng = np.random.default_rng(0)
    q, k, v = _qkv(rng, 10, 11, 4, 2, 3)
    o, _, lse, _ = packed.attention(q, k, v, SPANS, 0.7, causal)
    for q0, n, k0, m in SPANS:
        for i in range(n):
            for h in range(4):
                keys = [j for j in range(m) if not causal or j <= i + m - n]
                w = [math.exp(0.7 * sum(q[q0 + i, h, d] * k[k0 + j, h // 2, d] for d in range(3))) for j in keys]
                want = [sum(w[x] * v[k0 + j, h // 2, d] for x, j in enumerate(keys)) / sum(w) for d in range(3)] if keys else [0] * 3
                assert np.allclose(o[q0 + i, h], want, atol=1e-13)
                assert math.isclose(lse[h, q0 + i], math.log(sum(w)), abs_tol=1e-12) if keys else lse[h, q0 + i] == -math.inf


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients_by_differences(causal):
    rng = np.random.default_rng(1)
    t = dict(zip("qkv", _qkv(rng, 10, 11, 4, 2, 3)))
    spans = [s for s in SPANS if s[1]]
    d_o = rng.standard_normal(t["q"].shape)
    got, bound = packed.gradients(t["q"], t["k"], t["v"], d_o, spans, 0.7, causal)
    f = lambda: np.nansum(packed.attention(t["q"], t["k"], t["v"], spans, 0.7, causal)[0] * d_o)
    for x in "qkv":
        g = got["d" + x]
        for at in np.ndindex(t[x].shape):
            if np.isnan(g[at]):
                continue
            old, step = t[x][at], 1e-5
            t[x][at] = old + step
            up = f()
            t[x][at] = old - step
            down = f()
            t[x][at] = old
            assert abs((up - down) / (2 * step) - g[at]) < 1e-8
    assert all((b[np.isfinite(b)] >= 0).all() for b in bound.values())


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().double().numpy()


@pytest.mark.parametrize("causal", [True, False])
def test_deviations_hold_roundings_and_not_a_block_left_out(causal):
    # the kernels' roundings made in fp64, as they are and with 32 rows of one head missing from 32 keys' dk and dv
    T, H, D = 520, 4, 64
    rng = np.random.default_rng(3)
    q, k, v = (_bf16(t) for t in _qkv(rng, T, T, H, 1, D))
    d_o = _bf16(rng.standard_normal(q.shape))
    spans = [(0, T, 0, T)]
    want, _ = packed.gradients(q, k, v, d_o, spans, causal=causal)
    mean = packed.deviations(q, k, v, d_o, spans, causal=causal)
    scale = D ** -0.5
    for missing in (False, True):
        got = {x: np.zeros(t.shape) for x, t in want.items()}
        for h in range(H):
            P, _, _, _ = packed._head(q[:, h], k[:, 0], v[:, 0], scale, causal)
            o = _bf16(_bf16(P) @ v[:, 0])
            dS = _bf16(P * (d_o[:, h] @ v[:, 0].T - (d_o[:, h] * o).sum(1, keepdims=True)))
            P = _bf16(P)
            got["dq"][:, h] = scale * dS @ k[:, 0]
            if missing and h == 1:
                P[448:480, 32:64] = dS[448:480, 32:64] = 0
            got["dk"][:, 0] += scale * dS.T @ q[:, h]
            got["dv"][:, 0] += P.T @ d_o[:, h]
        for x in got:
            off, allowed = np.linalg.norm(_bf16(got[x]) - want[x]), math.sqrt(mean[x].sum())
            assert off < 0.6 * allowed if not missing or x == "dq" else off > 1.2 * allowed, x


def test_norm_by_loops_and_differences():
    rng = np.random.default_rng(2)
    h, w, dy, dh = rng.standard_normal((3, 8)), rng.standard_normal(8), rng.standard_normal((3, 8)), rng.standard_normal((3, 8))
    y = norm.norm(h, w, 1e-3)
    for t in range(3):
        i = 1 / math.sqrt(sum(x * x for x in h[t]) / 8 + 1e-3)
        assert np.allclose(y[t], [x * i * c for x, c in zip(h[t], w)], atol=1e-14)
    dx, dw, _, _ = norm.backward(h, w, dy, 1e-3, dh)
    f = lambda: (norm.norm(h, w, 1e-3) * dy).sum() + (h * dh).sum()
    for a, g in ((h, dx), (w, dw)):
        for at in np.ndindex(a.shape):
            old = a[at]
            a[at] = old + 1e-5
            up = f()
            a[at] = old - 1e-5
            down = f()
            a[at] = old
            assert abs((up - down) / 2e-5 - g[at]) < 1e-8


def test_stream_rounds_to_even():
    x, r = np.array([[256.0, 256.0, 258.0, -256.0]]), np.array([[1.0, 3.0, 1.0, -1.0]])
    assert norm.stream(x, r).tolist() == [[256.0, 260.0, 260.0, -256.0]]      # steps of 2 there: 257, 259, 259 lie between


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_balance_by_loops_and_differences(kind):
    rng = np.random.default_rng(3)
    T, E, k, starts = 9, 5, 2, [0, 4, 4, 8]
    l = rng.standard_normal((T, E))
    l[1, 2] = -np.inf
    idx = np.argsort(-l, 1)[:, :k]
    idx[3, 1] = -1
    counts, mean, loss = balance.loss(l, idx, starts, kind, 0.3)
    for s in range(3):
        toks = range(starts[s], starts[s + 1])
        f, P = [0] * E, [0.0] * E
        for t in toks:
            e = [1 / (1 + math.exp(-x)) if kind == "sigmoid" else math.exp(x) for x in l[t]]
            for j in range(E):
                P[j] += e[j] / sum(e) / len(toks)
            for j in idx[t]:
                if 0 <= j < E:
                    f[j] += 1
        assert counts[s].tolist() == f and np.allclose(mean[s], P, atol=1e-14)
        want = 0.3 * E * sum(f[j] / (k * len(toks)) * P[j] for j in range(E)) if toks else 0.0
        assert math.isclose(loss[s], want, abs_tol=1e-14)
    d = np.array([1.0, 2.0, -0.5])
    g, _ = balance.backward(l, counts, k, starts, kind, 0.3, d)
    assert np.isnan(g[8]).all()
    for t in range(8):
        for e in range(E):
            if np.isinf(l[t, e]):
                assert g[t, e] == 0
                continue
            ends = []
            for step in (1e-5, -1e-5):
                l2 = l.copy()
                l2[t, e] += step
                ends.append((balance.loss(l2, idx, starts, kind, 0.3)[2] * d).sum())
            assert abs((ends[0] - ends[1]) / 2e-5 - g[t, e]) < 1e-9
    assert np.allclose(np.nansum(g, 1) if kind == "softmax" else 0, 0, atol=1e-15)


def test_a_balanced_router_has_loss_alpha():
    E, k = 4, 2
    l = np.zeros((4, E))
    idx = np.array([[0, 1], [2, 3], [0, 2], [1, 3]])
    for kind in ("softmax", "sigmoid"):
        assert math.isclose(balance.loss(l, idx, [0, 4], kind, 0.01)[2][0], 0.01)
