"""CPU checks of the gate oracle: selections by brute force, weights' gradient by differences."""
import itertools

import numpy as np
import pytest

from oracle import gate


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("n_group,topk_group,top2", [(1, 1, False), (4, 2, False), (4, 2, True), (3, 1, True)])
def test_selection_is_the_best_set(kind, n_group, topk_group, top2):
    # over all k-subsets of the kept groups' experts the selection has the largest sum of keys, in order
    g = np.random.default_rng(0)
    E, k = 12, 3
    for _ in range(5):
        l, b = g.standard_normal((1, E)), 0.3 * g.standard_normal(E)
        key = (gate.scores(l, kind) + b)[0]
        size = E // n_group
        sums = [sum(sorted(key[i * size:(i + 1) * size])[-2 if top2 else -1:]) for i in range(n_group)]
        kept = sorted(range(n_group), key=lambda i: -sums[i])[:topk_group]
        allowed = [e for e in range(E) if e // size in kept]
        best = max(itertools.combinations(allowed, k), key=lambda c: sum(key[list(c)]))
        got = gate.select(l, k, kind, n_group, topk_group, top2, b)[0]
        assert sorted(got) == sorted(best)
        assert np.all(np.diff(key[got]) <= 0)


def test_ties_masks_and_empty_rows():
    inf = np.inf
    l = np.array([[0., 0., 0., 0.], [-inf, 1., -inf, 0.], [-inf] * 4, [np.nan, 0., 1., -inf]])
    idx, w = gate.route(l, 2, "sigmoid", renorm=True)
    assert idx.tolist() == [[0, 1], [1, 3], [0, 1], [2, 1]]
    assert w[2].tolist() == [0, 0] and np.allclose(w[:2].sum(1), 1)
    idx, _ = gate.route(l[1:2], 3, "softmax")
    assert idx.tolist() == [[1, 3, 0]]
    # a group with one live expert competes with that expert; a dead group comes last
    l = np.array([[3., -inf, -inf, -inf, 1., 1.]])
    assert gate.select(l, 2, "sigmoid", 3, 1, True)[0].tolist() == [4, 5]
    assert gate.select(l, 2, "sigmoid", 3, 2, True)[0].tolist() == [0, 4]
    l = np.array([[-inf, -inf, 3., -inf]])
    assert gate.select(l, 1, "sigmoid", 2, 1, True)[0].tolist() == [2]


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_is_the_weights_differences(kind, renorm):
    g = np.random.default_rng(3)
    T, E, k, h = 4, 9, 3, 1e-6
    l = g.standard_normal((T, E))
    idx = gate.select(l, k, kind)
    idx[1] = [2, 2, 5]                                   # an expert listed twice
    d_w = g.standard_normal((T, k))
    grad, mag = gate.backward(l, idx, d_w, kind, renorm, 2.5)
    assert np.all(np.abs(grad) <= mag * (1 + 1e-12))
    for e in range(E):
        step = np.zeros((T, E))
        step[:, e] = h
        up, down = (gate.weights(l + s, idx, kind, renorm, 2.5) for s in (step, -step))
        want = ((up - down) * d_w).sum(1) / (2 * h)
        # a central difference is off by h^2 / 6 times a third derivative of at most 6, and by rounding, 2^-52 / h
        assert np.allclose(grad[:, e], want, atol=1e-8)


def test_gradient_of_rows_without_weights():
    l = np.full((1, 4), -np.inf)
    for kind in ("sigmoid", "softmax"):
        for renorm in (False, True):
            grad, _ = gate.backward(l, np.array([[0, 1]]), np.ones((1, 2)), kind, renorm)
            assert not grad.any()


def test_gradient_of_saturated_sigmoids():
    """s (1 - s) = 1 / (2 + e^l + e^-l) where 1 - s cancels in 64 bits too."""
    l = np.array([[40.0, 30.0, -40.0, 8.0]])
    grad, mag = gate.backward(l, np.array([[0, 1, 2, 3]]), np.ones((1, 4)), "sigmoid")
    want = 1 / (2 + np.exp(l) + np.exp(-l))
    assert np.allclose(grad, want, rtol=1e-14, atol=0) and np.allclose(mag, want, rtol=1e-14, atol=0)


def test_order_of_scores_that_64_bits_cannot_tell_apart():
    """Without a bias by the logits; with one, as computed: equal, so to the lower index."""
    l = np.array([[38.0, 40.0, 39.0, -1.0, 41.0, 40.0]])
    assert gate.select(l, 4, "sigmoid")[0].tolist() == [4, 1, 5, 2]
    assert gate.select(l, 4, "sigmoid", bias=np.zeros(6))[0].tolist() == [0, 1, 2, 4]
    l = np.array([[-800.0, -790.0, 0.0, -799.0]])                  # softmax scores below 64 bits' range
    assert gate.select(l, 3, "softmax")[0].tolist() == [2, 1, 3]
    assert gate.select(l, 3, "softmax", bias=np.zeros(4))[0].tolist() == [2, 0, 1]
