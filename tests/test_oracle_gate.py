"""The float64 oracle of the routing by scores: against brute force over the definition, and its
gradient against differences."""
import itertools

import numpy as np
import pytest

from oracle import gate as OG


def _brute(h, k, score, bias, G, tg, group_score):
    """ids of one row by sorting (value, index) pairs in plain Python."""
    s = OG.scores(h[None], score)[0]
    c = list(h) if bias is None else [s[j] + bias[j] for j in range(len(h))]
    size = len(h) // G
    allowed = range(G)
    if tg < G:
        g = []
        for i in range(G):
            part = range(i * size, i * size + size)
            if group_score == "max":
                g.append(max(c[j] for j in part))
            else:
                v = [s[j] + (0.0 if bias is None else bias[j]) for j in part]
                g.append(max(a + b for a, b in itertools.combinations(v, 2)))
        allowed = sorted(range(G), key=lambda i: (-g[i], i))[:tg]
    pool = [j for i in allowed for j in range(i * size, i * size + size)]
    return sorted(pool, key=lambda j: (-c[j], j))[:k]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("G,tg,group_score", [(1, 1, "max"), (4, 2, "max"), (4, 2, "top2"),
                                              (6, 5, "top2"), (12, 3, "max")])
def test_choice_against_brute_force(score, with_bias, G, tg, group_score):
    rng = np.random.default_rng(3)
    h = np.round(rng.normal(0, 1.5, (20, 24)) * 4) / 4          # ties abound
    bias = np.round(rng.normal(0, 0.1, 24) * 64) / 64 if with_bias else None
    ids, w, _ = OG.gate(h, 4, score, bias, G, tg, group_score, False, 2.0)
    for t in range(len(h)):
        assert list(ids[t]) == _brute(h[t], 4, score, bias, G, tg, group_score)
    assert np.allclose(w, 2.0 * np.take_along_axis(OG.scores(h, score), ids, 1), rtol=1e-15)


def test_weights_sum_and_margin():
    h = np.array([[1.0, 1.0, 0.5, 0.0], [0.0, 3.0, 2.0, 1.0]])
    ids, w, margin = OG.gate(h, 2, "sigmoid", None, 1, 1, "max", True, 2.5)
    assert ids.tolist() == [[0, 1], [1, 2]]
    assert np.allclose(w.sum(axis=1), 2.5)
    assert margin.tolist() == [0.5, 1.0]      # ties decide nothing that rounding could change
    assert np.allclose(w, OG.weights(h, ids, "sigmoid", True, 2.5))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_against_differences(score, renormalize):
    rng = np.random.default_rng(5)
    h = rng.normal(0, 1.5, (6, 11))
    ids = np.stack([rng.permutation(11)[:4] for _ in range(6)])
    ids[2, 1] = -1
    ids[3] = -1
    dw = rng.normal(0, 1, (6, 4))
    got = OG.gradient(h, ids, dw, score, renormalize, 1.7)
    eps = 1e-6
    for t, j in itertools.product(range(6), range(11)):
        up, dn = h.copy(), h.copy()
        up[t, j] += eps
        dn[t, j] -= eps
        f = [(OG.weights(v, ids, score, renormalize, 1.7) * np.where(ids >= 0, dw, 0)).sum()
             for v in (up, dn)]
        assert abs((f[0] - f[1]) / (2 * eps) - got[t, j]) < 1e-7
