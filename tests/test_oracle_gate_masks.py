"""The float64 oracle of the routing by scores where experts are masked, against brute force over
the definition: a masked expert has score 0, no part in its group's score, and comes behind the
others of its group; a group of nothing else comes behind every other group."""
import math

import numpy as np
import pytest

from oracle import gate as OG

LOWEST = -(2 - 2.0 ** -7) * 2.0 ** 127     # of bf16: the largest logit that masks


def brute_force(h, k, score, bias, G, tg, group_score):
    """ids of one row by sorting in plain Python."""
    N, size = len(h), len(h) // G
    live = [v > LOWEST for v in h]
    s = OG.scores(np.where(live, h, -np.inf)[None], score)[0]
    key = list(h) if bias is None else [s[j] + bias[j] for j in range(N)]
    allowed = list(range(G))
    if tg < G:
        def rank(g):
            part = [j for j in range(g * size, (g + 1) * size) if live[j]]
            if not part:
                return (1, 0.0, g)
            if group_score == "max":
                return (0, -max(key[j] for j in part), g)
            best = sorted((s[j] + (0.0 if bias is None else bias[j]) for j in part), reverse=True)
            return (0, -sum(best[:2]), g)
        allowed = sorted(allowed, key=rank)[:tg]
    pool = [j for g in allowed for j in range(g * size, (g + 1) * size)]
    return sorted(pool, key=lambda j: (not live[j], -key[j] if live[j] else 0.0, j))[:k]


def masked_rows(rng, N, G, value=-math.inf):
    """Rows whose groups are masked wholly, but for one expert, in part, and not at all."""
    size = N // G
    h = rng.normal(0, 1.5, (12, N)).astype(np.float32)
    for t in range(len(h)):
        for g in range(G):
            kind = (t + g) % 4
            part = h[t, g * size:(g + 1) * size]
            if kind == 0:
                part[:] = value
            elif kind == 1:
                part[np.arange(size) != rng.integers(size)] = value
            elif kind == 2:
                part[rng.random(size) < 0.5] = value
    h[-1] = value
    return h


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("level", [None, -1.5, -0.2, 0.3])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("N,G,tg,k", [(4, 2, 1, 2), (64, 8, 1, 4), (64, 8, 3, 8), (60, 6, 5, 10)])
def test_choice_with_masks(N, G, tg, k, group_score, level, score):
    rng = np.random.default_rng(N + tg)
    h = masked_rows(rng, N, G)
    bias = None if level is None else level + 0.1 * rng.normal(0, 1, N)
    ids, w, _ = OG.gate(h, k, score, bias, G, tg, group_score, False)
    for t in range(len(h)):
        assert list(ids[t]) == brute_force(h[t], k, score, bias, G, tg, group_score), t
    assert (w[np.isneginf(np.take_along_axis(h, ids, 1))] == 0).all()


def test_a_group_of_masked_experts_beats_no_live_one():
    h = np.array([[0.0, 0.0, -np.inf, -np.inf]])
    for group_score in ("max", "top2"):
        ids, w, _ = OG.gate(h, 2, "sigmoid", np.full(4, -1.5), 2, 1, group_score)
        assert ids.tolist() == [[0, 1]] and w.tolist() == [[0.5, 0.5]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("value", [LOWEST, float(np.finfo(np.float32).min)])
def test_lowest_value_masks_as_infinity_does(value, group_score, score):
    for level in (-1.5, 0.3):
        args = (10, score, level + np.random.default_rng(1).normal(0, 1, 60), 6, 5, group_score)
        a = OG.gate(masked_rows(np.random.default_rng(2), 60, 6), *args)
        b = OG.gate(masked_rows(np.random.default_rng(2), 60, 6, value), *args)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    # the next value above bf16's lowest is a logit as others are
    assert OG.gate([[np.nextafter(value, 0)]], 1)[1] == (1.0 if value == LOWEST else 0.0)
