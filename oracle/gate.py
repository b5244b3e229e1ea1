"""Routing by scores, bias and groups (oracle side), in float64.

A token's scores are s_j = exp(h_j - max h) / sum (softmax) or 1 / (1 + exp(-h_j)) (sigmoid).
Experts rank by c_j = s_j + bias_j, or by h_j without a bias; a group's score is the largest
c_j of its N / G consecutive experts, or the sum of its two largest s_j (+ bias_j); ties go to
the lower index.  The k best experts of the top_groups best groups are taken, with weights
w_r = s_{id_r}, divided by their sum if asked, times `scale`.  A logit of -inf, or up to the
lowest value of bf16, masks its expert: score 0, ranked last, no part in a sum of two; a group
without any other expert ranks last.
"""
from __future__ import annotations

import numpy as np

MASK = -float.fromhex("0x1.FEp127")       # the largest logit that masks


def scores(h, score):
    h = np.asarray(h, np.float64)
    h = np.where(h <= MASK, -np.inf, h)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-h))
    m = h.max(axis=1, keepdims=True)
    e = np.exp(h - np.where(np.isfinite(m), m, 0.0))
    return e / np.maximum(e.sum(axis=1, keepdims=True), 2.0 ** -126)


def _best(values, n):
    """Indices of the n largest, best first, the lower index first on ties."""
    return np.argsort(-values, axis=1, kind="stable")[:, :n]


def gate(h, top_k, score="softmax", bias=None, n_groups=1, top_groups=1, group_score="max",
         renormalize=True, scale=1.0):
    """(ids [T, k], w [T, k], margin [T]): margin is the least difference of two unequal values
    that decided a row's choice or its order (inf where none did)."""
    h = np.asarray(h, np.float64)
    T, N = h.shape
    s = scores(h, score)
    masked = h <= MASK
    c = h if bias is None else np.where(masked, -np.inf, s + np.asarray(bias, np.float64))
    margin = np.full(T, np.inf)

    def gap(ranked):
        ranked = np.where(np.isfinite(ranked), ranked, -1e30)
        d = ranked[:, :-1] - ranked[:, 1:]
        return np.where(d > 0, d, np.inf).min(axis=1, initial=np.inf)

    if top_groups < n_groups:
        base = c
        if group_score == "top2":
            base = np.where(masked, -np.inf, s if bias is None else c)
        per = -np.sort(-base.reshape(T, n_groups, -1), axis=2)
        gs = per[:, :, 0]
        if group_score == "top2":
            gs = gs + np.where(np.isneginf(per[:, :, 1]), 0.0, per[:, :, 1])
        order = _best(gs, n_groups)
        at = np.take_along_axis(gs, order[:, top_groups - 1:top_groups + 1], 1)
        margin = np.minimum(margin, gap(at))
        keep = np.zeros((T, n_groups), bool)
        np.put_along_axis(keep, order[:, :top_groups], True, 1)
        # experts outside the groups come after the masked ones inside
        keep = np.repeat(keep, N // n_groups, axis=1)
        order = np.lexsort((-c, ~keep), axis=1)[:, :min(top_k + 1, N)]
        c = np.where(keep, c, -np.inf)
    else:
        order = _best(c, min(top_k + 1, N))
    ranked = np.take_along_axis(c, order, 1)
    margin = np.minimum(margin, gap(ranked))
    ids = order[:, :top_k]
    w = np.take_along_axis(s, ids, 1)
    if renormalize:
        w = w / np.maximum(w.sum(axis=1, keepdims=True), 2.0 ** -126)
    return ids, w * scale, margin


def weights(h, ids, score, renormalize, scale):
    """The weights of a given choice (ids outside [0, N) have none)."""
    s = scores(h, score)
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < s.shape[1])
    w = np.where(ok, np.take_along_axis(s, np.where(ok, ids, 0), 1), 0.0)
    if renormalize:
        w = w / np.maximum(w.sum(axis=1, keepdims=True), 2.0 ** -126)
    return w * scale


def gradient(h, ids, dw, score, renormalize, scale):
    """d(sum w dw) / dh by the chain rule."""
    h = np.asarray(h, np.float64)
    T, N = h.shape
    s = scores(h, score)
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < N)
    p = np.where(ok, np.take_along_axis(s, np.where(ok, ids, 0), 1), 0.0)
    dp = np.where(ok, scale * np.asarray(dw, np.float64), 0.0)
    if renormalize:
        total = p.sum(axis=1, keepdims=True)
        safe = np.where(total >= 2.0 ** -126, total, 1.0)
        dp = np.where(ok & (total >= 2.0 ** -126),
                      (dp - (dp * p).sum(axis=1, keepdims=True) / safe) / safe, 0.0)
    ds = np.zeros((T, N))
    for t in range(T):
        for r in range(ids.shape[1]):
            if ok[t, r]:
                ds[t, ids[t, r]] += dp[t, r]
    if score == "sigmoid":
        return ds * s * scores(-h, score)      # 1 - s, with all its bits
    return s * (ds - (ds * s).sum(axis=1, keepdims=True))
