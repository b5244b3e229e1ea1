"""xshare_gate where experts are masked: the choice against the brute force of
test_oracle_gate_masks over the rows whose choice hangs on 1e-5 or more (the kernel's scores err by
less than 2e-6), weights of 0 for what is masked, and no masked expert where the chosen groups
hold k others."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from oracle import gate as OG
from test_oracle_gate_masks import brute_force, masked_rows

pytestmark = pytest.mark.gpu
MARGIN = 1e-5


def _check(h, logits, k, score, bias, G, tg, group_score, masked):
    """h: the logits' values with -inf where an expert is masked."""
    from paper_2602_07265_amd import xshare as X
    got = X.gate(logits, k, score=score, n_groups=G, top_groups=tg, group_score=group_score,
                 bias=None if bias is None else torch.from_numpy(bias).to(DEV))
    ids, w = got["ids"].cpu().numpy(), got["w"].cpu().numpy()
    _, _, margin = OG.gate(h, k, score, bias, G, tg, group_score)
    assert (margin >= MARGIN).sum() >= len(h) // 2
    for t in np.flatnonzero(margin >= MARGIN):
        assert list(ids[t]) == brute_force(h[t], k, score, bias, G, tg, group_score), t
    hidden = np.take_along_axis(masked, ids, 1)
    assert np.isfinite(w).all() and (w[hidden] == 0).all()
    return ids, w


# groups that fill whole lanes, and others; one to several experts a lane
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("level", [None, -1.5, -0.2, 0.3])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("N,G,tg,k", [(4, 2, 1, 2), (64, 8, 1, 4), (256, 8, 3, 8), (60, 6, 5, 10),
                                      (513, 3, 1, 9), (1024, 64, 5, 20)])
def test_choice_with_masked_groups(N, G, tg, k, group_score, level, score):
    rng = np.random.default_rng(N + tg)
    h = masked_rows(rng, N, G)
    bias = None if level is None else (level + 0.1 * rng.normal(0, 1, N)).astype(np.float32)
    say(f"gate case masked groups N={N} G={G} top_groups={tg} {group_score} {score} bias {level}")
    _check(h, torch.from_numpy(h).to(DEV), k, score, bias, G, tg, group_score, np.isneginf(h))


def test_a_group_of_masked_experts_beats_no_live_one():
    h = np.array([[0.0, 0.0, -np.inf, -np.inf]], np.float32)
    say("gate case one live group of negative scores")
    for group_score in ("max", "top2"):
        ids, w = _check(h, torch.from_numpy(h).to(DEV), 2, "sigmoid", np.full(4, -1.5, np.float32),
                        2, 1, group_score, np.isneginf(h))
        assert ids.tolist() == [[0, 1]] and w.tolist() == [[0.5, 0.5]]


# ------------------------------------------------------------------ masks of the lowest value

FORMS = [dict(score="softmax", renormalize=True), dict(score="softmax", renormalize=False),
         dict(score="sigmoid", renormalize=True, scale=2.5),
         dict(score="sigmoid", renormalize=False)]


@pytest.mark.parametrize("form", range(4))
@pytest.mark.parametrize("kind", ["fp32", "bf16", "bf16 in fp32"])
def test_lowest_value_masks_as_infinity_does(kind, form):
    """Logits masked with their type's lowest value, whatever the biases: the choice and weights
    that -inf gives (no bias ranks by the logits, where both come last), and gradients of 0."""
    from paper_2602_07265_amd import xshare as X
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    value = torch.finfo(torch.float32 if kind == "fp32" else torch.bfloat16).min
    rng = np.random.default_rng(5 + form)
    f = FORMS[form]
    for N, G, tg, k in ((64, 8, 2, 6), (60, 6, 5, 10), (40, 1, 1, 9)):
        h = torch.from_numpy(masked_rows(rng, N, max(G, 4))).to(dtype).float()
        masked = torch.isneginf(h)
        low = torch.where(masked, torch.full_like(h, value), h).to(dtype)
        for bias in (None, 2 * torch.randn(N, device=DEV), torch.full((N,), -3.0, device=DEV)):
            for group_score in ("max", "top2"):
                say(f"gate case lowest value {kind} N={N} G={G} {group_score} {f}")
                kw = dict(bias=bias, n_groups=G, top_groups=tg, group_score=group_score, **f)
                a = X.gate(h.to(DEV, dtype), k, **kw)
                b = X.gate(low.to(DEV), k, **kw)
                assert torch.equal(a["ids"], b["ids"]) and torch.equal(a["w"], b["w"])
                hidden = masked.to(DEV).gather(1, b["ids"].long())
                assert (b["w"][hidden] == 0).all() and torch.isfinite(b["w"]).all()
                d = X.gate_backward(low.to(DEV), b["ids"], torch.randn(len(h), k, device=DEV), **f)
                assert torch.isfinite(d).all() and (d[masked.to(DEV)] == 0).all()
