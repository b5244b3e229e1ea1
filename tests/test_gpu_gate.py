"""xshare_gate and xshare_gate_backward against the float64 oracle.

The choice must be the oracle's.  Two correct computations of a score in fp32 may differ in
its last bits, so rows whose choice hangs on less than 1e-5 are drawn again (the kernel's scores
err by less than 2e-6); exact ties stay, and go to the lower index.  Weights: an exponential
(2 ulp), a sum of up to 1024 terms in 16 + 6 additions, three more roundings and the sum of the
chosen: at most 64 * 2^-24.  Gradients: the same factors against terms of size |ds| s, within
256 * 2^-24 of the row's largest such term."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from oracle import gate as OG
from test_gpu_guards import IN_FILL, OUT_FILL, Guarded

pytestmark = pytest.mark.gpu
W_TOL, G_TOL, MARGIN = 64 * 2.0 ** -24, 256 * 2.0 ** -24, 1e-5


def _bf16(v):
    return torch.from_numpy(np.asarray(v, np.float32)).to(torch.bfloat16).float().numpy()


def _rows(rng, T, N, kw, dtype, spread=1.5):
    h = rng.normal(0, spread, (T, N)).astype(np.float32)
    h = _bf16(h) if dtype == "bf16" else h
    for _ in range(50):
        bad = OG.gate(h, **kw)[2] < MARGIN
        if not bad.any():
            return h
        new = rng.normal(0, spread, (T, N)).astype(np.float32)
        h[bad] = (_bf16(new) if dtype == "bf16" else new)[bad]
    raise AssertionError("no rows of a clear choice")


def _device(h, dtype):
    return torch.from_numpy(np.ascontiguousarray(h)).to(
        DEV, torch.bfloat16 if dtype == "bf16" else torch.float32)


def _check(h, dtype, kw, label):
    from paper_2602_07265_amd import xshare as X
    say(f"gate case {label} T={h.shape[0]} N={h.shape[1]} {dtype} {kw}")
    dev = dict(kw)
    if dev.get("bias") is not None:
        dev["bias"] = torch.from_numpy(np.asarray(dev["bias"], np.float32)).to(DEV)
    k = dev.pop("top_k")
    got = X.gate(_device(h, dtype), k, **dev)
    torch.cuda.synchronize()
    ids, w, _ = OG.gate(h, **kw)
    assert np.array_equal(got["ids"].cpu().numpy(), ids), label
    err = np.abs(got["w"].cpu().numpy() - w) / np.maximum(np.abs(w), 1e-30)
    assert err.max(initial=0.0) <= W_TOL, (label, err.max())
    return got


FORMS = [dict(score="softmax", renormalize=True), dict(score="softmax", renormalize=False),
         dict(score="sigmoid", renormalize=True, scale=2.5),
         dict(score="sigmoid", renormalize=False)]


@pytest.mark.parametrize("form", range(4))
@pytest.mark.parametrize("N,k", [(1, 1), (2, 2), (8, 2), (60, 6), (64, 1), (65, 4), (128, 8),
                                 (160, 32), (256, 8), (257, 10), (513, 8), (1024, 32)])
def test_choice_and_weights(N, k, form):
    rng = np.random.default_rng(N * 37 + form)
    for T, dtype in ((1, "fp32"), (33, "bf16"), (5, "fp32")):
        for bias in (None, rng.normal(0, 0.05, N).astype(np.float32)):
            kw = dict(top_k=k, bias=bias, **FORMS[form])
            _check(_rows(rng, T, N, kw, dtype), dtype, kw, "plain")


@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("N,G,tg,k", [(8, 4, 1, 2), (24, 4, 2, 3), (256, 8, 4, 8), (256, 8, 8, 8),
                                      (160, 8, 3, 6), (96, 6, 5, 16), (128, 64, 32, 8),
                                      (1024, 64, 3, 20), (1022, 2, 1, 9), (63, 3, 1, 21)])
@pytest.mark.parametrize("form", [0, 2])
def test_groups(N, G, tg, k, group_score, form):
    rng = np.random.default_rng(N + G + tg)
    for T, dtype, with_bias in ((1, "fp32", True), (19, "fp32", False), (37, "bf16", True)):
        bias = rng.normal(0, 0.05, N).astype(np.float32) if with_bias else None
        kw = dict(top_k=k, bias=bias, n_groups=G, top_groups=tg, group_score=group_score,
                  **FORMS[form])
        _check(_rows(rng, T, N, kw, dtype), dtype, kw, "groups")


@pytest.mark.parametrize("T", [2, 3, 4, 7, 63, 64, 65, 1000, 4099])
def test_batches(T):
    rng = np.random.default_rng(T)
    kw = dict(top_k=8, score="sigmoid", bias=rng.normal(0, 0.05, 256).astype(np.float32),
              n_groups=8, top_groups=4, group_score="top2", scale=2.5)
    _check(_rows(rng, T, 256, kw, "fp32"), "fp32", kw, "batch")


@pytest.mark.parametrize("N,shift", [(256, 1), (256, 2), (128, 3), (65, 1)])
def test_bias_at_any_address(N, shift):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(N + shift)
    h = torch.from_numpy(rng.normal(0, 1, (9, N)).astype(np.float32)).to(DEV)
    bias = torch.full((N + 8,), float("nan"), device=DEV)
    bias[shift:shift + N] = torch.from_numpy(rng.normal(0, 0.3, N).astype(np.float32)).to(DEV)
    part = bias[shift:shift + N]
    say(f"gate case bias {shift} floats on N={N}")
    a = X.gate(h, 6, score="sigmoid", bias=part)
    b = X.gate(h, 6, score="sigmoid", bias=part.clone())
    assert torch.equal(a["ids"], b["ids"]) and torch.equal(a["w"], b["w"])


def test_ties_go_to_the_lower_index():
    kw = dict(top_k=5, score="sigmoid")
    h = np.zeros((3, 70), np.float32)
    h[1] = np.arange(70) % 3
    h[2, 10:] = -0.0                        # equal to +0
    got = _check(h, "fp32", kw, "ties")
    assert got["ids"][0].tolist() == [0, 1, 2, 3, 4]
    assert got["ids"][2].tolist() == [0, 1, 2, 3, 4]
    # equal groups: the lower ones; equal experts of them in order
    kw = dict(top_k=6, n_groups=8, top_groups=2, group_score="top2", score="sigmoid",
              bias=np.zeros(64, np.float32))
    got = _check(np.ones((2, 64), np.float32), "fp32", kw, "equal groups")
    assert got["ids"][0].tolist() == [0, 1, 2, 3, 4, 5]


def test_extreme_logits():
    # saturated sigmoids rank by the logit where there is no bias; scores that all underflow
    # give weights of zero
    h = np.array([[200, 300, 100, 150], [-300, -250, -400, -200], [88, -88, 0, 1]], np.float32)
    for score in ("sigmoid", "softmax"):
        _check(h, "fp32", dict(top_k=2, score=score, renormalize=False), "extreme " + score)
    got = _check(h[1:2], "fp32", dict(top_k=2, score="sigmoid", renormalize=True), "underflow")
    assert got["w"].tolist() == [[0.0, 0.0]]


@pytest.mark.parametrize("form", range(4))
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_masked_experts(form, group_score):
    """-inf masks an expert, whatever its bias; rows with fewer experts left than k, and with none,
    still give k indices, and weights of 0 for what is masked."""
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(40 + form)
    for N, G, tg, k in ((64, 1, 1, 6), (256, 8, 4, 8), (60, 4, 2, 5)):
        for bias in (None, (0.5 * rng.normal(0, 1, N)).astype(np.float32)):
            kw = dict(top_k=k, bias=bias, n_groups=G, top_groups=tg, group_score=group_score,
                      **FORMS[form])
            h = _rows(rng, 9, N, kw, "fp32")
            h[1, ::2] = h[2, 5:] = h[3, :-3] = h[4] = h[6, 0] = -np.inf
            keep = OG.gate(h, **kw)[2] >= MARGIN
            got = _check(h[keep], "fp32", kw, "masked")
            w = got["w"].cpu().numpy()
            hidden = np.isneginf(np.take_along_axis(h[keep], got["ids"].cpu().numpy(), 1))
            assert np.isfinite(w).all() and (w[hidden] == 0).all()
            dw = torch.randn(w.shape, device=DEV)
            d = X.gate_backward(_device(h[keep], "fp32"), got["ids"], dw, **FORMS[form])
            d = d.cpu().numpy()
            assert np.isfinite(d).all() and (d[np.isneginf(h[keep])] == 0).all()


def test_strided_rows_guards_and_empty_batch():
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(9)
    for dtype, size in (("fp32", 4), ("bf16", 2)):
        T, N, ld, k = 13, 77, 91, 5
        kw = dict(top_k=k, score="softmax")
        h = _rows(rng, T, N, kw, dtype)
        td = torch.bfloat16 if dtype == "bf16" else torch.float32
        buf = Guarded(T * ld * size, IN_FILL)          # NaN between the rows too
        view = buf.view(td, (T, ld))[:, :N]
        view.copy_(_device(h, dtype))
        gi, gw = Guarded(T * k * 4, OUT_FILL), Guarded(T * k * 4, OUT_FILL)
        say(f"gate case strided {dtype}")
        X.gate(view, k, score="softmax", out=dict(ids=gi.view(torch.int32, (T, k)),
                                                  w=gw.view(torch.float32, (T, k))))
        dw = torch.randn((T, k), device=DEV)
        gd = Guarded(T * N * 4, OUT_FILL)
        X.gate_backward(view, gi.view(torch.int32, (T, k)), dw,
                        out=gd.view(torch.float32, (T, N)))
        torch.cuda.synchronize()
        ids, w, _ = OG.gate(h, **kw)
        assert np.array_equal(gi.view(torch.int32, (T, k)).cpu().numpy(), ids)
        assert np.allclose(gw.view(torch.float32, (T, k)).cpu().numpy(), w, rtol=W_TOL, atol=0)
        ref = OG.gradient(h, ids, dw.cpu().numpy(), "softmax", True, 1.0)
        assert np.abs(gd.view(torch.float32, (T, N)).cpu().numpy() - ref).max() < 1e-5
        assert gi.intact() and gw.intact() and gd.intact() and buf.intact()
    empty = torch.empty((0, 16), device=DEV)
    r = X.gate(empty, 3)
    assert r["ids"].shape == (0, 3) and r["w"].shape == (0, 3)
    assert X.gate_backward(empty, r["ids"], r["w"]).shape == (0, 16)


@pytest.mark.parametrize("form", range(4))
@pytest.mark.parametrize("N,k", [(1, 1), (8, 2), (65, 4), (128, 8), (256, 8), (300, 32), (1024, 9)])
def test_gradient(N, k, form):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(N + form)
    f = FORMS[form]
    scale = f.get("scale", 1.0)
    for T, dtype in ((1, "fp32"), (29, "bf16"), (6, "fp32")):
        h = rng.normal(0, 1.5, (T, N)).astype(np.float32)
        h = _bf16(h) if dtype == "bf16" else h
        ids = np.stack([rng.permutation(N)[:k] for _ in range(T)]).astype(np.int32)
        if T > 4:                           # pairs that are none: their dw must not be read
            ids[1, 0], ids[2], ids[3, -1] = -1, -1, N
        dw = rng.normal(0, 1, (T, k)).astype(np.float32)
        nan = np.where((ids < 0) | (ids >= N), np.nan, dw).astype(np.float32)
        say(f"gate gradient case N={N} k={k} T={T} {dtype} {f}")
        got = X.gate_backward(_device(h, dtype), torch.from_numpy(ids).to(DEV),
                              torch.from_numpy(nan).to(DEV), **f).cpu().numpy()
        ref = OG.gradient(h, ids, dw, f["score"], f["renormalize"], scale)
        # the terms that are added up: |ds| s of the chosen, before they cancel
        s = OG.scores(h, f["score"])
        ok = (ids >= 0) & (ids < N)
        p = np.where(ok, np.take_along_axis(s, np.where(ok, ids, 0), 1), 0.0)
        total = p.sum(1, keepdims=True) if f["renormalize"] else np.ones((T, 1))
        size = scale * (np.abs(dw) * p).max(1, keepdims=True) / np.maximum(total, 1e-30)
        assert (np.abs(got - ref) <= G_TOL * size + 1e-30).all()
        none = np.ones((T, N), bool)
        for t in range(T):
            none[t, ids[t][ok[t]]] = False
        if f["score"] == "sigmoid" or f["renormalize"]:
            assert (got[none] == 0).all()


def test_refusals_raise():
    from paper_2602_07265_amd import xshare as X
    h = torch.zeros((4, 64), device=DEV)
    for kw in (dict(top_k=65), dict(top_k=0), dict(top_k=4, n_groups=7),
               dict(top_k=33), dict(top_k=9, n_groups=8, top_groups=1)):
        with pytest.raises(X.XShareError):
            X.gate(h, **kw)
    with pytest.raises(ValueError):
        X.gate(h, 4, bias=torch.zeros(63, device=DEV))
    with pytest.raises(ValueError):
        X.gate(h.t(), 4)
    with pytest.raises(ValueError):
        X.gate_backward(h, torch.zeros((4, 2), dtype=torch.int64, device=DEV),
                        torch.zeros((4, 2), device=DEV))
