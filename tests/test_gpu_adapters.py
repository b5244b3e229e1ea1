"""Low-rank adapters and their gradients against the float64 oracle: one token to many, every width of
the rank's tiles, tokens and adapters without the other."""
import pytest
import torch

from group_bounds import adapter_rel, factor_rel, within
from helpers import DEV, say
from oracle import groups as OG

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _case(T, L, r, n, d, seed, none=0.25, pad=0, runs=False):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def rows(cols):
        m = torch.full((T, cols + pad), NAN, dtype=torch.bfloat16, device=DEV)[:, :cols]
        m.copy_(torch.randn(T, cols, generator=g, device=DEV))
        return m

    bf = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    ids = torch.randint(0, L, (T,), generator=g, device=DEV)
    if runs:
        ids = ids.sort().values
    off = torch.rand(T, generator=g, device=DEV) < none
    ids = torch.where(off, torch.where(ids % 2 == 0, -1, L + 3), ids).to(torch.int32)
    x, dy = rows(d), rows(n)
    return dict(x=x, dy=dy, a=bf(L, r, d), b=bf(L, n, r), ids=ids,
                scales=torch.randn(L, generator=g, device=DEV), base=rows(n), base_dx=rows(d))


SHAPES = [(1, 3, 8, 8, 8), (1, 4, 16, 4096, 4096), (2, 5, 24, 264, 520), (17, 3, 128, 136, 1000),
          (64, 20, 32, 2048, 712), (65, 20, 32, 520, 712), (65, 1, 16, 64, 72), (200, 7, 64, 328, 456),
          (300, 2, 40, 1032, 72), (333, 64, 8, 136, 264), (700, 1, 128, 264, 136),
          (1500, 3, 16, 200, 1160), (513, 5, 104, 72, 520), (8300, 2, 72, 136, 328), (8200, 70, 48, 72, 200),
          (256, 8, 24, 264, 520), (257, 8, 24, 264, 520), (200, 3, 128, 1032, 72)]


@pytest.mark.parametrize("T,L,r,n,d", SHAPES)
@pytest.mark.parametrize("full,pad", [(True, 8), (False, 0)])
def test_adapters(T, L, r, n, d, full, pad):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters case T={T} L={L} r={r} n={n} d={d} full={full}")
    c = _case(T, L, r, n, d, T + r, pad=pad, runs=full)
    scales, base = (c["scales"], c["base"]) if full else (None, None)
    y = X.adapters(c["x"], c["a"], c["b"], c["ids"], scales=scales, base=base)
    torch.cuda.synchronize()
    ref, mag = OG.adapters(c["x"], c["a"], c["b"], c["ids"], scales, base)
    within(y, ref, mag, adapter_rel(r, d), "y")
    if base is not None:
        off = (c["ids"] < 0) | (c["ids"] >= L)
        assert torch.equal(y[off], base[off])


@pytest.mark.parametrize("T,L,r,n,d", SHAPES)
@pytest.mark.parametrize("full,pad", [(True, 8), (False, 0)])
def test_gradients(T, L, r, n, d, full, pad):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters gradient case T={T} L={L} r={r} n={n} d={d} full={full}")
    c = _case(T, L, r, n, d, T + r, pad=pad, runs=full)
    scales, base = (c["scales"], c["base_dx"]) if full else (None, None)
    got = X.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"], scales=scales, base=base)
    torch.cuda.synchronize()
    ref, mag = OG.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"], scales, base)
    within(got["dx"], ref["dx"], mag["dx"], adapter_rel(r, n), "dx")
    within(got["da"], ref["da"], mag["da"], factor_rel(T, n), "da")
    within(got["db"], ref["db"], mag["db"], factor_rel(T, d), "db")


@pytest.mark.parametrize("T", [5, 100])
def test_in_place_of_the_base(T):
    from paper_2602_07265_amd import xshare as X
    c = _case(T, 4, 16, 264, 136, 3, pad=8)
    want = X.adapters(c["x"], c["a"], c["b"], c["ids"], scales=c["scales"], base=c["base"])
    got = X.adapters(c["x"], c["a"], c["b"], c["ids"], scales=c["scales"], base=c["base"],
                     out=c["base"])
    g = X.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"], base=c["base_dx"])
    h = X.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"], base=c["base_dx"],
                            out=dict(dx=c["base_dx"]))
    torch.cuda.synchronize()
    assert got is c["base"] and torch.equal(got, want)
    assert h["dx"] is c["base_dx"] and torch.equal(h["dx"], g["dx"])


@pytest.mark.parametrize("T", [6, 150])
def test_tokens_without_an_adapter_have_no_part(T):
    from paper_2602_07265_amd import xshare as X
    c = _case(T, 3, 16, 136, 264, 4, none=0.5)
    off = (c["ids"] < 0) | (c["ids"] >= 3)
    clean = {name: v.clone() for name, v in c.items()}
    c["x"][off], c["dy"][off] = NAN, float("inf")
    for s in (c, clean):
        s["y"] = X.adapters(s["x"], s["a"], s["b"], s["ids"], base=clean["base"])
        s["g"] = X.adapters_backward(s["dy"], s["x"], s["a"], s["b"], s["ids"])
    torch.cuda.synchronize()
    assert torch.equal(c["y"], clean["y"])
    for name in ("dx", "da", "db"):
        assert torch.equal(c["g"][name], clean["g"][name]), name
    assert (c["g"]["dx"][off] == 0).all()


@pytest.mark.parametrize("T", [0, 3, 90])
def test_no_tokens_or_no_adapters(T):
    from paper_2602_07265_amd import xshare as X
    c = _case(T, 3, 16, 136, 264, 4, none=1.0)
    y = X.adapters(c["x"], c["a"], c["b"], c["ids"], base=c["base"])
    z = X.adapters(c["x"], c["a"], c["b"], c["ids"])
    g = X.adapters_backward(c["dy"], c["x"], c["a"], c["b"], c["ids"])
    torch.cuda.synchronize()
    assert torch.equal(y, c["base"]) and (z == 0).all() and (g["dx"] == 0).all()
    assert (g["da"] == 0).all() and (g["db"] == 0).all()


def test_an_infinity_stays_in_its_token():
    from paper_2602_07265_amd import xshare as X
    for T in (8, 200):
        c = _case(T, 2, 16, 136, 264, 6, none=0.0)
        ref = X.adapters(c["x"], c["a"], c["b"], c["ids"])
        c["x"][3, 5] = float("inf")
        y = X.adapters(c["x"], c["a"], c["b"], c["ids"])
        torch.cuda.synchronize()
        other = torch.arange(T, device=DEV) != 3
        assert torch.equal(y[other], ref[other]) and not y[3].isfinite().any()


def test_one_workspace_and_the_same_bits_again():
    from paper_2602_07265_amd import xshare as X
    L, r, n, d = 6, 24, 264, 520
    ws = torch.empty(X.adapters_workspace_bytes(900, L, r, n, d, True), dtype=torch.uint8, device=DEV)
    for T in (900, 300, 65, 64, 2):
        c = _case(T, L, r, n, d, T)
        args = (c["x"], c["a"], c["b"], c["ids"])
        y = [X.adapters(*args, base=c["base"], **kw) for kw in ({}, dict(workspace=ws)) * 2]
        g = [X.adapters_backward(c["dy"], *args, **kw) for kw in ({}, dict(workspace=ws)) * 2]
        torch.cuda.synchronize()
        for i in range(1, 4):
            assert torch.equal(y[i], y[0])
            for name in ("dx", "da", "db"):
                assert torch.equal(g[i][name], g[0][name]), name


@pytest.mark.parametrize("r", [8, 24, 40, 48, 56, 72, 96, 104, 112, 120])
def test_ranks_between_the_tiles_with_every_row_used(r):
    from paper_2602_07265_amd import xshare as X
    T, L, n, d = 257, 2, 136, 72
    c = _case(T, L, r, n, d, r, none=0.0)
    need = X.adapters_workspace_bytes(T, L, r, n, d, True)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    args = (c["x"], c["a"], c["b"], c["ids"])
    y = X.adapters(*args, base=c["base"], workspace=ws[:need])
    got = X.adapters_backward(c["dy"], *args, workspace=ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 0xA5).all()
    within(y, *OG.adapters(*args, None, c["base"]), adapter_rel(r, d), "y")
    ref, mag = OG.adapters_backward(c["dy"], *args, None, None)
    within(got["dx"], ref["dx"], mag["dx"], adapter_rel(r, n), "dx")
    within(got["da"], ref["da"], mag["da"], factor_rel(T, n), "da")
    within(got["db"], ref["db"], mag["db"], factor_rel(T, d), "db")
