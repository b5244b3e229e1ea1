"""Adapters at sizes where their kernels' loops go round again (test_adapter_paths checks that these
do): many columns of a workgroup, whose next ones are loaded while the last are stored, and adapters with
more tokens than a chunk of the factors' gradients, some with very many and others with none."""
import pytest
import torch

from group_bounds import adapter_rel, factor_rel, within
from helpers import DEV, say
from oracle import groups as OG
from test_gpu_adapters import _case

pytestmark = pytest.mark.gpu
# more columns than a wave's first in the forward call, in the backward call
WIDE = [(3000, 2, 16, 4104, 2056), (4000, 2, 32, 3080, 520), (8200, 1, 24, 8200, 72)]
WIDE_BACK = [(3000, 2, 24, 264, 4104), (4000, 2, 8, 520, 3080)]
# one adapter with most of the tokens
HEAVY = [(9000, 64, r, 200, 232) for r in (8, 32, 64, 120)] + [(4700, 70, 16, 136, 264)]
MOST = 0.6
# as many adapters as there may be, about as many of which have tokens as not; the shortest rows
MANY = [(300, 1024, 8, 64, 72), (300, 512, 8, 64, 72), (1500, 1024, 16, 136, 72), (5000, 1000, 40, 72, 136)]
SHORT = [(300, 3, r, n, d) for r in (8, 32, 40, 128) for n, d in ((8, 8), (8, 16), (136, 8))]


def _check(c, T, r, n, d, based):
    from paper_2602_07265_amd import xshare as X
    args = (c["x"], c["a"], c["b"], c["ids"])
    base, base_dx = (c["base"], c["base_dx"]) if based else (None, None)
    y = X.adapters(*args, scales=c["scales"], base=base)
    got = X.adapters_backward(c["dy"], *args, scales=c["scales"], base=base_dx)
    torch.cuda.synchronize()
    within(y, *OG.adapters(*args, c["scales"], base), adapter_rel(r, d), "y")
    ref, mag = OG.adapters_backward(c["dy"], *args, c["scales"], base_dx)
    within(got["dx"], ref["dx"], mag["dx"], adapter_rel(r, n), "dx")
    within(got["da"], ref["da"], mag["da"], factor_rel(T, n), "da")
    within(got["db"], ref["db"], mag["db"], factor_rel(T, d), "db")
    if based:                                          # the same bits in place of the base
        X.adapters(*args, scales=c["scales"], base=base, out=base)
        h = X.adapters_backward(c["dy"], *args, scales=c["scales"], base=base_dx,
                                out=dict(dx=base_dx))
        torch.cuda.synchronize()
        assert torch.equal(base, y)
        for name in ("dx", "da", "db"):
            assert torch.equal(h[name], got[name]), name


@pytest.mark.parametrize("T,L,r,n,d", WIDE + WIDE_BACK)
@pytest.mark.parametrize("based", [True, False])
def test_many_columns(T, L, r, n, d, based):
    say(f"adapters of many columns: T={T} L={L} r={r} n={n} d={d} based={based}")
    _check(_case(T, L, r, n, d, T + r, pad=8 * based), T, r, n, d, based)


def heavy_ids(T, L, seed):
    """Most tokens with adapter 5, no token with 9, some without one."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(-1, L, (T,), generator=g)
    ids = torch.where(torch.rand(T, generator=g) < MOST, torch.full_like(ids, 5), ids)
    return torch.where(ids == 9, torch.full_like(ids, 5), ids).to(torch.int32)


@pytest.mark.parametrize("T,L,r,n,d", HEAVY)
def test_an_adapter_with_most_tokens(T, L, r, n, d):
    say(f"adapters, most tokens of one: T={T} L={L} r={r} n={n} d={d}")
    c = _case(T, L, r, n, d, T + r)
    c["ids"] = heavy_ids(T, L, r).to(DEV)
    _check(c, T, r, n, d, False)


@pytest.mark.parametrize("T,L,r,n,d", MANY + SHORT)
def test_many_adapters_and_short_rows(T, L, r, n, d):
    say(f"adapters, many or of short rows: T={T} L={L} r={r} n={n} d={d}")
    _check(_case(T, L, r, n, d, T + r, pad=8), T, r, n, d, True)
