"""Adapters of few tokens in one launch and in two, on both sides of every edge of the rule between them
(test_adapter_paths checks which are which)."""
import pytest
import torch

from group_bounds import adapter_rel, within
from helpers import say
from oracle import groups as OG
from test_gpu_adapters import _case

pytestmark = pytest.mark.gpu
ONE = [(1, 3, 16, 264, 8200), (3, 4, 40, 1032, 72), (5, 2, 48, 2056, 520), (1, 3, 48, 1000, 1360),
       (7, 3, 32, 2040, 2040), (1, 2, 24, 8200, 2056), (51, 2, 16, 4104, 8200), (128, 5, 8, 2056, 4104)]
TWO = [(1, 3, 24, 264, 8200), (1, 3, 48, 1000, 1368), (7, 3, 32, 2040, 2056), (9, 3, 56, 264, 520),
       (52, 2, 16, 4104, 8200), (1, 2, 64, 4096, 4096), (2, 4, 120, 136, 72)]


@pytest.mark.parametrize("T,L,r,n,d", ONE + TWO)
@pytest.mark.parametrize("based", [True, False])
def test_few_tokens(T, L, r, n, d, based):
    from paper_2602_07265_amd import xshare as X
    say(f"adapters of few tokens: T={T} L={L} r={r} n={n} d={d} based={based}")
    c = _case(T, L, r, n, d, T + r, pad=8 * based)
    args = (c["x"], c["a"], c["b"], c["ids"])
    scales, base = (c["scales"], c["base"]) if based else (None, None)
    y = X.adapters(*args, scales=scales, base=base)
    torch.cuda.synchronize()
    within(y, *OG.adapters(*args, scales, base), adapter_rel(r, d), "y")
    off = (c["ids"] < 0) | (c["ids"] >= L)
    if based:
        assert torch.equal(y[off], base[off])
        X.adapters(*args, scales=scales, base=base, out=base)
        torch.cuda.synchronize()
        assert torch.equal(base, y)
    else:
        assert (y[off] == 0).all()
