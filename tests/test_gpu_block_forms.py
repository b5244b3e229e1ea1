"""block_linear in the form of 16 weight rows and 32 tokens, which the rule chooses in few places
(test_block_launches checks that it does here): lengths that end inside a block, rows past the last
whole tile."""
import numpy as np
import pytest

from helpers import DEV, say
from test_gpu_blocks import _check_linear, _weight, _x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,T,n,k", [("16x32", 90, 1350, 400), ("16x32", 81, 1360, 128),
                                        ("16x32", 96, 1345, 1040)])
def test_linear(form, T, n, k):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(T + n)
    x, (q, s) = _x(rng, T, k), _weight(rng, n, k)
    say(f"linear case form {form} T={T} n={n} k={k}")
    codes, scales = X.block_quantize(x.to(DEV))
    _check_linear(x, q, s, X.block_linear(codes, q.to(DEV), s.to(DEV), x_scale=scales))
