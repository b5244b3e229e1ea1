"""xshare_gate_backward where a score nears 0 or 1: the gradient relative to itself.

A sigmoid's slope s (1 - s) = e / (1 + e)^2 with e = exp(-|h|): an exponential (2 ulp) and four
more roundings, within 16 * 2^-24 of the exact slope."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from test_oracle_gate_gradient import slope

pytestmark = pytest.mark.gpu
TOL = 16 * 2.0 ** -24


@pytest.mark.parametrize("N", [8, 64, 200, 1000])
def test_gradient_of_saturated_sigmoids(N):
    from paper_2602_07265_amd import xshare as X
    say(f"gate gradient case saturated N={N}")
    h = np.concatenate([np.linspace(-80, 80, 4 * N).reshape(4, N),
                        np.linspace(12, 30, N)[None]]).astype(np.float32)
    rng = np.random.default_rng(N)
    k = 8
    ids = np.stack([rng.permutation(N)[:k] for _ in range(5)]).astype(np.int32)
    dw = rng.normal(0, 1, (5, k)).astype(np.float32)
    d = X.gate_backward(torch.from_numpy(h).to(DEV), torch.from_numpy(ids).to(DEV),
                        torch.from_numpy(dw).to(DEV), score="sigmoid", renormalize=False)
    ref = np.zeros((5, N))
    np.put_along_axis(ref, ids.astype(np.int64), dw.astype(np.float64), 1)
    ref *= slope(h)
    assert (np.abs(d.cpu().numpy() - ref) <= TOL * np.abs(ref)).all()
