"""One workspace, of the largest batch, for calls of any size: the results of calls with their own,
and no byte outside of what the size itself asks for."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from test_gpu_blocks import _expert_weights, _routing, _x
from test_gpu_guards import OUT_FILL, Guarded

pytestmark = pytest.mark.gpu


# few-row gate/up up to 16 rows an expert and then tiles (of few experts); one expert as a shared one;
# tiles of 32 and of 128; one token's own form and past its limit
@pytest.mark.parametrize("E,k,d,f,sizes", [
    (8, 2, 256, 1408, (130, 68, 67, 40, 33, 32, 3, 2, 1)), (1, 1, 256, 4096, (40, 17, 16, 8, 1)),
    (100, 4, 528, 272, (330, 300, 299, 60, 24, 1)), (5, 4, 96, 8208, (24, 20, 1)),
    (40, 8, 272, 144, (130, 85, 84, 45, 44, 2, 1))])
def test_experts_in_the_largest_batchs_workspace(E, k, d, f, sizes):
    from paper_2602_07265_amd import xshare as X
    rng = np.random.default_rng(E + f)
    mats = [(q.to(DEV), s.to(DEV)) for q, s in _expert_weights(rng, E, d, f)]
    x = _x(rng, sizes[0], d).to(DEV)
    ids, w = _routing(rng, sizes[0], E, k)
    ids = torch.from_numpy(ids.astype(np.int32)).to(DEV)
    w = torch.from_numpy(w.astype(np.float32)).to(DEV)
    big = torch.empty(X.block_experts_workspace_bytes(sizes[0], k, E, d, f), dtype=torch.uint8,
                      device=DEV)

    def call(T, **kw):
        return X.block_experts(x[:T], ids[:T], w[:T], *(m[0] for m in mats),
                               *(m[1] for m in mats), **kw).view(torch.int16)

    for T in sizes:
        say(f"workspace case T={T} E={E} k={k} d={d} f={f}")
        need = X.block_experts_workspace_bytes(T, k, E, d, f)
        own = Guarded(need, OUT_FILL)
        a = call(T, workspace=own.view(torch.uint8, (need,)))
        b = call(T, workspace=big)
        torch.cuda.synchronize()
        assert own.intact() and torch.equal(a, b)
