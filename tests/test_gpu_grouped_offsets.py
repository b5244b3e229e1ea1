"""Offsets that are none, at the sizes where tiles of 256 x 256 are split and joined: what they give is
not said, and nothing past the buffers, the workspace's among them, is touched."""
import pytest
import torch

from helpers import DEV, say
from test_gpu_grouped import SKEW, _case

pytestmark = pytest.mark.gpu
P = sum(SKEW)
TOP, LOW = 2 ** 31 - 1, -2 ** 31
# falling, groups over each other, past either end, all of the rows in every second group, extremes
BAD = [[0, 5000, 2000, 7000, 3000, P], [-5, 4000, 100, 8000, 50, 3 * P], [P, 0, P, 0, P, 0],
       [0, P, 0, P, 0, P], [TOP, LOW, 0, TOP, 5, TOP], [LOW, TOP, LOW, TOP, LOW, TOP]]
# (test_grouped_offsets checks that these run turns_kernel and join_kernel)
SIZES = [("linear", 2048, 4104), ("x", 2056, 4104), ("w", 264, 520)]


@pytest.mark.parametrize("what,n,k", SIZES)
@pytest.mark.parametrize("bad", range(len(BAD)))
def test_offsets_that_are_none_stay_inside_the_buffers(what, n, k, bad):
    from paper_2602_07265_amd import xshare as X
    say(f"offsets that are none: {what} n={n} k={k} {BAD[bad]}")
    counts, edges = (SKEW, BAD[bad]) if what != "w" else ([P], [BAD[bad][0], BAD[bad][1]])
    _, _, _, x, dy, w = _case(counts, n, k, 2)
    offsets = torch.tensor(edges, dtype=torch.int32, device=DEV)
    need = X.grouped_linear_workspace_bytes(P, len(counts), n, k)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    if what == "w":
        buf = torch.full((len(counts) + 2, n, k), 5.0, device=DEV)
        X.grouped_linear_backward_w(dy, x, offsets, out=buf[1:-1], workspace=ws[:need])
    else:
        buf = torch.full((P + 2, n if what == "linear" else k), 5.0, dtype=torch.bfloat16, device=DEV)
        if what == "linear":
            X.grouped_linear(x, w, offsets, y=buf[1:-1], workspace=ws[:need])
        else:
            X.grouped_linear_backward_x(dy, w, offsets, out=buf[1:-1], workspace=ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 0xA5).all() and (buf[0] == 5.0).all() and (buf[-1] == 5.0).all()
