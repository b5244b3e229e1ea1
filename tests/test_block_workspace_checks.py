"""What the block-scaled FP8 calls refuse of a workspace: on the host, before any HIP call."""
import ctypes

import pytest
import torch

import test_abi_blocks as A
from paper_2602_07265_amd import xshare as X


@pytest.mark.parametrize("shift", [1, 2, 4, 8])
def test_workspaces_off_their_alignment(shift):
    ws = ctypes.c_void_p((1 << 20) + shift)
    assert A._linear(ws=ws) == X.EINVAL
    assert A._experts(ws=ws) == X.EINVAL
    assert A._experts(ws=ws, ws_bytes=16) == X.EWORKSPACE


def test_workspaces_that_hold_less_than_their_elements():
    dev = torch.device("cpu")
    assert X._workspace(dev, torch.empty(300, dtype=torch.uint8)) == 300
    assert X._workspace(dev, torch.empty(300)) == 1200
    for t in (torch.empty(1, dtype=torch.uint8).expand(1 << 30),
              torch.empty(64, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            X._workspace(dev, t)
    with pytest.raises(ValueError, match="is on"):
        X._workspace(torch.device("cuda", 0), torch.empty(300))
