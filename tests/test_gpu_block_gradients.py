"""Inputs that require a gradient pass under torch.no_grad() and detached, with the same results."""
import numpy as np
import pytest
import torch

from helpers import DEV, say
from test_gpu_blocks import _weight, _x

pytestmark = pytest.mark.gpu


def test_no_grad_and_detached():
    from paper_2602_07265_amd import xshare as X
    say("gradient case no_grad and detached")
    rng = np.random.default_rng(3)
    h = torch.randn(5, 64, device=DEV, requires_grad=True)
    x = _x(rng, 5, 144).to(DEV).requires_grad_(True)
    q, s = (t.to(DEV) for t in _weight(rng, 100, 144))
    with torch.no_grad():
        a, y = X.gate(h, 4), X.block_linear(x, q, s)
    b, z = X.gate(h.detach(), 4), X.block_linear(x.detach(), q, s)
    assert torch.equal(a["ids"], b["ids"]) and torch.equal(a["w"], b["w"]) and torch.equal(y, z)
    with pytest.raises(ValueError, match="logits requires a gradient"):
        X.gate(h, 4)
    # weights that are parameters are quantised as any others: codes have no gradient
    X.block_quantize(x, 128)
    # and a gradient call takes the logits that the graph holds
    X.gate_backward(h, a["ids"], a["w"])
