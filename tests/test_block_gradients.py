"""Inputs that require a gradient: the calls record none, so they refuse them while autograd would
expect one, before anything is allocated or called."""
import pytest
import torch

from paper_2602_07265_amd import xshare as X
from test_block_sizes import OnGpu


def _t(dtype, *shape, grad=False):
    t = torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)
    return t.requires_grad_(grad)


def _calls():
    bf16, u8, f32, i32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
    q, s, ids = _t(u8, 2, 16, 16), _t(f32, 2, 1, 1), _t(i32, 4, 2)
    return {"logits": lambda: X.gate(_t(f32, 4, 8, grad=True), 2),
            "x of linear": lambda: X.block_linear(_t(bf16, 4, 16, grad=True), q[0], s[0]),
            "x of experts": lambda: X.block_experts(_t(bf16, 4, 16, grad=True), ids,
                                                    _t(f32, 4, 2), q, q, q, s, s, s),
            "w of experts": lambda: X.block_experts(_t(bf16, 4, 16), ids,
                                                    _t(f32, 4, 2, grad=True), q, q, q, s, s, s)}


@pytest.mark.parametrize("name", list(_calls()))
def test_a_gradient_is_not_dropped_without_a_word(name):
    with pytest.raises(ValueError, match=f"{name.split()[0]} requires a gradient"):
        _calls()[name]()


def test_without_autograd_they_pass():
    t = _t(torch.float32, 4, 8, grad=True)
    with torch.no_grad():
        X._no_gradient(t, "t", "")
    X._no_gradient(t.detach(), "t", "")
