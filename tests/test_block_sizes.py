"""Sizes past 32 bits, which the C ABI's int32 arguments would take for smaller ones: refused by
the binding before anything is allocated or called."""
import pytest
import torch

from paper_2602_07265_amd import xshare as X

BIG = (1 << 32) + 1


class OnGpu(torch.Tensor):
    """A tensor without memory that says it is on the GPU."""
    is_cuda = True


def _t(dtype, *shape):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)


def _refused(call):
    with pytest.raises(X.XShareError) as e:
        call()
    assert e.value.status == X.EUNSUPPORTED


@pytest.mark.parametrize("block_rows", [BIG, BIG + 127, -(1 << 40)])
def test_quantize_block_rows(block_rows):
    x = _t(torch.bfloat16, 300, 256)
    if block_rows > 0:
        _refused(lambda: X.block_quantize(x, block_rows))
    else:
        assert X._past_32_bits(block_rows)


def test_sizes_of_tensors():
    bf16, u8, f32, i32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
    _refused(lambda: X.block_quantize(_t(bf16, BIG, 16)))
    _refused(lambda: X.gate(_t(f32, BIG, 8), 2))
    _refused(lambda: X.gate_backward(_t(f32, BIG, 8), _t(i32, BIG, 2), _t(f32, BIG, 2)))
    _refused(lambda: X.block_linear(_t(bf16, BIG, 16), _t(u8, 8, 16), _t(f32, 1, 1)))
    _refused(lambda: X.block_linear(_t(bf16, 4, 16), _t(u8, BIG, 16), _t(f32, BIG, 1)))
    q, s = _t(u8, 2, BIG, 16), _t(f32, 2, BIG, 1)
    _refused(lambda: X.block_experts(_t(bf16, 4, 16), _t(i32, 4, 2), _t(f32, 4, 2), q, q, q, s, s, s))


def test_sizes_of_the_choice():
    h = _t(torch.float32, 4, 64)
    for kw in (dict(top_k=BIG + 3), dict(top_k=4, n_groups=BIG + 7),
               dict(top_k=4, n_groups=8, top_groups=BIG + 1)):
        _refused(lambda: X.gate(h, **kw))


def test_workspaces():
    assert X.block_linear_workspace_bytes(BIG, 16, 16) == 0
    assert X.block_experts_workspace_bytes(BIG, 2, 4, 256, 128) == 0
    assert X.block_experts_workspace_bytes(8, 2, BIG + 3, 256, 128) == 0
    assert X.block_linear_workspace_bytes(-1, 16, 16) == 0
