"""A gradient that is itself to be differentiated: the backward calls record nothing, so they refuse an
incoming gradient that requires one while autograd is on, before anything is allocated or called.  The
other operands may be a program's parameters: their first gradients are what the calls give."""
import pytest
import torch

from paper_2602_07265_amd import xshare as X
from test_block_sizes import OnGpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _t(dtype, *shape, grad=False):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu).requires_grad_(grad)


def _calls(grad, others=False):
    """Each backward call: its incoming gradient's name and the call, whose sizes are none (a
    reduction of 12, a rank of 12, 33 ranks), so that past the binding the library refuses it."""
    o, p = dict(rows=_t(I32, 4, 33)), others
    return {
        "gate_backward": ("dw", lambda: X.gate_backward(_t(F32, 4, 8, grad=p), _t(I32, 4, 33),
                                                        _t(F32, 4, 33, grad=grad))),
        "dispatch_backward": ("drows", lambda: X.dispatch_backward(_t(BF, 132, 16, grad=grad), o)),
        "combine_backward": ("dy", lambda: X.combine_backward(
            _t(BF, 4, 16, grad=grad), _t(BF, 132, 16, grad=p), _t(F32, 4, 33, grad=p), o)),
        "grouped_linear_backward_x": ("dy", lambda: X.grouped_linear_backward_x(
            _t(BF, 4, 12, grad=grad), _t(BF, 2, 12, 16, grad=p), _t(I32, 3))),
        "grouped_linear_backward_w": ("dy", lambda: X.grouped_linear_backward_w(
            _t(BF, 4, 12, grad=grad), _t(BF, 4, 16, grad=p), _t(I32, 3))),
        "adapters_backward": ("dy", lambda: X.adapters_backward(
            _t(BF, 4, 8, grad=grad), _t(BF, 4, 16, grad=p), _t(BF, 2, 12, 16, grad=p),
            _t(BF, 2, 8, 12, grad=p), _t(I32, 4)))}


@pytest.mark.parametrize("name", list(_calls(False)))
def test_a_second_gradient_is_not_dropped_without_a_word(name):
    what, call = _calls(True)[name]
    with pytest.raises(ValueError, match=f"{what} requires a gradient"):
        call()


@pytest.mark.parametrize("name", list(_calls(False)))
def test_without_autograd_and_with_parameters_they_pass(name, monkeypatch):
    monkeypatch.setattr(X, "_stream_of", lambda x, stream: None)    # (there is no GPU to ask)

    def reaches_the_library(call):
        with pytest.raises(X.XShareError) as e:
            call()
        assert e.value.status in (X.EINVAL, X.EUNSUPPORTED)
    with torch.no_grad():
        reaches_the_library(_calls(True, others=True)[name][1])
    reaches_the_library(_calls(False, others=True)[name][1])
