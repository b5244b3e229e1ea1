"""Calls on another stream than the current one: what they allocate belongs to that stream; calls
on another device than the current one: they run on their tensors'.  On the CPU, with stand-ins for
torch's streams and devices; the library is not called."""
import contextlib
import inspect

import pytest
import torch

from paper_2602_07265_amd import xshare as X


class Stream:
    def __init__(self, handle, device=0):
        self.cuda_stream, self.device = handle, torch.device("cuda", device)


class Out(torch.Tensor):
    """A tensor that says it is on the GPU and notes the streams that are recorded for it."""
    is_cuda = True

    def record_stream(self, stream):
        self.recorded = [*getattr(self, "recorded", []), stream]


@pytest.fixture
def streams(monkeypatch):
    now = [Stream(0)]

    @contextlib.contextmanager
    def use(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "stream", use)
    return now


def test_every_call_with_a_stream_is_ordered():
    calls = [f for f in vars(X).values() if inspect.isfunction(f)
             and f.__module__ == X.__name__ and not f.__name__.startswith("_")
             and "stream" in inspect.signature(f).parameters]
    assert len(calls) >= 18
    for f in calls:
        assert f.__code__ is X._placed(f).__code__, f.__name__


@pytest.mark.parametrize("shape", ["tensor", "tuple", "dict"])
def test_a_call_runs_with_its_stream_current(streams, shape):
    seen = []

    @X._placed
    def call(x, *, stream=None):
        seen.append((torch.cuda.current_stream(), stream))
        y = torch.zeros(2).as_subclass(Out)
        return y if shape == "tensor" else (y, 3) if shape == "tuple" else dict(y=y, n=3)

    first = lambda r: r if shape == "tensor" else r[0] if shape == "tuple" else r["y"]  # noqa: E731
    own, side = streams[0], Stream(7)
    y = first(call(1, stream=side))
    assert seen == [(side, side)] and y.recorded == [own] and streams == [own]
    for same in (None, own, Stream(0)):
        y = first(call(1, stream=same))
        assert seen[-1] == (own, same) and not hasattr(y, "recorded")


def test_a_stream_given_by_position(streams):
    @X._placed
    def call(x, stream=None):
        return torch.cuda.current_stream()

    side = Stream(7)
    assert call(1, side) is side and call(1, stream=side) is side and call(1) is streams[0]


class In(torch.Tensor):
    """A tensor of device 1."""

    def get_device(self):
        return 1


def test_a_call_runs_on_its_tensors_device(streams, monkeypatch):
    now = [0]

    @contextlib.contextmanager
    def use(device):
        now.append(device)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "device", use)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[-1], raising=False)

    @X._placed
    def call(x, more=None, *, stream=None):
        return now[-1]

    x = torch.zeros(2).as_subclass(In)
    assert call(x) == 1 and call(x=x) == 1 and call(more=3, x=x) == 1 and now == [0]
    assert call(torch.zeros(2)) == 0 and call(None) == 0 and call(3) == 0
    now[0] = 1
    assert call(x) == 1
    # and not on a stream of another device
    with pytest.raises(ValueError, match="cuda:1"):
        call(x, stream=Stream(7, 0))
    call(x, stream=Stream(7, 1))
