"""Which stream's memory the binding takes for tensors that a call makes, seen
from the host: no GPU."""
import contextlib

import pytest

S = pytest.importorskip("paper_2608_03228_amd.saki")
torch = pytest.importorskip("torch")


class Tensor:
    def __init__(self, stream):
        self.stream, self.used_on = stream, []

    def record_stream(self, stream):
        self.used_on.append(stream)


class Torch:
    """What the binding uses of torch to make a tensor."""
    uint8 = torch.uint8

    def __init__(self):
        self.cuda = self
        self.now = "current"

    def current_stream(self, device=None):
        return self.now

    @contextlib.contextmanager
    def stream(self, stream):
        was, self.now = self.now, stream
        yield
        self.now = was

    def empty(self, shape, dtype=None, device=None):
        return Tensor(self.now)


def test_new_tensors_belong_to_the_stream_that_writes_them(monkeypatch):
    """A block that the current stream's pool hands out may still be read by what
    is queued there; a call on another stream, which waits for none of that,
    takes its memory from its own pool."""
    fake = Torch()
    monkeypatch.setattr(S, "_torch_mod", fake)
    t = S._new("side", (3,), torch.uint8, "cuda:0")
    assert t.stream == "side" and fake.now == "current"
    assert t.used_on == ["current"]  # the caller's, who reads it after waiting
    t = S._new("side", (3,), torch.uint8, "cuda:0", result=False)
    assert t.stream == "side" and t.used_on == []  # no other stream keeps a workspace back
    t = S._new(None, (3,), torch.uint8, "cuda:0")
    assert t.stream == "current" and t.used_on == []


class Stream:
    def __init__(self, device_index):
        self.device_index, self.cuda_stream = device_index, 4096 + device_index


def test_streams_of_another_device_are_refused(monkeypatch):
    """The serving calls check that tensors lie on the current device, on which
    kernels are launched and new tensors made: its streams alone are taken."""
    monkeypatch.setattr(S, "_torch_mod", Torch())
    monkeypatch.setattr(S, "_get_device", lambda: 0)
    assert S._current(Stream(0))[1:] == (0, 4096)
    with pytest.raises(ValueError, match="stream is on cuda:1"):
        S._current(Stream(1))
