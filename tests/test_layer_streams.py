"""Which stream and device the calls of DeviceLayer and DeviceBlock run on: a
stand-in for torch's streams records them (no GPU needed)."""
import contextlib

import numpy as np
import pytest
import torch

from paper_2608_10392_amd import _lib, ops
from paper_2608_10392_amd.layer import DeviceBlock, DeviceLayer

N, D, K, B, M = 4, 8, 2, 2, 4
CFG = dict(n_tokens=N, d_model=D, n_experts=K, n_blocks=B, block_width=M, mass_threshold=0.7, dtype="f32")


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Streams:
    """Streams by handle; 0 is the default stream. `seen` holds, for every
    workspace and every call of the library, the stream current then and (for
    calls) the handle it was given."""

    def __init__(self, monkeypatch):
        self.now, self.seen = Stream(0), []
        cuda = torch.cuda
        monkeypatch.setattr(cuda, "Stream", Stream)
        monkeypatch.setattr(cuda, "default_stream", lambda device=None: Stream(0))
        monkeypatch.setattr(cuda, "current_stream", lambda device=None: self.now)
        # as torch's: a handle of 0 counts as not given, a stream of torch's own comes back
        monkeypatch.setattr(cuda, "ExternalStream", lambda handle, device=None: Stream(handle or 0xABCD))
        monkeypatch.setattr(cuda, "stream", self.use)
        alloc = _lib.alloc_workspace
        monkeypatch.setattr(_lib, "alloc_workspace", lambda *a: (self.note("workspace"), alloc(*a))[1])
        for mod in (_lib, ops):
            for name in ("route", "layer_forward", "block_forward", "layer_backward", "stats", "diversity_loss",
                         "balance_loss", "residual_forward", "residual_backward"):
                if hasattr(mod, name):
                    monkeypatch.setattr(mod, name, lambda *a, name=name, stream=None, **k: self.note(name, stream))
                    monkeypatch.setattr(mod, name + "_workspace_size", lambda *a: 16, raising=False)

    def note(self, what, stream=None):
        handle = self.now.cuda_stream if stream is None else getattr(stream, "cuda_stream", stream)
        self.seen.append((what, self.now.cuda_stream, handle))

    @contextlib.contextmanager
    def use(self, stream):
        assert isinstance(stream, Stream)   # torch's takes no other
        was, self.now = self.now, stream
        yield
        self.now = was


def make():
    z = lambda *s: np.zeros(s, np.float32)
    dev = DeviceLayer(CFG, z(N, D), None, z(K + 1, D), z(B, D), z(K + 1, B * M, D), z(K + 1, D, B * M), device="cpu")
    block = DeviceBlock.__new__(DeviceBlock)
    block.layer, block.params, block.before, block.behind = dev, {}, None, None
    return dev, block


X = torch.zeros(N, D)
BLK = dict(norm="none", residual=True, ln_eps=1e-6)
NEW = dict(block_forward=lambda dev, block, **s: block.forward(X, **s),
           block_backward=lambda dev, block, **s: block.backward(X, X, {}, 0.5, **s),
           balance=lambda dev, block, **s: dev.balance_loss({}, **s),
           diversity=lambda dev, block, **s: dev.diversity_loss(0.5, X, **s))


@pytest.mark.parametrize("name", list(NEW))
def test_handles(name, monkeypatch):
    """A raw handle, 0 (the null stream) among them, is the stream that is used
    and that the call's memory belongs to; so is another object's."""
    streams, (dev, block) = Streams(monkeypatch), make()

    class Foreign:
        """Another library's stream."""
        cuda_stream = 78

    for given, handle in ((0, 0), (77, 77), (Foreign(), 78)):
        for now in (Stream(0), Stream(5)):
            streams.now, streams.seen = now, []
            NEW[name](dev, block, stream=given)
            assert streams.seen and {s[1:] for s in streams.seen} == {(handle, handle)}, streams.seen
            assert streams.now is now


OLD = dict(forward=lambda dev, *s, **k: dev.forward(*s, **k), route=lambda dev, *s, **k: dev.route(None, *s, **k),
           stats=lambda dev, *s, **k: dev.stats(*s, **k), backward=lambda dev, *s, **k: dev.backward(X, *s, **k),
           layer_block=lambda dev, *s, **k: dev.block_forward(BLK, None, *s, **k))


@pytest.mark.parametrize("name", list(OLD))
def test_layer_memory_belongs_to_the_stream(name, monkeypatch):
    """Workspaces and outputs of a call on another stream are allocated on that
    stream, whichever way it is given; without one, on the current stream."""
    streams = Streams(monkeypatch)
    for given, want in (((), 5), ((Stream(9),), 9), ((9,), 9), ((0,), 0)):
        for by_name in (False, True):
            dev, _ = make()
            streams.now, streams.seen = Stream(5), []
            OLD[name](dev, **dict(zip(("stream",), given))) if by_name else OLD[name](dev, *given)
            assert [s[0] for s in streams.seen].count("workspace") == 1
            assert {s[1:] for s in streams.seen} == {(want, want)}, streams.seen
    with pytest.raises(TypeError):
        OLD[name](dev, Stream(9), stream=Stream(9))


def test_the_other_arguments_keep_their_places(monkeypatch):
    streams, (dev, _) = Streams(monkeypatch), make()
    seen = []
    monkeypatch.setattr(_lib, "layer_forward", lambda *a, routing, stream: seen.append((routing is None, stream)))
    s = Stream(3)
    for call in (lambda: dev.forward(s, False), lambda: dev.forward(s, routing=False),
                 lambda: dev.forward(stream=s, routing=False), lambda: dev.forward(routing=False, stream=s)):
        assert call() is dev.Y and seen.pop() == (True, s)
    assert dev.forward() is dev.Y and seen.pop() == (False, None)
    out = object()
    assert dev.route(out, s) is out and dev.route() is dev.routing


@pytest.mark.parametrize("name", list(NEW) + list(OLD))
def test_the_device_of_the_layer_is_current(name, monkeypatch):
    """A layer on another device than the current one: the call runs with its
    device current, and afterwards the other one is again."""
    Streams(monkeypatch)
    now, seen = [0], []

    @contextlib.contextmanager
    def device(index):
        was, now[0] = now[0], index
        yield
        now[0] = was

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    dev, block = make()
    monkeypatch.setattr(Streams, "note", lambda self, what, stream=None: seen.append(now[0]))

    class OnTheSecond:
        """The layer's output as it would be on device 1."""
        def get_device(self):
            return 1
        dtype, shape, device = dev.Y.dtype, dev.Y.shape, dev.Y.device

    monkeypatch.setattr(torch, "empty_like", lambda t, **k: torch.empty(t.shape, dtype=t.dtype))
    dev.Y = OnTheSecond()
    (NEW[name] if name in NEW else lambda d, b: OLD[name](d))(dev, block)
    assert seen and set(seen) == {1} and now == [0]
