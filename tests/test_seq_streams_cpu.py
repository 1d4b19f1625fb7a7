"""Streams of the token-sequence calls without a GPU: tensors on the host, a
library that only notes its arguments, and a mode that notes on which stream
each torch operation is issued."""
import contextlib
from types import SimpleNamespace

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2103_08802_gb300 import seq, seqnet


class Issued(TorchDispatchMode):
    """(operation, stream) of everything torch does."""

    def __init__(self, world):
        super().__init__()
        self.world, self.ops = world, []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.ops.append((func.overloadpacket.__name__, self.world.current))
        return func(*args, **(kwargs or {}))

    def streams_of(self, *names):
        return [s for n, s in self.ops if n in names]


@pytest.fixture
def world(monkeypatch):
    """current: the handle of torch's current stream; calls: (entry point, stream) as the library sees them."""
    w = SimpleNamespace(current=1, calls=[], other=SimpleNamespace(cuda_stream=2))

    @contextlib.contextmanager
    def on(stream):
        before, w.current = w.current, stream.cuda_stream
        yield
        w.current = before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if not name.endswith(("_bytes", "_size")):
                    w.calls.append((name, args[-1]))
                return 0
            return call

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # what a host tensor's get_device() is
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: SimpleNamespace(cuda_stream=w.current))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: w.current, raising=False)
    monkeypatch.setattr(seq, "load", Lib)
    return w


def test_rows_of_dout_are_copied_on_the_stream_of_the_call(world):
    """A dout whose rows cannot be viewed as a matrix is copied; on any other stream the copy would race with the call."""
    ids, dout = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, 3, 8).transpose(0, 1)
    for stream, handle in ((world.other, 2), (None, 1)):
        with Issued(world) as seen:
            seq.embed_grad(ids, dout, vocab=5, stream=stream)
        copies = seen.streams_of("clone", "copy_", "contiguous", "_to_copy")
        assert copies and set(copies) == {handle}
        assert set(seen.streams_of("empty", "empty_like", "new_empty")) <= {handle}
        assert world.calls.pop() == ("pnn_embed_backward", handle)


def test_the_network_runs_on_the_current_stream(world, monkeypatch):
    """Its convolutions (on the legacy default stream unless told otherwise) beside its sequence operators."""
    def conv_run(mode, instances, impl="auto", stream=None, repeat=0):
        world.calls.append((mode, 0 if stream is None else stream.cuda_stream))
    monkeypatch.setattr(seqnet.pnn, "conv_run", conv_run)
    net = object.__new__(seqnet.SeqNet)
    net.vocab, net.width, net.layers, net.heads, net.scale = 16, 8, 2, 8, 1.0
    net.params = {k: torch.zeros(16 if k in ("embed", "out") else 8, 8) for k in ("embed", "out", "z0", "x0", "o0", "z1", "x1", "o1")}
    x = torch.zeros(2, 3, dtype=torch.int32)
    ids, teacher = torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, 4)
    with torch.cuda.stream(world.other):
        net.forward(x)
        net.train_step(0.1, x, ids, teacher, labels=x)
        net.step(x[:, 0].contiguous(), [torch.zeros(2, 8), torch.zeros(2, 8)])
    assert len(world.calls) > 30 and {s for _, s in world.calls} == {2}
