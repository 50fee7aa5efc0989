"""The streams of the 4-bit MLP block, with stand-ins for streams and buffers: what its first call and the later ones wait for, and
which buffers the allocator is told of."""

import pytest
import torch

from paper_2605_28803_gb300 import fp4_mlp
from tests.test_fp4_mlp_host import block

BUFFERS = ("codes", "scales", "row_scales", "hidden", "out", "next", "work")
HERE = torch.device("cuda", 0)


class Stream:
    def __init__(self):
        self.waited = []

    def wait_stream(self, other):
        self.waited.append(other)


class Buffer:
    is_cuda, device = True, HERE

    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream)


@pytest.fixture
def on(monkeypatch):
    """on(stream) makes it the current one."""
    monkeypatch.setattr(fp4_mlp.torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(fp4_mlp.torch, "empty", lambda *a, **kw: Buffer())
    return lambda stream: monkeypatch.setattr(fp4_mlp.torch.cuda, "current_stream", lambda device=None: stream)


def test_the_first_call_waits_for_the_stream_of_the_construction(on):
    made, first, second = Stream(), Stream(), Stream()
    on(made)
    b = block()
    on(first)
    assert b._stream() is first and first.waited == [made]
    assert all(getattr(b, name).streams == [first] for name in BUFFERS)
    assert b._stream() is first and first.waited == [made]  # nothing new
    on(second)
    assert b._stream() is second and second.waited == [first]
    assert all(getattr(b, name).streams == [first, second] for name in BUFFERS)


def test_calls_on_the_stream_of_the_construction_wait_for_nothing(on):
    made = Stream()
    on(made)
    b = block()
    assert b._stream() is made and made.waited == []
    assert all(getattr(b, name).streams == [] for name in BUFFERS)
