"""What the 4-bit MLP block refuses because it lies on another device: shown with stand-ins for tensors, before any call of the
library."""

from types import SimpleNamespace

import pytest
import torch

from paper_2605_28803_gb300 import fp4_mlp
from paper_2605_28803_gb300 import qvla as Q
from tests.test_fp4_mlp_host import block, norm
from tests.test_fp4_mlp_streams_host import Buffer, Stream

CUDA0, CUDA1 = torch.device("cuda", 0), torch.device("cuda", 1)


def tokens(device, dtype=torch.bfloat16):
    return SimpleNamespace(shape=(3, 128), dtype=dtype, device=device, is_contiguous=lambda: True)


@pytest.fixture
def current(monkeypatch):
    """A machine of two GPUs; buffers lie on cuda:0, and current(n) makes device n the current one."""
    at = [0]
    monkeypatch.setattr(fp4_mlp.torch, "empty", lambda *a, **kw: Buffer())
    monkeypatch.setattr(fp4_mlp.torch.cuda, "current_device", lambda: at[0])
    streams = [Stream(), Stream()]
    monkeypatch.setattr(fp4_mlp.torch.cuda, "current_stream", lambda device=None: streams[at[0] if device is None else device.index])
    monkeypatch.setattr(fp4_mlp.torch.cuda, "is_current_stream_capturing", lambda: False)
    return lambda n: at.__setitem__(0, n)


def test_inputs_on_another_device(current):
    b = block()
    assert b._check(tokens(CUDA0), tokens(CUDA0)) == 3
    for bad in ((tokens(CUDA1), tokens(CUDA0)), (tokens(CUDA0), tokens(CUDA1)), (tokens(torch.device("cpu")), tokens(CUDA0))):
        with pytest.raises(ValueError, match="must lie on cuda:0"):
            b._check(*bad)


def test_a_call_while_another_device_is_current(current):
    b = block()
    current(1)
    with pytest.raises(ValueError, match="the current device"):
        b._check(tokens(CUDA0), tokens(CUDA0))
    current(0)
    assert b._check(tokens(CUDA0), tokens(CUDA0)) == 3


def test_the_stream_is_that_of_the_blocks_device(current):
    current(1)  # (made with device="cuda:0", say)
    b = block()
    current(0)
    stream = b._stream()
    assert stream is b._last and stream.waited == []


@pytest.mark.parametrize("which", ["before", "after"])
def test_norms_of_another_device(which):
    elsewhere = Q.BlockNorm(Q.NORM_RMS, Q.BF16, pre_weight=torch.zeros(128, dtype=torch.bfloat16))  # on the CPU, the block on `meta`
    with pytest.raises(ValueError, match="must lie on"):
        fp4_mlp.Fp4Mlp(*_layers(), **{"before": norm(), "after": norm(), which: elsewhere}, max_tokens=4, device="meta")
    assert block(**{which: elsewhere}) is not None


def _layers():
    from tests.test_fp4_mlp_host import layer
    return layer(256, 128, True), layer(128, 256, False)
