"""The 4-bit MLP block made on one stream and called first on another, with work of both streams under way."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from paper_2605_28803_gb300.fp4_mlp import Fp4Mlp
from tests import gpu_helpers as G
from tests.test_gpu_fp4_mlp import Setup

pytestmark = pytest.mark.gpu
BUFFERS = ("codes", "scales", "row_scales", "hidden", "out", "next", "work")
DELAY = 20_000_000  # cycles, about 10 ms


def again(s, tokens):
    """Another block of the same layers and norms."""
    return Fp4Mlp(s.gate_up, s.down, *s.norms, tokens, s.block.rdt)


def test_the_first_call_waits_for_what_the_constructing_stream_still_does():
    s = Setup(F.NV, "bf16", "bf16", 512, 1024, 512, 1024, False, 0, 300)
    r, y = s.inputs(300)
    want_r = r.clone()
    want = s.block(want_r, y).clone()
    side, rr = torch.cuda.Stream(), r.clone()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # the block's memory is what work of this stream still writes when the call on the other one is made
    sizes = [getattr(s.block, name).nbytes for name in BUFFERS]
    earlier = [torch.empty(n, dtype=torch.uint8, device=G.DEV) for n in sizes]
    torch.cuda._sleep(DELAY)
    for t in earlier:
        t.fill_(0xFF)
    places = {t.data_ptr() for t in earlier}
    del earlier, t
    block = again(s, 300)
    assert places & {getattr(block, name).data_ptr() for name in BUFFERS}  # (else this shows nothing)
    with torch.cuda.stream(side):
        got = block(rr, y).clone()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(rr, want_r)
    Q.qvla_check_device(G.stream())


def test_a_dropped_block_keeps_its_buffers_until_the_other_stream_is_done():
    s = Setup(F.MX, "f16", "f32", 512, 1024, 512, 1024, False, 0, 300)
    r, y = s.inputs(300)
    want_r = r.clone()
    want = s.block(want_r, y).clone()
    side, rr = torch.cuda.Stream(), r.clone()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    block = again(s, 300)
    places = [(getattr(block, name).data_ptr(), getattr(block, name).nbytes) for name in BUFFERS]
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
        got = block(rr, y)
    del block
    later = [torch.full((n,), 0xFF, dtype=torch.uint8, device=G.DEV) for _, n in places]
    with torch.cuda.stream(side):
        got = got.clone()
    torch.cuda.synchronize()
    assert not {p for p, _ in places} & {t.data_ptr() for t in later}
    assert torch.equal(got, want) and torch.equal(rr, want_r)
    Q.qvla_check_device(G.stream())
