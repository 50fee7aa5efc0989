"""The attention block's sequences are apart: what one gets does not depend on its neighbours' pasts."""

import numpy as np
import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H
from tests.test_gpu_attention_block import DIM, K, KV, heads_of, linear, make_block

pytestmark = pytest.mark.gpu


def tokens(seed, n):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((n, K), dtype=np.float32)).to(torch.bfloat16).to(H.DEV)


def read_back(block, b, n):
    k, v = (torch.empty(n, KV, DIM, dtype=torch.bfloat16, device=H.DEV) for _ in range(2))
    Q.qvla_kv4_gather(block.cache, 1, H.ints([0, n]), n, block.table[b: b + 1], block.width, None, k, v, Q.BF16, H.stream())
    return k, v


@pytest.mark.parametrize("causal", [True, False])
def test_a_prompt_that_starts_beside_one_that_continues(causal):
    block = make_block(5, 4)
    block.prefill(tokens(6, 61), [20, 0, 41, 0], causal)
    x = tokens(7, 45)
    got = block.prefill(x, [5, 30, 0, 10], causal)
    assert block.lens == [25, 30, 41, 10]
    q, k, v = heads_of(linear(block.qkv, x))
    a = [H.prompt(q[:5], *read_back(block, 0, 25), [5], [25], causal)]  # continues: over what the cache gives back
    for new in (slice(5, 35), slice(35, 45)):                           # start: over their own keys and values
        n = new.stop - new.start
        a.append(H.prompt(q[new], k[new], v[new], [n], [n], causal))
    assert torch.equal(got, linear(block.o, torch.cat(a).reshape(45, -1)))
    Q.qvla_check_device(H.stream())


def test_calls_on_different_streams_run_one_after_the_other():
    """A call on a stream of its own finds what the latest one stored, although that one's stream is still held up."""
    x = [tokens(8 + i, 3 * n) for i, n in enumerate((40, 1, 1, 30, 2))]
    block, want = make_block(9, 3), []
    for i, t in enumerate(x):
        want.append(block.prefill(t, [len(t) // 3] * 3) if i in (0, 3) else block.step(t))
    block, got = make_block(9, 3), []
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for i, (t, stream) in enumerate(zip(x, streams)):
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)  # some 10 ms
            got.append(block.prefill(t, [len(t) // 3] * 3) if i in (0, 3) else block.step(t))
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_a_denoising_loop_over_one_observation():
    """Every step's action tokens see the observation and one another, and none of an earlier step."""
    observation, steps = tokens(20, 60 + 33), [tokens(21 + t, 2 * 9) for t in range(4)]
    block = make_block(11, 2)
    block.prefill(observation, [60, 33], causal=False)
    for x in steps:
        got = block.step(x, causal=False)
        block.rewind([60, 33])
        alone = make_block(11, 2)
        alone.prefill(observation, [60, 33], causal=False)
        assert torch.equal(got, alone.step(x, causal=False))
    block.rewind([0, 33])  # a sequence ends, and another takes its place
    x = tokens(30, 17)
    assert torch.equal(block.prefill(x, [17, 0]), make_block(11, 2).prefill(x, [17, 0]))
    assert block.lens == [17, 33]
    Q.qvla_check_device(H.stream())
