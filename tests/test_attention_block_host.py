"""What the attention block refuses, before any call of the library or of CUDA."""

from types import SimpleNamespace

import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from paper_2605_28803_gb300.attention import AttentionBlock

HEADS, KV, DIM, K = 4, 2, 64, 256


def make_block(batch=2, max_tokens=50, **kw):
    qkv = SimpleNamespace(N=(HEADS + 2 * KV) * DIM, K=K, xdt=Q.BF16, ydt=Q.BF16)
    o = SimpleNamespace(N=K, K=HEADS * DIM, xdt=Q.BF16, ydt=Q.BF16)
    return AttentionBlock(qkv, o, HEADS, KV, DIM, batch, max_tokens, page_size=16, device="cpu", **kw)


def tokens(n, k=K, dtype=torch.bfloat16):
    return torch.zeros(n, k, dtype=dtype)


@pytest.mark.parametrize("x,lens", [
    (tokens(8), [5, 4]), (tokens(10), [5, 4]),              # fewer and more rows than lens says
    (tokens(9), [9]), (tokens(9), [5, 4, 0]), (tokens(4), [5, -1]),
    (tokens(9, K - 8), [5, 4]), (tokens(9, dtype=torch.float32), [5, 4]), (tokens(9, dtype=torch.int8), [5, 4]),
    (tokens(K, 9).T, [5, 4]), (tokens(18)[::2], [5, 4]), (tokens(9).reshape(-1), [5, 4]),
    (tokens(51), [51, 0]), (torch.zeros(9, K, dtype=torch.bfloat16, device="meta"), [5, 4])])
def test_prompts_that_do_not_fit_are_refused(x, lens):
    block = make_block()
    with pytest.raises(ValueError):
        block.prefill(x, lens)
    assert block.lens == [0, 0]


@pytest.mark.parametrize("x", [tokens(3), tokens(4, K + 8), tokens(4, dtype=torch.float16), tokens(8)[::2], tokens(102)])
def test_steps_that_do_not_fit_are_refused(x):
    block = make_block()
    with pytest.raises(ValueError):
        block.step(x)
    assert block.lens == [0, 0]


@pytest.mark.parametrize("lens", [[11, 4], [10, 5], [10], [10, 4, 0], [-1, 4]])
def test_rewinds_to_tokens_that_are_not_there_are_refused(lens):
    block = make_block()
    block.lens = [10, 4]
    with pytest.raises(ValueError):
        block.rewind(lens)
    assert block.lens == [10, 4]
