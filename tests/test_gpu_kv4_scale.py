"""The cache kernel's scales are max / 7 rounded once, and its codes the exact quotient's, for every float16 significand."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from tests import attention_helpers as H
from tests.test_gpu_kv4_cache import append, stored
from tests.test_kv4_scale_host import TOPS, heads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scales_of_every_significand(dim):
    x = torch.from_numpy(heads(dim)).reshape(len(TOPS), 1, dim).to(H.DEV)
    p = H.Paged(np.random.default_rng(dim), [len(TOPS)], 1, dim, 64, False)
    append(p, x, 2 * x, [len(TOPS)], [0])
    pool = p.device.cpu().numpy()
    _, _, ks, vs = A.pool_parts(pool, p.page, dim)
    pos = np.arange(len(TOPS))
    at = p.table[0, pos // 64], 0, pos % 64
    want = TOPS / np.float32(7.0)  # one float32 division
    assert np.array_equal(ks[at], want) and np.array_equal(vs[at], 2 * want)
    assert np.array_equal(pool, stored(p, x, 2 * x, [len(TOPS)], [0]))
