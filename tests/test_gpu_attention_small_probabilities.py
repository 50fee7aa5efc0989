"""Many keys that are each far below a leading one: together they count, so their probabilities must not be lost to float16's
smallest numbers."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu

KEYS = 1 << 18
LEAD = 16.90625  # the leading key's score: 2^24.39 in the probabilities' ratio


def expected(n):
    """The others' share, and its bound: probabilities and output of 11 bits, 2^-32 of the leading one absolutely for each key, float32
    sums of n / 64 steps."""
    one = float(np.exp(-LEAD))
    total = 1.0 + (n - 1) * one
    want = (n - 1) * one / total
    return want, want * (2.0 ** -11 + 2.0 ** -11 + n / 64 * 2.0 ** -23 + 2.0 ** -20) + n * 2.0 ** -32 / total + 2.0 ** -25


@pytest.mark.parametrize("others", [0, 299], ids=["shared", "alone"])  # sequences without tokens: the keys are then one CTA's
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_prompt_of_many_keys(dim, others):
    k, v = (torch.zeros(KEYS, 1, dim, dtype=torch.float16, device=H.DEV) for _ in range(2))
    q = torch.zeros(1, 1, dim, dtype=torch.float16, device=H.DEV)
    q[0, 0, 0], k[0, 0, 0] = 1.0, LEAD
    v[1:] = 1.0
    got = H.f64(H.prompt(q, k, v, [1] + [0] * others, [KEYS] + [0] * others, False, scale=1.0))
    Q.qvla_check_device(H.stream())
    want, tol = expected(KEYS)
    assert np.abs(got - want).max() <= tol, (got.ravel()[0], want, tol)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_cache_of_many_tokens(dim):
    page = 256
    pages = KEYS // page
    pool = np.zeros((pages, 1, page * (dim + 8)), np.uint8)
    kc, vc, ks, vs = A.pool_parts(pool, page, dim)
    kc[0, 0, 0, 0] = 1  # the first token's key: code 1 in channel 0
    ks[...], vs[...] = LEAD, 1.0
    vc[...] = 0x11
    vc[0, 0, 0] = 0
    p = H.Paged(np.random.default_rng(0), [0], 1, dim, page, False)
    device = torch.from_numpy(pool).to(H.DEV)
    p.device, p.cache = device, Q.Kv4Cache(device, pages, page, 1, dim, False)
    p.width, p.table_device = pages, H.ints(range(pages)).reshape(1, -1)
    q = torch.zeros(1, 1, dim, dtype=torch.float16, device=H.DEV)
    q[0, 0, 0] = 1.0
    want, tol = expected(KEYS)
    for ws in (0, None):  # without room for a split a warp has a quarter of the tokens
        got = H.f64(H.kv4(p, q, [1], [KEYS], True, scale=1.0, ws_bytes=ws))
        Q.qvla_check_device(H.stream())
        assert np.abs(got - want).max() <= tol, (ws, got.ravel()[0], want, tol)
