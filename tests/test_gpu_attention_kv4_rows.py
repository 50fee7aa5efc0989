"""Attention over the 4-bit cache under the row-wise bound: splits and joins of long, ragged and many contexts, and rotated queries
whose last bits count."""

import numpy as np
import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests import attention_bounds as B
from tests import attention_helpers as H
from tests.test_attention_bounds_host import sharp_queries

pytestmark = pytest.mark.gpu


def q_unit(p, q):
    """Of the rounding that queries get: none without a rotation, two float16 parts of a rotated float16 one, one of a bfloat16 one."""
    return 0.0 if not p.rotate else 2.0 ** -21 if q.dtype == torch.float16 else 2.0 ** -11


def check(p, q, lens_q, lens_k, causal, scale=None, sizes=(None,), **kw):
    want, tol = B.statement(p, q, lens_q, lens_k, causal, scale, q_unit(p, q), **kw)
    for ws in sizes:
        got = H.f64(H.kv4(p, q.to(H.DEV), lens_q, lens_k, causal, scale, ws_bytes=ws))
        Q.qvla_check_device(H.stream())
        assert not np.isnan(got).any()
        worst = np.max(B.error(got, want) - tol)
        assert worst <= 0, (ws, worst)


@pytest.mark.parametrize("dim,kv,n,rotate,dt", [(128, 1, 20000, True, "bf16"), (256, 1, 12345, True, "bf16"), (64, 2, 9001, False, "f16"),
                                                 (256, 1, 817, True, "f16"), (128, 2, 2100, True, "bf16")])
def test_one_context(dim, kv, n, rotate, dt):
    rng = np.random.default_rng(dim + n)
    p = H.Paged(rng, [n], kv, dim, 64, rotate)
    p.fill(rng, [n])
    q = H.draw_heads(rng, 1, 4 * kv, dim, dt)
    need = Q.qvla_attention_kv4_workspace_bytes(4 * kv, kv, dim, 1, 1, 1, n)
    check(p, q, [1], [n], True, sizes=(None, 0, need // 3 // 256 * 256, 2 * need))


@pytest.mark.parametrize("seed", range(8))
def test_ragged_contexts_are_split_and_joined_at_the_same_places(seed):
    """The kernels that attend and that join work out the split apart from one another, from the lengths: a part that one of them
    places elsewhere would be lost."""
    rng = np.random.default_rng(seed)
    dim, heads, kv = [(64, 8, 2), (128, 8, 8), (256, 8, 1), (128, 12, 4)][seed % 4]
    batch = [3, 17, 32, 33, 70, 1, 29, 40][seed]
    lens = [int(n) for n in np.exp(rng.uniform(0, np.log(9000), batch))]
    n = 1 if seed < 6 else 3
    lens = [max(m, n) for m in lens]
    p = H.Paged(rng, lens, kv, dim, 16, seed % 2 == 0)
    p.fill(rng, lens)
    q = H.draw_heads(rng, n * batch, heads, dim, "f16" if seed % 3 else "bf16")
    need = Q.qvla_attention_kv4_workspace_bytes(heads, kv, dim, batch, n * batch, n, max(lens))
    check(p, q, [n] * batch, lens, True, sizes=(None, 0, need // 2 // 256 * 256))


def test_rotated_float16_queries_keep_their_bits():
    p, q = sharp_queries(np.random.default_rng(7))
    check(p, q, [8], [600], False)
