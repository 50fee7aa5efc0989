"""The row-wise bound of attention over the 4-bit cache can fail: a result of zeros, one that lost a chunk of tokens, and one from
queries rounded to fewer bits are all outside it."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from tests import attention_bounds as B
from tests import attention_helpers as H


@pytest.fixture(autouse=True)
def on_the_host(monkeypatch):
    monkeypatch.setattr(H, "DEV", "cpu")


@pytest.mark.parametrize("dim,kv,n,rotate,dt", [(128, 1, 20000, True, "bf16"), (256, 1, 12345, True, "bf16"), (64, 2, 9001, False, "f16"),
                                                 (256, 1, 817, True, "f16"), (128, 2, 2100, True, "bf16")])
def test_zeros_and_a_lost_chunk_are_outside(dim, kv, n, rotate, dt):
    rng = np.random.default_rng(dim + n)
    p = H.Paged(rng, [n], kv, dim, 64, rotate)
    p.fill(rng, [n])
    q = H.draw_heads(rng, 1, 4 * kv, dim, dt)
    want, tol = B.statement(p, q, [1], [n], True, q_unit=2.0 ** -11)
    assert (tol < 0.02 * np.linalg.norm(want, axis=-1)).all()
    for first in (0, n // 128 * 64, (n - 1) // 64 * 64 - 64):  # 64 tokens: no chunk is smaller but a sequence's last
        lost, _ = B.statement(p, q, [1], [n], True, leave=(first, first + 64))
        assert (B.error(lost, want) > tol).all()


def sharp_queries(rng):
    """Scores of some hundreds, whose leading tokens are close in some rows, where a score's last bits count."""
    p = H.Paged(rng, [600], 2, 128, 64, True)
    p.fill(rng, [600])
    return p, (H.draw_heads(rng, 8, 16, 128, "f16").float() * 100).to(torch.float16)


def test_queries_of_eleven_bits_are_outside():
    p, q = sharp_queries(np.random.default_rng(7))
    want, tol = B.statement(p, q, [8], [600], False, q_unit=2.0 ** -21)
    rotated = H.f64(q) @ A.hadamard(128)
    top = 2.0 ** np.ceil(np.log2(np.abs(rotated).max(-1, keepdims=True)))
    coarse = torch.from_numpy((np.float64(np.float16(rotated / top)) * top) @ A.hadamard(128))
    got, _ = B.statement(p, coarse, [8], [600], False)
    assert (B.error(got, want) > tol).sum() >= 3
