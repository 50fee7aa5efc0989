"""Bounds on a launch's rows: max_q is any upper bound, but no sequence has more queries than total_q, and row numbers are 32-bit."""

import pytest

from paper_2605_28803_gb300 import qvla as Q
from tests.test_attention_host import cache, kv4_args


@pytest.mark.parametrize("heads,kv,dim", [(256, 1, 64), (8, 8, 128), (14, 2, 256)])
@pytest.mark.parametrize("total_q", [1, 4, 300])
def test_a_loose_max_q_makes_the_same_plan(heads, kv, dim, total_q):
    """With 256 heads on one and max_q = 2^24 there were 2^28 tiles of 16 rows, whose first rows pass 32 bits."""
    want = Q.qvla_attention_kv4_workspace_bytes(heads, kv, dim, 1, total_q, total_q, 5000)
    assert want > 0 or total_q == 300  # (rows enough to fill the SMs without a split)
    for max_q in (total_q + 1, 1000, 1 << 20, 1 << 24):
        assert Q.qvla_attention_kv4_workspace_bytes(heads, kv, dim, 1, total_q, max_q, 5000) == want


def test_rows_past_32_bits_are_refused():
    c = cache(kv_heads=1)
    for max_q in (1, 1 << 24):
        assert Q._lib.qvla_attention_kv4(*kv4_args(c, heads=256, qs=256 * 64, total_q=1 << 23, max_q=max_q)) == 2
        assert b"rows" in Q._lib.qvla_last_error()
    assert Q._lib.qvla_attention_kv4(*kv4_args(c, heads=1024, qs=1024 * 64, total_q=1 << 24, max_q=1 << 24)) == 2
    assert Q.qvla_attention_kv4_workspace_bytes(1024, 1, 64, 1, 1 << 24, 1 << 24, 5000) == 0
