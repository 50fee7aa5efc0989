"""Attention over the 4-bit cache against the float64 statement on the values the cache holds."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu


def check(p, q, lens_q, lens_k, causal, scale=None, **kw):
    dt = "f16" if q.dtype == torch.float16 else "bf16"
    got = H.f64(H.kv4(p, q.to(H.DEV), lens_q, lens_k, causal, scale, **kw))
    Q.qvla_check_device(H.stream())
    ref, mag, top, terms = H.kv4_reference(p, q, lens_q, lens_k, causal, scale)
    # probabilities rounded to 16 bits (bfloat16's at worst), queries to float16; a rotated output is a float32 sum of dim terms more
    tol = H.bound(ref, mag, top, terms, p.dim, dt, H.UNIT["bf16"] + (p.dim * 2.0 ** -23 if p.rotate else 0.0), H.UNIT["f16"], 0.0)
    assert not np.isnan(got).any()
    worst = np.max(np.abs(got - ref) - tol) if got.size else 0.0
    assert worst <= 0, worst
    return got


CASES = [
    # heads, kv_heads, dim, dtype, page, rotate, queries, cached tokens
    (8, 1, 256, "bf16", 64, True, [1], [817]),
    (8, 1, 256, "bf16", 16, True, [50, 50], [866, 66]),
    (32, 8, 128, "f16", 16, False, [1] * 6, [1, 63, 64, 65, 1290, 17]),
    (8, 8, 128, "bf16", 32, True, [1, 3, 0, 2], [300, 3, 9, 100]),
    (14, 2, 64, "f16", 128, True, [1, 1], [129, 4000]),
    (5, 5, 64, "bf16", 256, False, [7], [7]),
    (12, 4, 256, "f16", 64, False, [2, 1], [70, 511]),
    (16, 4, 128, "bf16", 64, True, [33], [2100]),
    (40, 1, 128, "f16", 16, True, [1, 5], [90, 200]),
    (300, 1, 64, "bf16", 16, True, [2], [31]),
    (1, 1, 256, "f16", 16, True, [1], [1]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_against_the_float64_statement(case, causal):
    heads, kv, dim, dt, page, rotate, lens_q, lens_k = case
    rng = np.random.default_rng(heads * 100 + dim)
    p = H.Paged(rng, lens_k, kv, dim, page, rotate)
    p.fill(rng, lens_k)
    q = H.draw_heads(rng, sum(lens_q), heads, dim, dt)
    check(p, q, lens_q, lens_k, causal)
    check(p, q, lens_q, lens_k, causal, ws_bytes=0)                       # no room for a split
    check(p, q, lens_q, lens_k, causal, max_len=p.width * page, max_q=max(lens_q) + 5)  # loose bounds


@pytest.mark.parametrize("dim,kv,lens", [(128, 1, [20000]), (64, 2, [9001, 3]), (256, 1, [12345]), (128, 8, [5000, 100])])
def test_long_caches_are_split_and_joined(dim, kv, lens):
    rng = np.random.default_rng(dim)
    p = H.Paged(rng, lens, kv, dim, 64, True)
    p.fill(rng, lens)
    q = H.draw_heads(rng, len(lens), 4 * kv, dim, "bf16")
    full = check(p, q, [1] * len(lens), lens, True)
    need = Q.qvla_attention_kv4_workspace_bytes(4 * kv, kv, dim, len(lens), len(lens), 1, max(lens))
    for ws in (256, need // 3 // 256 * 256, 2 * need):
        got = check(p, q, [1] * len(lens), lens, True, ws_bytes=ws)
        assert np.abs(got - full).max() < 0.05


@pytest.mark.parametrize("dim,kv,queries", [(64, 2, 1), (128, 8, 1), (256, 1, 3)])
def test_more_sequences_than_a_warp_has_lanes(dim, kv, queries):
    rng = np.random.default_rng(dim + 5)
    lens = [int(n) for n in rng.integers(0, 300, 67)] + [2600, 0, 1, 5000]
    lens_q = [queries if n >= queries else 0 for n in lens]
    p = H.Paged(rng, lens, kv, dim, 32, True)
    p.fill(rng, lens)
    q = H.draw_heads(rng, sum(lens_q), 4 * kv, dim, "bf16")
    check(p, q, lens_q, lens, True)
    check(p, q, lens_q, lens, False)


def test_scores_that_grow_along_the_cache_and_sharp_rows():
    rng = np.random.default_rng(2)
    lens = [3000]
    p = H.Paged(rng, lens, 2, 128, 32, False)
    p.fill(rng, lens)
    kc, vc, ks, vs = A.pool_parts(p.pool, p.page, p.dim)
    pos = np.arange(3000)
    ks[p.table[0, pos // 32], :, pos % 32] *= np.linspace(0.01, 8.0, 3000, dtype=np.float32)[:, None]
    p.device.copy_(torch.from_numpy(p.pool))
    q = H.draw_heads(rng, 1, 8, 128, "bf16")
    q[:, 3:] *= 20.0
    check(p, q, [1], lens, True)
    check(p, q, [1], lens, True, scale=1e-4)


@pytest.mark.parametrize("size", [1e-4, 1.0, 3e3])
def test_queries_and_values_of_any_size(size):
    """Rows of the largest and smallest float16 numbers, and value scales from tiny to huge."""
    rng = np.random.default_rng(21)
    lens = [200, 40]
    p = H.Paged(rng, lens, 1, 64, 16, True)
    p.fill(rng, lens, k_scale=0.3 / size, v_scale=size * size * 1e-3)
    q = (H.draw_heads(rng, 2, 8, 64, "bf16").float() * size).to(torch.bfloat16)
    check(p, q, [1, 1], lens, True)


def test_a_head_of_zeros_and_a_query_of_zeros():
    rng = np.random.default_rng(22)
    p = H.Paged(rng, [50], 1, 128, 16, True)
    p.fill(rng, [50])
    kc, vc, ks, vs = A.pool_parts(p.pool, p.page, p.dim)
    ks[...] = 0.0
    vs[p.table[0, 0], 0, :8] = 0.0
    p.device.copy_(torch.from_numpy(p.pool))
    q = H.draw_heads(rng, 1, 8, 128, "f16")
    q[:, 2] = 0.0
    check(p, q, [1], [50], True)


def test_rows_that_see_nothing_are_zero():
    rng = np.random.default_rng(23)
    lens_q, lens_k = [4, 9, 2], [0, 3, 2]
    p = H.Paged(rng, lens_k, 2, 64, 16, True)
    p.fill(rng, lens_k)
    q = H.draw_heads(rng, sum(lens_q), 4, 64, "f16")
    got = check(p, q, lens_q, lens_k, True)
    assert (got[:4] == 0).all() and (got[4:10] == 0).all() and (got[10:] != 0).any()
    got = check(p, q, lens_q, lens_k, False)
    assert (got[:4] == 0).all()
    assert (H.f64(H.kv4(p, q.to(H.DEV), lens_q, [0, 0, 0], False, max_len=0)) == 0).all()


def test_nan_scales_reach_only_those_who_see_them():
    rng = np.random.default_rng(24)
    lens = [100]
    p = H.Paged(rng, lens, 2, 128, 16, False)
    p.fill(rng, lens)
    q = H.draw_heads(rng, 4, 4, 128, "bf16").to(H.DEV)
    clean = H.kv4(p, q, [4], lens, True)
    kc, vc, ks, vs = A.pool_parts(p.pool, p.page, p.dim)
    vs[p.table[0, 98 // 16], 0, 98 % 16] = np.nan  # seen by the last two queries of the first key/value head
    ks[p.table[0, 99 // 16], 1, 99 % 16] = np.nan  # by the last query of the second one
    p.device.copy_(torch.from_numpy(p.pool))
    got = H.kv4(p, q, [4], lens, True)
    assert torch.equal(got[:2], clean[:2]) and torch.equal(got[2, 2:], clean[2, 2:])
    assert torch.isnan(got[2:, :2].float()).all() and torch.isnan(got[3, 2:].float()).all()


def test_strided_queries_and_repeated_calls():
    rng = np.random.default_rng(25)
    lens = [700, 90]
    p = H.Paged(rng, lens, 2, 128, 32, True)
    p.fill(rng, lens)
    x = H.draw_heads(rng, 4, 8 + 5, 128, "bf16").to(H.DEV)
    q = x[:, 2:10]
    first = H.kv4(p, q.contiguous(), [2, 2], lens, True)
    for _ in range(10):
        assert torch.equal(H.kv4(p, q, [2, 2], lens, True), first)


def test_sequences_that_exceed_the_bounds_are_skipped_and_reported():
    rng = np.random.default_rng(26)
    lens = [90, 30]
    p = H.Paged(rng, lens, 2, 64, 16, True)
    p.fill(rng, lens)
    q = H.draw_heads(rng, 4, 4, 64, "f16").to(H.DEV)
    want = H.kv4(p, q, [2, 2], lens, True)
    Q.qvla_check_device(H.stream())
    for kw in (dict(max_len=50), dict(kv_len=H.ints([-1, 30])), dict(kv_len=H.ints([91 + 16 * p.width, 30]))):
        got = H.kv4(p, q, [2, 2], lens, True, **kw)
        with pytest.raises(Q.QvlaError) as e:
            Q.qvla_check_device(H.stream())
        assert e.value.status == 1
        assert torch.isnan(got[:2].float()).all() and torch.equal(got[2:], want[2:])
    got = H.kv4(p, q, [3, 1], lens, True, max_q=2)
    with pytest.raises(Q.QvlaError):
        Q.qvla_check_device(H.stream())
    assert torch.isnan(got[:3].float()).all() and not torch.isnan(got[3:].float()).any()


def test_a_page_that_is_not_there_is_skipped_and_reported():
    rng = np.random.default_rng(27)
    lens = [64, 64]
    p = H.Paged(rng, lens, 1, 64, 16, False)
    p.fill(rng, lens)
    q = H.draw_heads(rng, 2, 4, 64, "f16").to(H.DEV)
    want = H.kv4(p, q, [1, 1], lens, True)
    p.table[0, 3] = p.pages + 5
    p.table_device.copy_(torch.from_numpy(p.table))
    got = H.kv4(p, q, [1, 1], lens, True)
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_check_device(H.stream())
    assert e.value.status == 1
    assert torch.equal(got[1], want[1])
    short = H.kv4(p, q, [1, 1], [48, 64], False)
    assert torch.allclose(got[0].float(), short[0].float(), atol=1e-2)  # the first 48 tokens are attended


def test_another_stream_and_a_graph_with_growing_lengths():
    rng = np.random.default_rng(28)
    lens = [400, 60]
    p = H.Paged(rng, lens, 2, 128, 16, True)
    p.fill(rng, lens)
    q = H.draw_heads(rng, 2, 8, 128, "bf16").to(H.DEV)
    cu, ln = H.ints([0, 1, 2]), H.ints([100, 7])
    need = Q.qvla_attention_kv4_workspace_bytes(8, 2, 128, 2, 2, 1, 400)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=H.DEV)
    o = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=H.DEV)
    call = lambda st: Q.qvla_attention_kv4(p.cache, q, Q.BF16, 8, q.stride(0), 2, cu, 2, 1, p.table_device, p.width, ln, 400,  # noqa: E731
                                           128 ** -0.5, True, o, ws, ws.numel(), st)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(side)
    side.synchronize()
    assert torch.equal(o, H.kv4(p, q, [1, 1], [100, 7], True, max_len=400))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream())
    for now in ([101, 8], [400, 60], [1, 0]):
        ln.copy_(H.ints(now))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, H.kv4(p, q, [1, 1], now, True, max_len=400))


def test_append_then_attend_matches_attention_over_the_gathered_values():
    """The three operators together: a prompt's keys and values enter the cache, the last token attends to them there, and to
    their read-back values through the prompt operator."""
    rng = np.random.default_rng(29)
    n, heads, kv, dim = 333, 8, 2, 128
    p = H.Paged(rng, [n], kv, dim, 64, True)
    q = H.draw_heads(rng, n, heads, dim, "f16").to(H.DEV)
    k, v = (H.draw_heads(rng, n, kv, dim, "f16", outliers=True).to(H.DEV) for _ in range(2))
    cu = H.ints([0, n])
    Q.qvla_kv4_append(p.cache, k, v, Q.F16, k.stride(0), v.stride(0), 1, cu, n, p.table_device, p.width, None, H.stream())
    gk, gv = torch.empty_like(k), torch.empty_like(v)
    Q.qvla_kv4_gather(p.cache, 1, cu, n, p.table_device, p.width, None, gk, gv, Q.F16, H.stream())
    p.pool = p.device.cpu().numpy()
    got = check(p, q[-1:].cpu(), [1], [n], True)
    over = H.f64(H.prompt(q, gk, gv, [n], [n], True))[-1:]
    assert np.abs(got - over).max() < 2e-2
