"""Attention over packed prompts against the float64 statement: head layouts, lengths from none to hundreds, strides, queries that
see nothing, NaN and infinities where nobody looks, and every refusal's neighbourhood."""

import numpy as np
import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu


def check(q, k, v, lens_q, lens_k, causal, scale=None):
    dt = "f16" if q.dtype == torch.float16 else "bf16"
    got = H.f64(H.prompt(q.to(H.DEV), k.to(H.DEV), v.to(H.DEV), lens_q, lens_k, causal, scale))
    Q.qvla_check_device(H.stream())
    ref, mag, top, terms = H.reference(H.f64(q), H.f64(k), H.f64(v), lens_q, lens_k, causal, scale)
    tol = H.bound(ref, mag, top, terms, q.shape[-1], dt, H.UNIT[dt], 0.0, float(np.abs(H.f64(v)).sum(0).max()) if len(v) else 0.0)
    assert got.shape == ref.shape
    assert not np.isnan(got).any()
    worst = np.max(np.abs(got - ref) - tol) if got.size else 0.0
    assert worst <= 0, worst
    return got


CASES = [
    # heads, kv_heads, dim, dtype, lens_q, lens_k
    (8, 8, 128, "f16", [50], [50]),
    (8, 1, 256, "bf16", [130], [130]),
    (14, 2, 64, "bf16", [1, 37, 129, 0, 64], [1, 37, 200, 5, 64]),
    (8, 2, 128, "bf16", [300, 1, 257], [300, 500, 257]),
    (12, 4, 256, "f16", [33, 65], [33, 190]),
    (5, 5, 64, "f16", [257], [257]),
    (16, 4, 128, "bf16", [127, 128, 129], [127, 128, 129]),
    (1, 1, 64, "bf16", [1], [1]),
    (3, 1, 128, "f16", [86, 43], [86, 600]),
    (32, 8, 64, "bf16", [100], [389]),
    (130, 1, 64, "f16", [3], [70]),  # more query heads on a key/value head than a tile has rows
    (300, 1, 128, "bf16", [2], [9]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:4])))
def test_against_the_float64_statement(case, causal):
    heads, kv, dim, dt, lens_q, lens_k = case
    rng = np.random.default_rng(heads * 1000 + dim + len(lens_q))
    q = H.draw_heads(rng, sum(lens_q), heads, dim, dt)
    k = H.draw_heads(rng, sum(lens_k), kv, dim, dt, outliers=True)
    v = H.draw_heads(rng, sum(lens_k), kv, dim, dt)
    check(q, k, v, lens_q, lens_k, causal)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_prompt_with_growing_scores(dim):
    """Scores that keep growing along the keys move the running maximum at every tile; sharp and flat rows."""
    rng = np.random.default_rng(dim)
    n, heads, kv = 700, 4, 2
    q = H.draw_heads(rng, n, heads, dim, "bf16")
    k = H.draw_heads(rng, n, kv, dim, "bf16")
    ramp = torch.linspace(0.0, 6.0, n)[:, None]
    q[:, 0, 0] = 8.0
    k[:, 0, 0] = (ramp[:, 0] * 4).to(k.dtype)
    q[:, 1] *= 30.0
    v = H.draw_heads(rng, n, kv, dim, "bf16")
    check(q, k, v, [n], [n], True)
    check(q, k, v, [n], [n], False)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", [
    (8, 1, 256, "bf16", [40], [1100]),  # a key range of several CTAs' worth for a tile or two
    (8, 2, 128, "f16", [300], [1500]),
    (6, 6, 64, "bf16", [1], [2048]),
    (4, 2, 64, "f16", [17, 0, 200], [1900, 1500, 90]),  # long, without queries, and shorter than one CTA's share
    (4, 1, 128, "bf16", [1300], [1030]),  # the first 270 queries see nothing where it is causal
    (140, 1, 64, "bf16", [3], [1025]),
], ids=lambda c: "-".join(map(str, c[:4])))
def test_few_queries_on_long_sequences(case, causal):
    heads, kv, dim, dt, lens_q, lens_k = case
    rng = np.random.default_rng(heads * 77 + dim)
    q = H.draw_heads(rng, sum(lens_q), heads, dim, dt)
    k = H.draw_heads(rng, sum(lens_k), kv, dim, dt, outliers=True)
    v = H.draw_heads(rng, sum(lens_k), kv, dim, dt)
    check(q, k, v, lens_q, lens_k, causal)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_a_query_does_not_see_on_a_long_sequence(dim):
    """NaN in keys and values behind the last query of interest, an infinite value that only the last rows see."""
    rng = np.random.default_rng(dim + 1)
    n, m = 30, 1400
    q = H.draw_heads(rng, n, 2, dim, "bf16").to(H.DEV)
    k = H.draw_heads(rng, m + 100, 1, dim, "bf16").to(H.DEV)
    v = H.draw_heads(rng, m + 100, 1, dim, "bf16").to(H.DEV)
    cu_k = H.ints([0, m])
    clean = H.prompt(q, k, v, [n], [m], True, cu_k=cu_k)
    k2, v2 = k.clone(), v.clone()
    k2[m - 5:], v2[m - 5:] = float("nan"), float("nan")
    v2[m - 10, 0, 3] = float("inf")
    got = H.prompt(q, k2, v2, [n], [m], True, cu_k=cu_k)
    Q.qvla_check_device(H.stream())
    assert torch.equal(got[: n - 10], clean[: n - 10])
    assert (got[n - 10: n - 5, :, 3] == float("inf")).all()
    assert torch.equal(got[n - 10: n - 5, :, 4:], clean[n - 10: n - 5, :, 4:])
    assert torch.isnan(got[n - 5:].float()).all()


def test_scores_of_one_size_and_a_large_scale():
    rng = np.random.default_rng(5)
    q = torch.zeros(40, 2, 64, dtype=torch.float16)
    k = H.draw_heads(rng, 40, 1, 64, "f16")
    v = H.draw_heads(rng, 40, 1, 64, "f16")
    check(q, k, v, [40], [40], True)  # every score 0: means of the values
    q = H.draw_heads(rng, 40, 2, 64, "f16")
    check(q, k, v, [40], [40], True, scale=16.0)
    check(q, k, v, [40], [40], True, scale=1e-6)


@pytest.mark.parametrize("dim,heads,kv", [(64, 6, 2), (128, 4, 4), (256, 8, 1)])
def test_more_sequences_than_a_warp_has_lanes(dim, heads, kv):
    rng = np.random.default_rng(dim + 6)
    lens_q = [int(n) for n in rng.integers(0, 40, 75)] + [130, 0, 1]
    lens_k = [int(n + m) for n, m in zip(lens_q, rng.integers(0, 60, 78))]
    q = H.draw_heads(rng, sum(lens_q), heads, dim, "bf16")
    k = H.draw_heads(rng, sum(lens_k), kv, dim, "bf16")
    v = H.draw_heads(rng, sum(lens_k), kv, dim, "bf16")
    check(q, k, v, lens_q, lens_k, True)
    check(q, k, v, lens_q, lens_k, False)


def test_slices_of_a_fused_projection():
    rng = np.random.default_rng(8)
    heads, kv, dim, lens = 8, 2, 128, [70, 200]
    x = H.draw_heads(rng, sum(lens), heads + 2 * kv + 1, dim, "bf16").to(H.DEV)  # a row longer than its heads
    q, k, v = x[:, :heads], x[:, heads: heads + kv], x[:, heads + kv: heads + 2 * kv]
    got = H.prompt(q, k, v, lens, lens, True)
    dense = H.prompt(q.contiguous(), k.contiguous(), v.contiguous(), lens, lens, True)
    assert torch.equal(got, dense)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_an_output_at_any_16_bytes(dim):
    """Aligned to 16 bytes and not to 32, between bytes that stay as they are."""
    rng = np.random.default_rng(dim + 2)
    lens = [150, 3]
    q, k, v = (H.draw_heads(rng, sum(lens), h, dim, "f16").to(H.DEV) for h in (4, 2, 2))
    want = H.prompt(q, k, v, lens, lens, True)
    room = torch.full((want.numel() + 24,), 7.0, dtype=q.dtype, device=H.DEV)
    o = room[8: 8 + want.numel()].view(want.shape)
    cu = H.ints(H.offsets(lens))
    Q.qvla_attention_prompt(q, k, v, Q.F16, 4, 2, dim, q.stride(0), k.stride(0), v.stride(0), 2, cu, sum(lens), cu, sum(lens), dim ** -0.5,
                            True, o, H.stream())
    Q.qvla_check_device(H.stream())
    assert o.data_ptr() % 32 == 16
    assert torch.equal(o, want) and (room[:8] == 7).all() and (room[8 + want.numel():] == 7).all()


def test_queries_that_see_nothing_are_zero():
    rng = np.random.default_rng(9)
    lens_q, lens_k = [5, 200, 7, 3], [2, 60, 0, 3]  # causal: the first 3, 140 and 7 queries see no key
    q = H.draw_heads(rng, sum(lens_q), 4, 64, "bf16")
    k = H.draw_heads(rng, sum(lens_k), 2, 64, "bf16")
    v = H.draw_heads(rng, sum(lens_k), 2, 64, "bf16")
    got = check(q, k, v, lens_q, lens_k, True)
    assert (got[:3] == 0).all() and (got[5:145] == 0).all() and (got[205:212] == 0).all()
    got = check(q, k, v, lens_q, lens_k, False)
    assert (got[205:212] == 0).all()
    q0 = H.draw_heads(rng, 4, 4, 64, "bf16").to(H.DEV)  # no keys at all
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=H.DEV)
    assert (H.prompt(q0, none, none, [4], [0], False) == 0).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_query_does_not_see_has_no_effect(dim, bad):
    """NaN and infinities in later keys and values of a causal sequence, in the next sequence, and behind the last one."""
    rng = np.random.default_rng(11)
    lens = [150, 150]
    q = H.draw_heads(rng, 300, 4, dim, "bf16").to(H.DEV)
    k = H.draw_heads(rng, 340, 2, dim, "bf16").to(H.DEV)
    v = H.draw_heads(rng, 340, 2, dim, "bf16").to(H.DEV)
    clean = H.prompt(q, k[:300], v[:300], lens, lens, True)
    k2, v2 = k.clone(), v.clone()
    k2[300:], v2[300:] = bad, bad
    # tokens 100 to 149 of the first sequence, and all of the second one
    v2[100:150, 0, 3] = bad
    k2[120:150] = bad
    v2[150:300] = bad
    cu = H.ints([0, 150, 300])
    got = H.prompt(q, k2, v2, lens, lens, True, cu_k=cu)
    Q.qvla_check_device(H.stream())
    assert torch.equal(got[:100], clean[:100])
    # the value of token 100 reaches channel 3 of the first key/value head's queries from token 100 on, and nothing else
    assert torch.equal(got[100:120, :, :3], clean[100:120, :, :3]) and torch.equal(got[100:120, 2:], clean[100:120, 2:])
    assert not torch.isfinite(got[100:120, :2, 3].float()).any()
    assert torch.isnan(got[120:150].float()).all() if bad != bad else True
    full = H.prompt(q[:150], k2, v, lens[:1], lens[:1], False, cu_k=H.ints([0, 100]), cu_q=H.ints([0, 150]))
    want = H.prompt(q[:150], k[:100], v[:100], [150], [100], False)
    assert torch.equal(full, want)  # the keys behind the first 100 belong to nobody here


def test_repeated_calls_give_the_same_bits():
    rng = np.random.default_rng(12)
    lens = [333, 1, 700]
    x = [H.draw_heads(rng, sum(lens), h, 128, "f16").to(H.DEV) for h in (8, 2, 2)]
    first = H.prompt(*x, lens, lens, True)
    for _ in range(10):
        assert torch.equal(H.prompt(*x, lens, lens, True), first)


def test_sequences_do_not_depend_on_their_neighbours():
    rng = np.random.default_rng(13)
    lens = [90, 17, 400, 1]
    x = [H.draw_heads(rng, sum(lens), h, 64, "bf16").to(H.DEV) for h in (6, 2, 2)]
    packed = H.prompt(*x, lens, lens, True)
    at = H.offsets(lens)
    for b, n in enumerate(lens):
        alone = H.prompt(*(t[at[b]: at[b + 1]] for t in x), [n], [n], True)
        assert torch.equal(packed[at[b]: at[b + 1]], alone)


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(14)
    lens = [120, 60]
    q, k, v = (H.draw_heads(rng, 180, h, 128, "bf16").to(H.DEV) for h in (8, 2, 2))
    want = H.prompt(q, k, v, lens, lens, True)
    cu = H.ints(H.offsets(lens))
    o = torch.zeros_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = lambda st: Q.qvla_attention_prompt(q, k, v, Q.BF16, 8, 2, 128, q.stride(0), k.stride(0), v.stride(0), 2, cu, 180, cu,  # noqa: E731
                                              180, 128 ** -0.5, True, o, st)
    call(side)
    side.synchronize()
    assert torch.equal(o, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream())
    q.copy_(torch.randn_like(q.float()).to(q.dtype))
    cu.copy_(H.ints([0, 100, 180]))  # other lengths of the same total
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, H.prompt(q, k, v, [100, 80], [100, 80], True))


def test_offsets_that_leave_the_buffers():
    """Offsets beyond the totals are cut off; decreasing ones leave rows out.  Nothing is read or written elsewhere."""
    rng = np.random.default_rng(15)
    q, k, v = (H.draw_heads(rng, 64, h, 64, "bf16").to(H.DEV) for h in (4, 2, 2))
    want = H.prompt(q, k, v, [64], [64], False)
    got = H.prompt(q, k, v, [64], [64], False, cu_q=H.ints([0, 1 << 30]), cu_k=H.ints([-5, 1 << 30]))
    assert torch.equal(got, want)
    got = H.prompt(q, k, v, [0, 64], [0, 64], False, cu_q=H.ints([32, 32, 64]), cu_k=H.ints([0, 0, 64]))
    assert torch.isnan(got[:32].float()).all() and torch.equal(got[32:], want[32:])
    try:
        Q.qvla_check_device(H.stream())
    except Q.QvlaError as e:
        assert e.status == 1
