"""Tokens into the 4-bit cache and out again: codes and scales to the bit, places, and what is left alone."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu


def append(p, k, v, lens, start):
    dt = Q.F16 if k.dtype == torch.float16 else Q.BF16
    Q.qvla_kv4_append(p.cache, k, v, dt, k.stride(0), v.stride(0), len(lens), H.ints(H.offsets(lens)), k.shape[0], p.table_device,
                      p.width, None if start is None else H.ints(start), H.stream())


def gather(p, lens, start, dt):
    n = sum(lens)
    k, v = (torch.full((n, p.kv, p.dim), float("nan"), dtype=H.TORCH[dt], device=H.DEV) for _ in range(2))
    Q.qvla_kv4_gather(p.cache, len(lens), H.ints(H.offsets(lens)), n, p.table_device, p.width,
                      None if start is None else H.ints(start), k, v, Q.DTYPE_CODES[dt], H.stream())
    return k, v


def stored(p, k, v, lens, start):
    """The pool after an append, by the oracle."""
    pool = p.pool.copy()
    kc, vc, ks, vs = A.pool_parts(pool, p.page, p.dim)
    at = H.offsets(lens)
    for b, n in enumerate(lens):
        pos = np.arange(n) + start[b]
        page, slot = p.table[b, pos // p.page], pos % p.page
        for x, codes, scales in ((k, kc, ks), (v, vc, vs)):
            c, d = A.quantize_heads(x[at[b]: at[b + 1]].float().cpu().numpy(), p.rotate)
            codes[page, :, slot], scales[page, :, slot] = A.pack_nibbles(c), d
    return pool


CASES = [
    # kv_heads, dim, dtype, page, rotate, new tokens, tokens before
    (1, 256, "bf16", 64, True, [1, 1, 1], [7, 63, 64]),
    (8, 128, "f16", 16, True, [100, 0, 33, 1], [0, 5, 31, 200]),
    (2, 64, "bf16", 32, False, [65], [0]),
    (3, 64, "f16", 256, True, [5, 300], [250, 0]),
    (5, 128, "bf16", 128, False, [1, 129], [127, 1]),
    (7, 256, "f16", 16, True, [17] * 40, list(range(40))),
    (1, 64, "bf16", 16, True, [1], [0]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_append_and_gather_to_the_bit(case):
    kv, dim, dt, page, rotate, lens, start = case
    rng = np.random.default_rng(kv * 100 + dim)
    total = [n + s for n, s in zip(lens, start)]
    p = H.Paged(rng, total, kv, dim, page, rotate)
    x = H.draw_heads(rng, sum(lens), 2 * kv + 1, dim, dt, outliers=True).to(H.DEV)
    k, v = x[:, :kv], x[:, kv + 1:]
    append(p, k, v, lens, start)
    Q.qvla_check_device(H.stream())
    want = stored(p, k, v, lens, start)
    got = p.device.cpu().numpy()
    assert np.array_equal(got, want)  # also: no other byte of the pool has changed
    p.pool = want
    gk, gv = gather(p, lens, start, dt)
    Q.qvla_check_device(H.stream())
    for name, g, ref in zip("kv", (gk, gv), p.read_back(lens, start)):
        assert torch.equal(g.cpu(), torch.from_numpy(ref).to(H.TORCH[dt])), name
    # and they are within half a step of what was stored, plus the rounding of the output and the rotations
    for g, x in ((gk, k), (gv, v)):
        y = A.rotate_f32(H.f64(x)) if rotate else H.f64(x)
        err = (H.f64(g) - H.f64(x)) @ A.hadamard(dim) if rotate else H.f64(g) - H.f64(x)
        step = np.abs(y).max(-1, keepdims=True) / 7
        slack = H.UNIT[dt] * np.abs(H.f64(g)).max(-1, keepdims=True) * np.sqrt(dim) + 1e-5
        assert (np.abs(err) <= 0.5 * step + slack).all()


@pytest.mark.parametrize("kv,dim,tokens", [(7, 64, 9000), (7, 64, 17100), (9, 256, 3400), (3, 128, 30000), (8, 256, 14700), (40, 64, 6100)])
def test_long_calls_equal_short_ones_to_the_bit(kv, dim, tokens):
    """Warps that take several heads in a row, against calls of a few hundred tokens."""
    rng = np.random.default_rng(tokens + dim)
    lens = [tokens // 2, 0, 1, tokens // 3]
    lens.append(tokens - sum(lens))
    start = [3, 5, 0, 200, 63]
    p = H.Paged(rng, [n + s for n, s in zip(lens, start)], kv, dim, 32, True)
    before = p.device.clone()
    x = H.draw_heads(rng, tokens, 2 * kv, dim, "bf16").to(H.DEV)
    k, v = x[:, :kv], x[:, kv:]
    append(p, k, v, lens, start)
    gk, gv = gather(p, lens, start, "bf16")
    after = p.device.clone()
    p.device.copy_(before)
    at, table = H.offsets(lens), p.table_device
    for b, n in enumerate(lens):
        p.table_device = table[b: b + 1]
        for i in range(0, n, 600):
            m = min(600, n - i)
            part = slice(at[b] + i, at[b] + i + m)
            append(p, k[part], v[part], [m], [start[b] + i])
            pk, pv = gather(p, [m], [start[b] + i], "bf16")
            assert torch.equal(pk, gk[part]) and torch.equal(pv, gv[part])
    Q.qvla_check_device(H.stream())
    assert torch.equal(p.device, after)


def test_ties_zeros_and_small_numbers():
    """Exact half-integer quotients round to even; a head of zeros has scale 0; subnormal heads keep their codes."""
    rng = np.random.default_rng(3)
    p = H.Paged(rng, [6], 1, 64, 16, False)
    x = torch.zeros(6, 2, 64, dtype=torch.float32)
    x[0, :, 0] = 7.0
    x[0, :, 1:15] = torch.arange(14) * 0.5  # scale 1: quotients 0, 0.5, 1, ...
    x[1, :, 0] = 3.5
    x[1, :, 1:15] = -torch.arange(14) * 0.25
    x[3] = 2.0 ** -24 * torch.randint(-7, 8, (2, 64), generator=torch.Generator().manual_seed(1))
    x[4] = 65504.0
    x[5] = torch.randn(2, 64, generator=torch.Generator().manual_seed(2)) * 1e-4
    x = x.to(torch.float16).to(H.DEV)
    append(p, x[:, :1], x[:, 1:], [6], [0])
    assert np.array_equal(p.device.cpu().numpy(), stored(p, x[:, :1], x[:, 1:], [6], [0]))
    b = H.Paged(rng, [4], 1, 128, 16, True)
    y = (torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(4)) *
         torch.tensor([1e-36, 1e-30, 1e30, 1e-20])[:, None, None]).to(torch.bfloat16).to(H.DEV)
    append(b, y[:, :1], y[:, 1:], [4], [0])
    assert np.array_equal(b.device.cpu().numpy(), stored(b, y[:, :1], y[:, 1:], [4], [0]))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rotate", [True, False])
def test_heads_with_nan_or_infinity_read_back_as_nan(bad, rotate):
    rng = np.random.default_rng(4)
    p = H.Paged(rng, [3], 2, 128, 16, rotate)
    k = H.draw_heads(rng, 3, 2, 128, "bf16").to(H.DEV)
    v = H.draw_heads(rng, 3, 2, 128, "bf16").to(H.DEV)
    k[1, 0, 77] = bad
    v[2, 1, 0] = bad
    append(p, k, v, [3], None)
    gk, gv = gather(p, [3], None, "bf16")
    nk, nv = torch.isnan(gk.float()).all(-1), torch.isnan(gv.float()).all(-1)
    assert nk.nonzero().tolist() == [[1, 0]] and nv.nonzero().tolist() == [[2, 1]]
    assert torch.isnan(gk.float()).any(-1).sum() == 1 and torch.isnan(gv.float()).any(-1).sum() == 1


def test_places_that_do_not_exist_are_skipped_and_reported():
    rng = np.random.default_rng(5)
    p = H.Paged(rng, [40, 20], 2, 64, 16, True)
    p.table[0, 1] = p.pages        # a page behind the pool
    p.table[1, 0] = -3
    p.table_device.copy_(torch.from_numpy(p.table))
    x = H.draw_heads(rng, 60, 2, 64, "f16").to(H.DEV)
    before = p.device.clone()
    append(p, x, x, [40, 20], [0, 0])
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_check_device(H.stream())
    assert e.value.status == 1
    Q.qvla_check_device(H.stream())  # reported once
    # the tokens with a place are there: pages 0 and 2 of the first sequence, page 1 of the second
    k, _ = gather(p, [40, 20], [0, 0], "f16")
    with pytest.raises(Q.QvlaError):
        Q.qvla_check_device(H.stream())
    assert (k[16:32] == 0).all() and (k[40:56] == 0).all()
    assert (k[:16] != 0).any() and (k[32:40] != 0).any() and (k[56:] != 0).any()
    untouched = np.setdiff1d(np.arange(p.pages), [p.table[0, 0], p.table[0, 2], p.table[1, 1]])
    assert torch.equal(p.device[untouched], before[untouched])
    append(p, x[:1], x[:1], [1], [p.width * 16])  # behind the table's row
    append(p, x[:1], x[:1], [1], [-1])
    with pytest.raises(Q.QvlaError):
        Q.qvla_check_device(H.stream())


def test_a_pool_past_four_gigabytes():
    """Pages whose offsets pass 32 bits."""
    kv, dim, page = 8, 256, 256
    block = page * (dim + 8) * kv
    pages = (1 << 32) // block + 40
    pool = torch.zeros(pages, kv, page * (dim + 8), dtype=torch.uint8, device=H.DEV)
    cache = Q.Kv4Cache(pool, pages, page, kv, dim, True)
    rng = np.random.default_rng(6)
    x = H.draw_heads(rng, 300, kv, dim, "bf16").to(H.DEV)
    table = H.ints([pages - 1, pages - 7])
    cu = H.ints([0, 300])
    Q.qvla_kv4_append(cache, x, x, Q.BF16, x.stride(0), x.stride(0), 1, cu, 300, table, 2, None, H.stream())
    k, v = torch.empty_like(x), torch.empty_like(x)
    Q.qvla_kv4_gather(cache, 1, cu, 300, table, 2, None, k, v, Q.BF16, H.stream())
    Q.qvla_check_device(H.stream())
    assert torch.equal(k, v) and (k.float() - x.float()).abs().max() < 1.0
    used = pool.view(pages, -1).any(1).nonzero().flatten().tolist()
    assert used == [pages - 7, pages - 1]
