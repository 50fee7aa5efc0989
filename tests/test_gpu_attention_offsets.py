"""Offsets in device memory that begin below 0, decrease or pass their total: cut off, and reported, by every operator."""

import numpy as np
import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu

N = 64
BEYOND, BELOW = [0, 1 << 30], [-5, N]
FALLING = [0, 40, 32, 32]  # the first has 40 tokens, the second none, the third none
WELL = [0, 20, 20, 60]     # a gap at the end is none of the kind


def reported():
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_check_device(H.stream())
    Q.qvla_check_device(H.stream())  # once
    return e.value.status == 1


def long_falling(n=100, at=77):
    """Offsets of more sequences than a warp has lanes; number `at` is larger than the next."""
    cu = list(range(n + 1))
    cu[at] = at + 2
    return cu


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts(dim):
    rng = np.random.default_rng(dim)
    q, k, v = (H.draw_heads(rng, N, h, dim, "bf16").to(H.DEV) for h in (4, 2, 2))
    want = H.prompt(q, k, v, [N], [N], False)
    Q.qvla_check_device(H.stream())
    for cu in (BEYOND, BELOW):
        assert torch.equal(H.prompt(q, k, v, [N], [N], False, cu_q=H.ints(cu)), want) and reported()
        assert torch.equal(H.prompt(q, k, v, [N], [N], False, cu_k=H.ints(cu)), want) and reported()
    got = H.prompt(q, k, v, [0] * 3, [0] * 3, False, cu_q=H.ints(FALLING), cu_k=H.ints([0, N, N, N]))
    assert torch.equal(got[:40], want[:40]) and torch.isnan(got[40:].float()).all() and reported()
    H.prompt(q, k, v, [0] * 3, [0] * 3, False, cu_q=H.ints([0, 20, 40, 60]), cu_k=H.ints(FALLING))
    assert reported()
    H.prompt(q, k, v, [0] * 3, [0] * 3, False, cu_q=H.ints(WELL), cu_k=H.ints(WELL))
    Q.qvla_check_device(H.stream())
    x = [H.draw_heads(rng, 100, h, dim, "bf16").to(H.DEV) for h in (4, 2, 2)]
    H.prompt(*x, [0] * 100, [0] * 100, False, cu_q=H.ints(range(101)), cu_k=H.ints(range(101)))
    Q.qvla_check_device(H.stream())
    H.prompt(*x, [0] * 100, [0] * 100, False, cu_q=H.ints(long_falling()), cu_k=H.ints(range(101)))
    assert reported()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_over_the_cache(dim):
    rng = np.random.default_rng(dim)
    for length in (300, 6000):  # within a cluster, and split with a second kernel
        p = H.Paged(rng, [length], 2, dim, 64, True)
        p.fill(rng, [length])
        q = H.draw_heads(rng, 4, 4, dim, "bf16").to(H.DEV)
        want = H.kv4(p, q, [4], [length], True)
        Q.qvla_check_device(H.stream())
        for cu in ([0, 1 << 30], [-5, 4]):
            for ws in (None, 0):
                got = H.kv4(p, q, [4], [length], True, cu_q=H.ints(cu), ws_bytes=ws)
                assert (got.float() - want.float()).abs().max() < 0.05 and reported()
                assert ws == 0 or torch.equal(got, want)
    lens = [50] * 100
    p = H.Paged(rng, lens, 1, dim, 16, False)
    p.fill(rng, lens)
    q = H.draw_heads(rng, 100, 4, dim, "f16").to(H.DEV)
    want = H.kv4(p, q, [1] * 100, lens, True, max_q=3)
    Q.qvla_check_device(H.stream())
    got = H.kv4(p, q, [1] * 100, lens, True, max_q=3, cu_q=H.ints(long_falling()))
    assert reported()
    assert torch.equal(got[:76], want[:76]) and torch.equal(got[80:], want[80:])


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_in_and_out(dim):
    rng = np.random.default_rng(dim)
    p = H.Paged(rng, [N], 2, dim, 16, True)
    x = H.draw_heads(rng, N, 2, dim, "bf16").to(H.DEV)

    def append(cu, batch=1):
        Q.qvla_kv4_append(p.cache, x, x, Q.BF16, x.stride(0), x.stride(0), batch, H.ints(cu), N, p.table_device, p.width, None, H.stream())
        return p.device.clone()

    def gather(cu, batch=1):
        k, v = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
        Q.qvla_kv4_gather(p.cache, batch, H.ints(cu), N, p.table_device, p.width, None, k, v, Q.BF16, H.stream())
        assert torch.equal(k, v)
        return k

    pool, back = append([0, N]), gather([0, N])
    Q.qvla_check_device(H.stream())
    for cu in (BEYOND, BELOW):
        assert torch.equal(append(cu), pool) and reported()
        assert torch.equal(gather(cu), back) and reported()
    p.table_device = p.table_device.repeat(100, 1)
    got = gather(FALLING, 3)
    assert torch.equal(got[:32], back[:32]) and (got[40:] == 3.0).all() and reported()
    gather(WELL, 3)
    Q.qvla_check_device(H.stream())
    gather(long_falling(60, 41), 60)
    assert reported()
