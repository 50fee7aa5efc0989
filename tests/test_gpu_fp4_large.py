"""Matrices whose offsets pass 32 bits, and the most rows: the last rows against the same rows in a call of their own."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu


def layer(n, k, fmt):
    g = torch.Generator().manual_seed(n + k)
    wq = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.int32).to(torch.uint8).numpy()
    lo, hi = (118, 124) if fmt == F.MX else (0x60, 0x7F)
    ws = torch.randint(lo, hi, (Q.qvla_fp4_scale_bytes(fmt, n, k),), generator=g, dtype=torch.int32).to(torch.uint8).numpy()
    row = (torch.rand(n, generator=g) * 1e-4).numpy() if fmt == F.NV else None
    return Q.qvla_fp4_layer_create(n, k, 64, fmt, Q.BF16, Q.BF16, wq, ws, row)


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,k,n", [(300_032, 8192, 48), (1 << 20, 128, 2304)])
def test_last_rows(fmt, m, k, n):
    """m k or m n elements are more than 2^31."""
    st, tail = G.stream(), 128
    x = torch.randn(m, k, generator=torch.Generator(device=G.DEV).manual_seed(1), device=G.DEV, dtype=torch.bfloat16)
    out = []
    lay = layer(n, k, fmt)
    norm = Q.BlockNorm(Q.NORM_RMS, Q.BF16, mod_tokens=0)
    for rows in (x, x[m - tail:]):
        t = rows.shape[0]
        xq, row = torch.empty(t, k // 2, dtype=torch.uint8, device=G.DEV), torch.empty(t, device=G.DEV)
        xs = torch.empty(Q.qvla_fp4_scale_bytes(fmt, t, k), dtype=torch.uint8, device=G.DEV)
        h, v, y = (torch.empty(t, c, dtype=torch.bfloat16, device=G.DEV) for c in (k, k, n))
        Q.qvla_block_norm_fp4(norm, rows, Q.BF16, k, None, k, t, k, None, h, 64, fmt, None, xq, xs, row, st)
        Q.qvla_fp4_dequantize_rows(xq, xs, row, fmt, t, k, v, Q.BF16, st)
        Q.qvla_gemm_fp4(lay, xq, xs, row, t, y, st)
        Q.qvla_check_device(st)
        out.append([a[-tail:].clone() for a in (h, v, y)])
        del xq, xs, row, h, v, y
    (h, v, y), (h1, v1, y1) = out
    assert torch.equal(h, h1) and torch.equal(v, v1)
    assert (y.float() - y1.float()).norm() <= 2.0 ** -8 * y1.float().norm()  # (the products' sums may be in another order)
    assert v.float().norm() > 0.5 * (tail * k) ** 0.5 and y.abs().max() > 0
    lay.close()
