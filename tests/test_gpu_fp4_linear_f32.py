"""The 4-bit linear of float32 activations (a layer's xdt may be F32, its output is of 16 bits): the bits of the quantiser on those rows and
of the product, one after the other, which have tests of their own against the definition."""

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_fp4_gemm import DT, Matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("ydtype", ["f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m,n,k,had", [(1, 256, 16384, 2048), (3, 272, 1152, 128), (4, 144, 1024, 64), (50, 1024, 512, 1), (300, 512, 2048, 2048), (817, 128, 4096, 4096)])
def test_float32_rows(fmt, ydtype, gated, m, n, k, had):
    n = n // 128 * 128 if gated else n  # units of a gated layer come in 128s
    w = Matrix(m + n, 2 * n if gated else n, k, fmt, k ** -0.5)
    create = Q.qvla_fp4_layer_create_gated if gated else Q.qvla_fp4_layer_create
    bias = np.random.default_rng(n).standard_normal(2 * n if gated else n).astype(np.float32) * 0.1
    layer = create(n, k, had, fmt, Q.F32, Q.DTYPE_CODES[ydtype], *w.host(), bias)
    # numbers that neither 16-bit type holds
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(m)).mul_(1.0 + 2.0 ** -20)
    x[:, ::97] *= 20
    x = x.to(G.DEV)
    steps = [None] if fmt == F.MX else [None, torch.tensor([0.004], device=G.DEV)]
    for step in steps:
        xq = torch.empty(m, k // 2, dtype=torch.uint8, device=G.DEV)
        xs = torch.full((Q.qvla_fp4_scale_bytes(fmt, m, k),), 0xFF, dtype=torch.uint8, device=G.DEV)
        row = torch.empty(m, device=G.DEV)
        want, got = (torch.full((m + 1, n), 7.0, dtype=DT[ydtype], device=G.DEV) for _ in range(2))
        Q.qvla_fp4_quantize_rows(x, Q.F32, k, m, k, had, fmt, step, xq, xs, row, G.stream())
        Q.qvla_gemm_fp4(layer, xq, xs, row, m, want, G.stream())
        size = Q.qvla_fp4_linear_workspace_bytes(layer, m)
        work = torch.empty(size, dtype=torch.uint8, device=G.DEV)
        Q.qvla_fp4_linear(layer, x, m, step, got, work, size, G.stream())
        Q.qvla_check_device(G.stream())
        assert torch.isfinite(want.float()).all() and torch.equal(got, want) and (got[m] == 7.0).all()
    layer.close()


def test_the_output_may_lie_over_the_rows():
    m, k, n = 70, 512, 512
    w = Matrix(9, n, k, F.NV, k ** -0.5)
    layer = Q.qvla_fp4_layer_create(n, k, 256, F.NV, Q.F32, Q.BF16, *w.host())
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(1)).to(G.DEV)
    size = Q.qvla_fp4_linear_workspace_bytes(layer, m)
    work = torch.empty(size, dtype=torch.uint8, device=G.DEV)
    for rows in (1, 4, 70):
        want = torch.empty(rows, n, dtype=torch.bfloat16, device=G.DEV)
        Q.qvla_fp4_linear(layer, x, rows, None, want, work, size, G.stream())
        over = x.clone()
        Q.qvla_fp4_linear(layer, over, rows, None, over, work, size, G.stream())
        Q.qvla_check_device(G.stream())
        assert torch.equal(over.view(torch.bfloat16).reshape(-1)[: rows * n].reshape(rows, n), want)
    layer.close()
