"""A junction and the product behind it, between passes of other data that nothing waits for: every pass has the bits of the first."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_block_norm import DT, Case
from tests.test_gpu_fp4_gemm import Matrix, layer_of

pytestmark = pytest.mark.gpu


class Pass:
    def __init__(self, seed, fmt, dtype, m, k, n, had, kw):
        self.c = Case(m, k, dtype, dtype, seed=seed, **kw)
        self.layer = layer_of(Matrix(seed, n, k, fmt, k ** -0.5), dtype)
        self.plan, self.fmt, self.had, self.code = self.c.plan(), fmt, had, Q.DTYPE_CODES[dtype]
        self.r, self.y = torch.empty(m, k, dtype=DT[dtype], device=G.DEV), torch.empty(m, n, dtype=DT[dtype], device=G.DEV)
        self.q, self.s = torch.empty(m, k // 2, dtype=torch.uint8, device=G.DEV), torch.zeros(Q.qvla_fp4_scale_bytes(fmt, m, k), dtype=torch.uint8, device=G.DEV)
        self.row = torch.zeros(m, device=G.DEV)

    def run(self):
        c, k = self.c, self.c.k
        Q.qvla_block_norm_fp4(self.plan, c.r, self.code, k, c.y, k, c.m, k, self.r, None, self.had, self.fmt, None, self.q, self.s, self.row, G.stream())
        Q.qvla_gemm_fp4(self.layer, self.q, self.s, self.row, c.m, self.y, G.stream())
        return self.r, self.q, self.s, self.row, self.y


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype,m,k,n,had,kw", [("bf16", 816, 2048, 2560, 2048, dict()), ("f16", 200, 1024, 4096, 1024, dict(layer=True, cond=50))])
def test_every_pass_has_the_same_bits(fmt, dtype, m, k, n, had, kw):
    one, other = (Pass(seed, fmt, dtype, m, k, n, had, kw) for seed in (1, 2))
    want = [t.clone() for t in one.run()]
    torch.cuda.synchronize()
    for i in range(60):
        for _ in range(i % 3):
            other.run()
        got = one.run()
        if i % 4 == 0:
            torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    Q.qvla_check_device(G.stream())
    fresh = Pass(1, fmt, dtype, m, k, n, had, kw)
    assert all(torch.equal(a, b) for a, b in zip(fresh.run(), want))
