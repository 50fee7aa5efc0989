"""The norm's output in the place of its branch, and the residual in place at the same time: the bits of a call with buffers apart, also
where a group of threads goes through many rows."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_block_norm import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant", [None, F.MX, F.NV])
@pytest.mark.parametrize("dtype,rdtype", [("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("m,k", [(1, 128), (5, 1152), (50, 1024), (3000, 2048), (1301, 1152), (320, 16384)])
@pytest.mark.parametrize("kw", [dict(), dict(post=True, cond=7, layer=True)])
def test_h_where_y_was(quant, dtype, rdtype, m, k, kw):
    c = Case(m, k, dtype, rdtype, **kw)
    plan, code, rcode = c.plan(), Q.DTYPE_CODES[dtype], Q.DTYPE_CODES[rdtype]

    def run(r_out, h):
        codes = [torch.full((m, k // 2), 0x33, dtype=torch.uint8, device=G.DEV),
                 torch.full((Q.qvla_fp4_scale_bytes(quant or 0, m, k),), 0x33, dtype=torch.uint8, device=G.DEV), torch.full((m,), 3.0, device=G.DEV)]
        if quant is None:
            Q.qvla_block_norm(plan, c.r, rcode, k, c.y, k, m, k, r_out, h, G.stream())
        else:
            Q.qvla_block_norm_fp4(plan, c.r, rcode, k, c.y, k, m, k, r_out, h, 128, quant, None, *codes, G.stream())
        Q.qvla_check_device(G.stream())
        return codes

    r, h = torch.empty_like(c.r), torch.empty_like(c.y)
    codes = run(r, h)
    before = c.r.clone(), c.y.clone()
    for _ in range(3):
        c.r.copy_(before[0])
        c.y.copy_(before[1])
        again = run(c.r, c.y)
        assert torch.equal(c.r, r) and torch.equal(c.y, h)
        assert all(torch.equal(a, b) for a, b in zip(again, codes))
    assert code == plan.dt
