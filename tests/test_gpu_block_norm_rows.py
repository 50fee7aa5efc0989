"""The norms on so many rows that a group of threads goes through several: the next row's operands asked for ahead, conditioning row by
row, slots of the sums in turn, rows that an index skips, and the rotations whose threads meet at a barrier.  Sizes by 152 SMs: norm_kernel has
608 CTAs of 256 threads at 2048 channels, 6 to 11 turns at 6500 rows; a CTA that quantises has two to four rows a group from 1300 on.
The references and bounds are those of test_gpu_block_norm.py."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_block_norm import DT, Case

pytestmark = pytest.mark.gpu
TYPES = [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")]
PLAIN, EVERYTHING = dict(), dict(post=True, cond=7, layer=True)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("m,k", [(6500, 2048), (6501, 1152), (2600, 4104), (20011, 256)])
@pytest.mark.parametrize("kw", [PLAIN, dict(post=True, pad=8), dict(cond=6500, layer=True), dict(cond=9, index=True, post=True, layer=True, alpha=0.5, pad=16)])
def test_many_rows(dtype, rdtype, m, k, kw):
    c = Case(m, k, dtype, rdtype, **kw)
    r, h = c.run()
    c.check_residual(r)
    c.check_h(h, r)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("m,k", [(6500, 2048), (6501, 1152), (700, 16384)])
@pytest.mark.parametrize("kw", [PLAIN, EVERYTHING])
def test_in_place(dtype, rdtype, m, k, kw):
    c = Case(m, k, dtype, rdtype, **kw)
    r, h = c.run()
    before = c.r.clone()
    for _ in range(3):
        c.r = before.clone()
        _, h2 = c.run(r_out=c.r)
        assert torch.equal(c.r, r) and torch.equal(h2, h)


class Junction:
    """One call with the quantiser, its outputs filled before it."""

    def __init__(self, c, had, fmt, step=None, h=True):
        m, k = c.m, c.k
        self.r = torch.full((m, k), 9.0, dtype=DT[c.rdtype], device=G.DEV)
        self.h = torch.full((m, k), 9.0, dtype=DT[c.dtype], device=G.DEV) if h else None
        self.codes = (torch.full((m, k // 2), 0x33, dtype=torch.uint8, device=G.DEV), torch.full((Q.qvla_fp4_scale_bytes(fmt, m, k),), 0x33, dtype=torch.uint8, device=G.DEV),
                      torch.full((m,), 3.0, device=G.DEV))
        Q.qvla_block_norm_fp4(c.plan(), c.r, Q.DTYPE_CODES[c.rdtype], c.r.stride(0), c.y, c.y.stride(0), m, k, self.r, self.h, had, fmt, step, *self.codes, G.stream())


def quantised(h, c, had, fmt, step=None):
    want = torch.full((c.m, c.k // 2), 0x33, dtype=torch.uint8, device=G.DEV), torch.full((Q.qvla_fp4_scale_bytes(fmt, c.m, c.k),), 0x33, dtype=torch.uint8, device=G.DEV), torch.full((c.m,), 3.0, device=G.DEV)
    Q.qvla_fp4_quantize_rows(h, Q.DTYPE_CODES[c.dtype], c.k, c.m, c.k, had, fmt, step, *want, G.stream())
    return want


SHAPES = [(1300, 2048, 2048), (1301, 4096, 4096), (1300, 16384, 2048), (640, 16384, 4096), (1303, 4096, 1024), (1301, 1536, 512), (1302, 1152, 128), (1400, 512, 256), (1300, 8192, 4096)]


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("m,k,had", SHAPES)
@pytest.mark.parametrize("kw", [PLAIN, EVERYTHING])
def test_several_rows_a_group_quantised(dtype, rdtype, m, k, had, kw):
    c = Case(m, k, dtype, rdtype, **kw)
    first = Junction(c, had, F.NV)
    Q.qvla_check_device(G.stream())
    c.check_residual(first.r)
    c.check_h(first.h, first.r)
    for fmt, step, h in ((F.NV, None, True), (F.NV, None, False), (F.NV, torch.tensor([0.004], device=G.DEV), False), (F.MX, None, True), (F.MX, None, False)):
        j = Junction(c, had, fmt, step, h)
        assert torch.equal(j.r, first.r) and (not h or torch.equal(j.h, first.h))
        assert all(torch.equal(a, b) for a, b in zip(j.codes, quantised(first.h, c, had, fmt, step)))
    Q.qvla_check_device(G.stream())


def some_skipped(c):
    """The index with rows out of range here and there, alone, in twos and in a run, and which they are."""
    good, rows = c.index.clone(), c.gate.shape[0]
    at = torch.tensor([0, 3, 4, 17, 400, 401, 402, 403, 700, c.m - 2] + list(range(1100, 1109)), device=G.DEV)
    c.index = good.clone()
    c.index[at[::2]], c.index[at[1::2]] = rows, -1
    skipped = torch.zeros(c.m, dtype=torch.bool, device=G.DEV)
    skipped[at] = True
    return good, skipped


def check_skips_reported():
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_check_device(G.stream())
    assert e.value.status == 1
    Q.qvla_check_device(G.stream())


@pytest.mark.parametrize("dtype,rdtype", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,k", [(6500, 2048), (6501, 1152)])
def test_skipped_rows_among_many(dtype, rdtype, m, k):
    c = Case(m, k, dtype, rdtype, layer=True, post=True, cond=9, index=True)
    want_r, want_h = c.run()
    _, skipped = some_skipped(c)
    r, h = torch.full_like(want_r, 9.0), torch.full_like(want_h, 9.0)
    Q.qvla_block_norm(c.plan(), c.r, Q.DTYPE_CODES[rdtype], k, c.y, k, m, k, r, h, G.stream())
    check_skips_reported()
    assert (r[skipped] == 9.0).all() and (h[skipped] == 9.0).all()
    assert torch.equal(r[~skipped], want_r[~skipped]) and torch.equal(h[~skipped], want_h[~skipped])


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype,rdtype", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,k,had", SHAPES[:3] + SHAPES[5:7])
def test_skipped_rows_quantised(fmt, dtype, rdtype, m, k, had):
    c = Case(m, k, dtype, rdtype, layer=True, cond=9, index=True)
    want = Junction(c, had, fmt)
    Q.qvla_check_device(G.stream())
    _, skipped = some_skipped(c)
    got = Junction(c, had, fmt)
    check_skips_reported()
    assert (got.r[skipped] == 9.0).all() and (got.h[skipped] == 9.0).all()
    assert torch.equal(got.r[~skipped], want.r[~skipped]) and torch.equal(got.h[~skipped], want.h[~skipped])
    (q, s, row), (wq, ws, wrow), blocks = got.codes, want.codes, k // (32 if fmt == F.MX else 16)
    tiles, wtiles = (torch.from_numpy(F.from_tiles(t.cpu().numpy(), m, blocks)).to(G.DEV) for t in (s, ws))
    assert (q[skipped] == 0x33).all() and (tiles[skipped] == 0x33).all() and (row[skipped] == 3.0).all()
    assert torch.equal(q[~skipped], wq[~skipped]) and torch.equal(tiles[~skipped], wtiles[~skipped]) and torch.equal(row[~skipped], wrow[~skipped])
