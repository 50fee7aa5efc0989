"""Products of 4-bit floating point on the GPU against the float64 product of the same codes.

The bound: codes times block scales multiply exactly, so what is off is the float32 sum and the last rounding.  A sum over K in
steps of 64 products, each step's addition off by at most 2^-22 (two float32 roundings that may cut off) of the sum of
magnitudes S = sum |x w| it runs over, and 64 products within a step likewise: (K / 64 + 8) 2^-22 S.  The scale product and
the fma add 2^-22 of the result's size, the last rounding half a step of the output's type."""

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half a step


class Matrix:
    """Random codes, block scales and row scales of `rows` rows."""

    def __init__(self, seed, rows, k, fmt, size=1.0):
        rng = np.random.default_rng([seed, rows, k])
        self.codes = rng.integers(0, 16, (rows, k)).astype(np.uint8)
        n = k // F.BLOCK[fmt]
        e = 127 + round(np.log2(size / 3))
        self.scale = (rng.integers(e - 3, e + 4, (rows, n)) if fmt == F.MX else rng.integers(0x50, 0x7F, (rows, n))).astype(np.uint8)
        self.row = ((rng.random(rows) + 0.5) * size / 500).astype(np.float32) if fmt == F.NV else None
        self.fmt = fmt

    def exact(self):
        v = F.values(self.codes, self.scale, self.fmt)
        return v if self.row is None else v * self.row.astype(np.float64)[:, None]

    def host(self):
        return F.pack(self.codes), F.to_tiles(self.scale), self.row

    def device(self, fill=0xFF):  # bytes of no row hold NaN: nothing may come of them
        return [None if a is None else torch.from_numpy(a).to(G.DEV) for a in (F.pack(self.codes), F.to_tiles(self.scale, fill), self.row)]


def layer_of(w, dtype, bias=None, gated=False, had=1):
    rows, k = w.codes.shape
    create = Q.qvla_fp4_layer_create_gated if gated else Q.qvla_fp4_layer_create
    return create(rows // 2 if gated else rows, k, had, w.fmt, Q.DTYPE_CODES[dtype], Q.DTYPE_CODES[dtype], *w.host(), bias)


def multiply(layer, x, m, dtype, stream=None):
    """y [m, n]; a guard row behind it has to stay."""
    y = torch.full((m + 1, layer.N), 7.0, dtype=DT[dtype], device=G.DEV)
    xq, xs, row = x.device()
    Q.qvla_gemm_fp4(layer, xq, xs, row, m, y, stream or G.stream())
    Q.qvla_check_device(stream or G.stream())
    assert (y[m] == 7.0).all()
    return y[:m]


def assert_product(y, x, w, bias, dtype, gated=False):
    k = x.codes.shape[1]
    a, b = x.exact(), w.exact()
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    if bias is not None:
        want, size = want + bias.astype(np.float64), size + np.abs(bias)
    off = (k / 64 + 8) * 2.0 ** -22 * size + 2.0 ** -22 * np.abs(want)
    if gated:
        n = want.shape[1] // 2
        gate, up = want[:, :n], want[:, n:]
        # |gelu'| <= 1.13; the kernel's gelu is a float32 expression whose exponential and quotient are good to 2^-20
        off = 1.13 * off[:, :n] * np.abs(up) + (np.abs(F.gelu(gate)) + off[:, :n]) * off[:, n:] + 2.0 ** -19 * np.abs(gate * up)
        want = F.gelu(gate) * up
    off = off + EPS[dtype] * (np.abs(want) + off) + (2.0 ** -25 if dtype == "f16" else 0)
    got = y.double().cpu().numpy()
    assert (np.abs(got - want) <= off).all(), (np.abs(got - want) / off).max()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [
    (1, 16, 128), (1, 2048, 1024), (2, 48, 384), (4, 272, 2176), (7, 128, 640), (16, 512, 256), (17, 144, 4224), (33, 1024, 512), (50, 1008, 1024), (64, 256, 128),
    (100, 4096, 256), (128, 128, 768), (129, 400, 1152), (200, 1024, 1024), (257, 272, 896), (300, 2576, 384), (513, 3008, 1280), (1000, 784, 512), (1, 64, 16384),
    (300, 192, 8192)])
def test_product(fmt, dtype, m, n, k):
    x, w = Matrix(1, m, k, fmt), Matrix(2, n, k, fmt, k ** -0.5)
    bias = np.random.default_rng(n).standard_normal(n).astype(np.float32) if (m + n // 16) % 2 else None
    layer = layer_of(w, dtype, bias)
    assert_product(multiply(layer, x, m, dtype), x, w, bias, dtype)
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,h,k,dtype", [(1, 128, 128, "bf16"), (3, 384, 1024, "f16"), (50, 1024, 512, "bf16"), (130, 256, 2176, "f16"), (300, 640, 256, "bf16"),
                                         (816, 1152, 384, "bf16"), (16, 2048, 2048, "bf16")])
def test_gated_product(fmt, m, h, k, dtype):
    x, w = Matrix(3, m, k, fmt), Matrix(4, 2 * h, k, fmt, k ** -0.5)
    bias = np.random.default_rng(h).standard_normal(2 * h).astype(np.float32) if m % 2 else None
    layer = layer_of(w, dtype, bias, gated=True)
    assert_product(multiply(layer, x, m, dtype), x, w, bias, dtype, gated=True)
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_a_scale_that_is_no_number_stays_in_its_row(fmt, m):
    k, n = 512, 256
    x, w = Matrix(5, m, k, fmt), Matrix(6, n, k, fmt, k ** -0.5)
    layer = layer_of(w, "bf16")
    y = multiply(layer, x, m, "bf16").clone()
    at = m // 2
    x.scale[at, 3] = 0xFF if fmt == F.MX else 0x7F
    z = multiply(layer, x, m, "bf16")
    assert torch.isnan(z[at]).all()
    keep = torch.arange(m, device=G.DEV) != at
    assert torch.equal(z[keep], y[keep])
    layer.close()


@pytest.mark.parametrize("m", [1, 50, 300])
def test_zeros(m):
    x, w = Matrix(5, m, 256, F.NV), Matrix(6, 64, 256, F.NV)
    x.row[:] = 0
    bias = np.arange(64, dtype=np.float32)
    layer = layer_of(w, "bf16", bias)
    assert torch.equal(multiply(layer, x, m, "bf16").float().cpu(), torch.from_numpy(bias).bfloat16().float().expand(m, 64))
    layer.close()


@pytest.mark.parametrize("m,n,k", [(1, 2048, 4096), (50, 1024, 1024), (300, 2560, 2048), (816, 4096, 512)])
def test_the_same_call_gives_the_same_bits(m, n, k):
    x, w = Matrix(7, m, k, F.NV), Matrix(8, n, k, F.NV, k ** -0.5)
    layer = layer_of(w, "bf16")
    first = multiply(layer, x, m, "bf16").clone()
    for _ in range(5):
        assert torch.equal(multiply(layer, x, m, "bf16"), first)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert torch.equal(multiply(layer, x, m, "bf16", side), first)
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,n,k,had,dtype", [(1, 2048, 2048, 2048, "bf16"), (50, 1024, 1024, 64, "f16"), (300, 272, 384, 1, "bf16"), (129, 512, 4096, 4096, "f16")])
def test_linear_is_the_quantiser_and_the_product(fmt, m, n, k, had, dtype):
    w = Matrix(9, n, k, fmt, k ** -0.5)
    layer = layer_of(w, dtype, had=had)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(m)).to(DT[dtype]).to(G.DEV)
    steps = [None] if fmt == F.MX else [None, torch.tensor([0.002], device=G.DEV)]
    for step in steps:
        xq = torch.empty(m, k // 2, dtype=torch.uint8, device=G.DEV)
        xs = torch.empty(Q.qvla_fp4_scale_bytes(fmt, m, k), dtype=torch.uint8, device=G.DEV)
        row = torch.empty(m, device=G.DEV)
        want, got = (torch.empty(m, n, dtype=DT[dtype], device=G.DEV) for _ in range(2))
        Q.qvla_fp4_quantize_rows(x, Q.DTYPE_CODES[dtype], k, m, k, had, fmt, step, xq, xs, row, G.stream())
        Q.qvla_gemm_fp4(layer, xq, xs, row, m, want, G.stream())
        size = Q.qvla_fp4_linear_workspace_bytes(layer, m)
        work = torch.full((size,), 0xFF, dtype=torch.uint8, device=G.DEV)
        Q.qvla_fp4_linear(layer, x, m, step, got, work, size, G.stream())
        Q.qvla_check_device(G.stream())
        assert torch.equal(got, want)
        if step is None:  # and is near the unquantised product: 4-bit codes are 12% of a value off at most, in the mean 5%
            z = F.hadamard32(x.float().cpu().numpy(), had).astype(np.float64) @ w.exact().T
            assert np.linalg.norm(got.double().cpu().numpy() - z) < 0.15 * np.linalg.norm(z)
    layer.close()


def test_workspace_and_device_refusals():
    w = Matrix(10, 64, 256, F.NV)
    layer = layer_of(w, "bf16")
    x, y = torch.zeros(8, 256, dtype=torch.bfloat16, device=G.DEV), torch.zeros(8, 64, dtype=torch.bfloat16, device=G.DEV)
    need = Q.qvla_fp4_linear_workspace_bytes(layer, 8)
    work = torch.zeros(need + 256, dtype=torch.uint8, device=G.DEV)
    for args in ((x, 8, None, y, work, need - 1), (x, 8, None, y, None, need), (x, 8, None, y, work[16:], need), (x, -1, None, y, work, need),
                 (x.view(-1)[4:], 7, None, y, work, need)):
        with pytest.raises(Q.QvlaError) as e:
            Q.qvla_fp4_linear(layer, *args, G.stream())
        assert e.value.status == 1
    Q.qvla_fp4_linear(layer, x, 0, None, y, None, 0, G.stream())
    Q.qvla_gemm_fp4(layer, x, x, None, 0, y, G.stream())
    with pytest.raises(Q.QvlaError):
        Q.qvla_gemm_fp4(layer, x, x, None, 8, y, G.stream())  # NVFP4 without the rows' scales
    with pytest.raises(Q.QvlaError):
        Q.qvla_gemm_fp4(layer, x, x, work, 8, y.view(-1)[4:], G.stream())
    Q.qvla_check_device(G.stream())
    layer.close()


@pytest.mark.parametrize("m", [1, 50, 300])
def test_a_wait_that_runs_out_is_reported(m):
    """The copies are held back (a test hook): the kernel gives up, writes nothing and reports it; afterwards it works again."""
    x, w = Matrix(11, m, 512, F.NV), Matrix(12, 256, 512, F.NV)
    layer = layer_of(w, "bf16")
    want = multiply(layer, x, m, "bf16").clone()
    xq, xs, row = x.device()
    y = torch.full((m, 256), 3.0, dtype=torch.bfloat16, device=G.DEV)
    Q.qvla_debug_set_hooks(2_000_000, True)
    try:
        Q.qvla_gemm_fp4(layer, xq, xs, row, m, y, G.stream())
        with pytest.raises(Q.QvlaError) as e:
            Q.qvla_check_device(G.stream())
        assert e.value.status == 6
    finally:
        Q.qvla_debug_set_hooks(0, False)
    assert (y == 3.0).all()
    assert torch.equal(multiply(layer, x, m, "bf16"), want)
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,n,k,dtype,gated", [(1025, 528, 128, "f16", False), (2100, 1040, 256, "bf16", False), (1800, 4096, 128, "bf16", False), (1111, 512, 128, "f16", True)])
def test_outputs_far_larger_than_the_weights(fmt, m, n, k, dtype, gated):
    """Here the work runs token tile by token tile."""
    x, w = Matrix(21, m, k, fmt), Matrix(22, n, k, fmt, k ** -0.5)
    layer = layer_of(w, dtype, gated=gated)
    assert_product(multiply(layer, x, m, dtype), x, w, None, dtype, gated)
    layer.close()
