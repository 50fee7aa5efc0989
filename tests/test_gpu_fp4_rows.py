"""Rows to 4-bit floating point and back on the GPU, against the oracle to the bit."""

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
FILL = 0xA5


def run(x, fmt, had=1, step=None, stride=None, stream=None):
    """(codes [m, k], scale bytes [m, blocks], Delta [m], the whole scale buffer) of rows x, a CPU tensor."""
    m, k = x.shape
    stride = stride or k
    xg = torch.full((max(m, 1), stride), float("nan"), dtype=x.dtype, device=G.DEV)
    xg[:m, :k] = x.to(G.DEV)
    xq = torch.full((m + 1, k // 2), FILL, dtype=torch.uint8, device=G.DEV)
    xs = torch.full((Q.qvla_fp4_scale_bytes(fmt, m, k) + 512,), FILL, dtype=torch.uint8, device=G.DEV)
    row = torch.full((m + 1,), 77.0, device=G.DEV)
    ss = None if step is None else torch.tensor([step], device=G.DEV)
    code = {torch.float16: Q.F16, torch.bfloat16: Q.BF16, torch.float32: Q.F32}[x.dtype]
    Q.qvla_fp4_quantize_rows(xg, code, stride, m, k, had, fmt, ss, xq, xs, row, stream or G.stream())
    Q.qvla_check_device(stream or G.stream())
    assert (xq[m] == FILL).all() and (xs[-512:] == FILL).all() and row[m] == 77.0  # nothing behind the last row
    if fmt == F.MX:
        assert (row == 77.0).all()
    tiles = xs[:-512].cpu().numpy()
    return F.unpack(xq[:m].cpu().numpy()), F.from_tiles(tiles, m, k // F.BLOCK[fmt]), row[:m].cpu().numpy(), tiles


def check(x, fmt, had=1, step=None, stride=None):
    got = run(x, fmt, had, step, stride)
    codes, scale, delta = F.quantize(F.hadamard32(x.float().numpy(), had), fmt, step)
    assert np.array_equal(got[1], scale)
    if fmt == F.NV:
        assert np.array_equal(got[2], delta)
    zero = (got[0] & 7) == 0
    assert np.array_equal(np.where(zero, 0, got[0]), np.where((codes & 7) == 0, 0, codes))  # a zero may carry a sign
    m = x.shape[0]
    rows = F.from_tiles(got[3], -(-m // 128) * 128, x.shape[1] // F.BLOCK[fmt])[m:]
    assert (rows == FILL).all()  # bytes of no row stay as they were


def rows(seed, m, k, dtype, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g)
    if outliers:
        x[:, torch.randperm(k, generator=g)[: max(1, k // 100)]] *= 20
    return x.to(DT[dtype])


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("m,k,had", [
    (1, 128, 1), (3, 128, 128), (5, 384, 2), (131, 128, 64), (40, 256, 256), (7, 640, 4), (65, 1024, 1), (2, 1152, 128), (17, 1024, 512), (9, 2048, 1024),
    (3, 2048, 2048), (129, 2432, 64), (5, 4096, 4096), (2, 6144, 2048), (1, 8192, 16), (33, 1280, 256), (2, 12288, 4096), (3, 16384, 2048), (1, 16384, 1),
    (300, 512, 32), (4, 896, 8)])
def test_codes_and_scales(fmt, dtype, m, k, had):
    check(rows(m * k + had, m, k, dtype), fmt, had)


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,k,stride", [(5, 256, 264), (33, 1024, 2048), (2, 128, 1000)])
def test_strided_rows(fmt, m, k, stride):
    check(rows(m, m, k, "bf16"), fmt, 128, stride=stride)


@pytest.mark.parametrize("dtype,step", [("bf16", 0.01), ("f16", 1e-3), ("f32", 0.25), ("f32", 1e-30), ("f32", 1e30), ("bf16", 3e-39), ("f32", 3e38)])
def test_a_steps_scale(dtype, step):
    x = rows(11, 9, 512, dtype)
    check(x, F.NV, 1, step=float(np.float32(step)))
    check(x, F.NV, 256, step=float(np.float32(step)))


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
def test_ties_of_values_and_scales(fmt):
    """Rows of few significant bits, many of whose quotients stand exactly on a tie or one rounding of Delta from it."""
    g = torch.Generator().manual_seed(5)
    x = torch.randint(-64, 65, (256, 1024), generator=g).float() / 8
    x[:, 0] = 48.0  # row maxima of 48: Delta = 48 / 2688 = 1/56, which float32 rounds
    x[128:, 0] = 42.0  # Delta 1/64: exact quotients, exact ties
    check(x, fmt)
    check(x.to(torch.bfloat16), fmt)
    check(x[:, :512] * 2.0 ** torch.randint(-20, 20, (256, 1), generator=g), fmt)


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("size", [1e-45, 1e-42, 3e-39, 1e-37, 1e-30, 1e-20, 1e20, 1e30, 3e38])
def test_extreme_sizes(fmt, size):
    x = (rows(2, 4, 256, "f32", outliers=False).clamp(-1, 1).double() * size).float()
    check(x, fmt)


def test_wide_range_within_a_row():
    g = torch.Generator().manual_seed(8)
    x = torch.randn(64, 1024, generator=g) * 10.0 ** torch.randint(-12, 12, (64, 1024 // 16), generator=g).float().repeat_interleave(16, 1)
    for fmt in (F.MX, F.NV):
        check(x, fmt)


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("had", [1, 256])
def test_zero_rows_and_blocks(fmt, had):
    x = rows(4, 6, 512, "bf16")
    x[1] = 0
    x[2, :256] = 0
    x[3, 32:64] = -0.0
    check(x, fmt, had)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite(bad):
    x = rows(4, 5, 512, "bf16")
    x[2, 300] = bad
    # MX: the block is marked, the others keep their values
    codes, scale, _ = F.quantize(np.delete(x.float().numpy(), 2, 0), F.MX)
    got = run(x, F.MX)
    assert got[1][2, 300 // 32] == 255 and (np.delete(got[1][2], 300 // 32) < 255).all()
    assert np.array_equal(np.delete(got[1], 2, 0), scale) and np.array_equal(np.delete(got[0], 2, 0), codes)
    # NV: the row has no scale
    codes, scale, delta = F.quantize(np.delete(x.float().numpy(), 2, 0), F.NV)
    got = run(x, F.NV)
    assert np.isnan(got[2][2]) and np.array_equal(np.delete(got[2], 2), delta) and np.array_equal(np.delete(got[1], 2, 0), scale)
    # with a step's scale an infinity is clamped, and a NaN marks its block
    got = run(x, F.NV, step=0.01)
    s = got[1][2, 300 // 16]
    assert (s == 0x7F) if np.isnan(bad) else (s == 0x7E and got[0][2, 300] == (15 if bad < 0 else 7))
    assert (np.delete(got[1][2], 300 // 16) < 0x7F).all()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("odt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("m,k", [(1, 128), (130, 384), (3, 16384)])
def test_read_back(fmt, odt, m, k):
    rng = np.random.default_rng(m + k)
    codes = rng.integers(0, 16, (m, k)).astype(np.uint8)
    n = k // F.BLOCK[fmt]
    scale = rng.integers(100, 140, (m, n)) if fmt == F.MX else rng.integers(0, 127, (m, n))
    scale = scale.astype(np.uint8)
    row = (rng.random(m) * 0.01 + 0.001).astype(np.float32)
    out = torch.full((m + 1, k), 5.0, dtype=DT[odt], device=G.DEV)
    dev = [torch.from_numpy(a).to(G.DEV) for a in (F.pack(codes), F.to_tiles(scale, 0xFF), row)]
    Q.qvla_fp4_dequantize_rows(*dev, fmt, m, k, out, Q.DTYPE_CODES[odt], G.stream())
    Q.qvla_check_device(G.stream())
    v = F.values(codes, scale, fmt).astype(np.float32)  # exact
    want = torch.from_numpy(v * row[:, None] if fmt == F.NV else v).to(DT[odt])
    assert torch.equal(out[:m].cpu(), want) and (out[m] == 5.0).all()


def test_another_stream_and_a_graph():
    x = rows(1, 50, 1024, "bf16")
    want = run(x, F.NV, 64)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run(x, F.NV, 64, stream=side)
    assert all(np.array_equal(a, b) for a, b in zip(want[:3], got[:3]))
    xg, out = x.to(G.DEV), torch.empty(50, 1024, device=G.DEV)
    xq, xs, row = torch.empty(50, 512, dtype=torch.uint8, device=G.DEV), torch.empty(8192, dtype=torch.uint8, device=G.DEV), torch.empty(50, device=G.DEV)

    def both():
        st = torch.cuda.current_stream()
        Q.qvla_fp4_quantize_rows(xg, Q.BF16, 1024, 50, 1024, 64, F.NV, None, xq, xs, row, st)
        Q.qvla_fp4_dequantize_rows(xq, xs, row, F.NV, 50, 1024, out, Q.F32, st)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    xg.copy_(rows(2, 50, 1024, "bf16"))
    g.replay()
    torch.cuda.synchronize()
    codes, scale, delta = F.quantize(F.hadamard32(xg.float().cpu().numpy(), 64), F.NV)
    assert np.array_equal(out.cpu().numpy(), (F.values(codes, scale, F.NV).astype(np.float32) * delta[:, None]))
