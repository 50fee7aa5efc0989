"""The 4-bit linear of 1 to 4 tokens, in one launch where that serves: the same bits as the quantiser and the product one after the
other.  Where the launch is one, the workspace stays as it was."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_fp4_gemm import DT, Matrix, layer_of

pytestmark = pytest.mark.gpu


def rows(m, k, dtype, seed=0):
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(31 * m + k + seed))
    x[:, ::97] *= 20
    return x.to(DT[dtype]).to(G.DEV)


def both(layer, x, fmt, had, dtype, step=None):
    """y of the linear, of the two calls, and whether the linear left its workspace alone."""
    m, k = x.shape
    xq = torch.empty(m, k // 2, dtype=torch.uint8, device=G.DEV)
    xs = torch.full((Q.qvla_fp4_scale_bytes(fmt, m, k),), 0xFF, dtype=torch.uint8, device=G.DEV)
    row = torch.empty(m, device=G.DEV)
    want, got = (torch.full((m + 1, layer.N), 7.0, dtype=DT[dtype], device=G.DEV) for _ in range(2))
    code = Q.DTYPE_CODES[dtype]
    Q.qvla_fp4_quantize_rows(x, code, k, m, k, had, fmt, step, xq, xs, row, G.stream())
    Q.qvla_gemm_fp4(layer, xq, xs, row, m, want, G.stream())
    size = Q.qvla_fp4_linear_workspace_bytes(layer, m)
    work = torch.full((size,), 0xA5, dtype=torch.uint8, device=G.DEV)
    Q.qvla_fp4_linear(layer, x, m, step, got, work, size, G.stream())
    Q.qvla_check_device(G.stream())
    assert (got[m] == 7.0).all()
    return got[:m], want[:m], bool((work == 0xA5).all())


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,n,k,had,dtype,one", [
    (1, 128, 128, 1, "bf16", True), (1, 16, 256, 16, "f16", True), (4, 144, 640, 64, "bf16", False), (4, 144, 1024, 64, "bf16", True), (1, 2048, 2048, 2048, "bf16", True),
    (2, 2048, 2048, 2048, "f16", True), (1, 2048, 16384, 2048, "bf16", True), (2, 2048, 16384, 2048, "bf16", True), (1, 1024, 4096, 4096, "f16", True),
    (1, 512, 16384, 4096, "bf16", True), (3, 272, 1152, 128, "f16", True), (4, 1024, 1024, 512, "bf16", True), (2, 1024, 2560, 512, "f16", True),
    (1, 80, 12928, 64, "bf16", True), (1, 640, 3200, 32, "f16", True), (4, 128, 8192, 256, "bf16", True), (3, 256, 8192, 1024, "f16", True),
    (4, 2048, 2048, 2048, "bf16", False), (3, 256, 4096, 4096, "bf16", False), (5, 1024, 1024, 64, "bf16", False)])
def test_the_same_bits(fmt, m, n, k, had, dtype, one):
    layer = layer_of(Matrix(m, n, k, fmt, k ** -0.5), dtype, had=had, bias=torch.randn(n, generator=torch.Generator().manual_seed(n)).numpy())
    x = rows(m, k, dtype)
    for step in [None] if fmt == F.MX else [None, torch.tensor([0.004], device=G.DEV)]:
        got, want, alone = both(layer, x, fmt, had, dtype, step)
        assert torch.isfinite(want.float()).all() and want.float().abs().max() > 0
        assert torch.equal(got, want)
        assert alone == one
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,h,k,had,dtype", [(1, 128, 128, 128, "bf16"), (1, 1024, 2048, 2048, "f16"), (4, 384, 1024, 256, "bf16"), (2, 640, 1152, 64, "f16")])
def test_gated(fmt, m, h, k, had, dtype):
    layer = layer_of(Matrix(m, 2 * h, k, fmt, k ** -0.5), dtype, had=had, gated=True)
    got, want, alone = both(layer, rows(m, k, dtype), fmt, had, dtype)
    assert alone and torch.equal(got, want)
    layer.close()


@pytest.mark.parametrize("m,k,had", [(3, 1024, 64), (2, 2048, 2048)])
def test_values_that_are_not_finite_stay_in_their_token(m, k, had):
    layer = layer_of(Matrix(5, 256, k, F.NV, k ** -0.5), "bf16", had=had)
    for bad in (float("nan"), float("inf")):
        x = rows(m, k, "bf16")
        clean, _, _ = both(layer, x, F.NV, had, "bf16")
        x[1, 700] = bad
        got, want, alone = both(layer, x, F.NV, had, "bf16")
        assert alone and torch.isnan(got[1].float()).all() and torch.isnan(want[1].float()).all()
        assert torch.equal(got[0], clean[0]) and torch.equal(got[2:], clean[2:])
    x = torch.zeros(m, k, dtype=torch.bfloat16, device=G.DEV)
    got, want, _ = both(layer, x, F.NV, had, "bf16")
    assert torch.equal(got, want) and (got == 0).all()
    layer.close()


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
def test_in_place_in_a_graph_and_behind_the_call_that_wrote_its_input(fmt):
    layer = layer_of(Matrix(8, 2048, 2048, fmt, 2048 ** -0.5), "bf16", had=2048)
    size = Q.qvla_fp4_linear_workspace_bytes(layer, 1)
    work = torch.empty(size, dtype=torch.uint8, device=G.DEV)
    start, x = rows(1, 2048, "bf16"), torch.empty(1, 2048, dtype=torch.bfloat16, device=G.DEV)
    want = start
    for _ in range(6):
        want = both(layer, want, fmt, 2048, "bf16")[1]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        x.copy_(start)
        Q.qvla_fp4_linear(layer, x, 1, None, x, work, size, s)
        s.synchronize()
        with torch.cuda.graph(g, stream=s):
            for _ in range(6):
                Q.qvla_fp4_linear(layer, x, 1, None, x, work, size, s)
        for _ in range(3):
            x.copy_(start)
            g.replay()
            s.synchronize()
            assert torch.equal(x, want)
        turn = torch.cuda.CUDAGraph()  # the same through another buffer: one launch a call
        y = torch.empty_like(x)
        work.fill_(0xA5)
        with torch.cuda.graph(turn, stream=s):
            for a, b in ((x, y), (y, x)) * 3:
                Q.qvla_fp4_linear(layer, a, 1, None, b, work, size, s)
        for _ in range(3):
            x.copy_(start)
            turn.replay()
            s.synchronize()
            assert torch.equal(x, want) and bool((work == 0xA5).all())
    layer.close()


@pytest.mark.parametrize("fmt,k,had", [(F.NV, 2048, 2048), (F.MX, 16384, 2048), (F.NV, 128, 1)])
def test_a_wait_that_runs_out_is_reported(fmt, k, had):
    """The copies and the CTAs' exchange are held back (a test hook): nothing is written, the time-out is reported, the next call is right."""
    layer = layer_of(Matrix(9, 256, k, fmt, k ** -0.5), "bf16", had=had)
    x = rows(1, k, "bf16")
    _, want, alone = both(layer, x, fmt, had, "bf16")
    assert alone
    y = torch.full((1, 256), 3.0, dtype=torch.bfloat16, device=G.DEV)
    size = Q.qvla_fp4_linear_workspace_bytes(layer, 1)
    work = torch.empty(size, dtype=torch.uint8, device=G.DEV)
    Q.qvla_debug_set_hooks(2_000_000, True)
    try:
        Q.qvla_fp4_linear(layer, x, 1, None, y, work, size, G.stream())
        with pytest.raises(Q.QvlaError) as e:
            Q.qvla_check_device(G.stream())
        assert e.value.status == 6
    finally:
        Q.qvla_debug_set_hooks(0, False)
    assert (y == 3.0).all()
    assert torch.equal(both(layer, x, fmt, had, "bf16")[0], want)
    layer.close()
