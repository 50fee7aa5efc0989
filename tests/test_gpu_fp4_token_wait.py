"""The one-launch linear behind a kernel that lets it start early and then runs longer than the limit of a wait.  What the linear's
warps do before the previous kernel has ended may not count against that limit: each CTA here has more k-blocks of weights than
places for them, so the warp that loads them has to wait for tokens."""

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_fp4_few_tokens import rows
from tests.test_gpu_fp4_gemm import Matrix, layer_of

pytestmark = pytest.mark.gpu
LIMIT_NS = 500_000  # every wait of either kernel takes some us
KEYS, BATCH, DIM = 1 << 20, 4096, 64  # one CTA goes through all keys; the sequences without any keep the call from sharing them out


def long_attention():
    """A call that takes about 10 ms on one SM and lets the next kernel start as soon as it has found its work."""
    g = torch.Generator(device=G.DEV).manual_seed(3)
    q = torch.randn(16, DIM, generator=g, device=G.DEV).bfloat16()
    k = torch.randn(KEYS, DIM, generator=g, device=G.DEV).bfloat16()
    cu_q = torch.full((BATCH + 1,), 16, dtype=torch.int32, device=G.DEV)
    cu_k = torch.full((BATCH + 1,), KEYS, dtype=torch.int32, device=G.DEV)
    cu_q[0] = cu_k[0] = 0
    o = torch.empty_like(q)

    def call():
        Q.qvla_attention_prompt(q, k, k, Q.BF16, 1, 1, DIM, DIM, DIM, DIM, BATCH, cu_q, 16, cu_k, KEYS, DIM ** -0.5, False, o, G.stream())
    return call


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
def test_a_long_kernel_ahead(fmt):
    n, k = 2048, 16384
    layer = layer_of(Matrix(5, n, k, fmt, k ** -0.5), "bf16", had=2048)
    x = rows(1, k, "bf16")
    size = Q.qvla_fp4_linear_workspace_bytes(layer, 1)
    work = torch.full((size,), 0xA5, dtype=torch.uint8, device=G.DEV)

    def output():
        y = torch.full((1, n), float("nan"), dtype=torch.bfloat16, device=G.DEV)
        torch.cuda.synchronize()  # (the fill is over: nothing but the attention lies ahead)
        return y

    ahead = long_attention()
    want = output()
    Q.qvla_fp4_linear(layer, x, 1, None, want, work, size, G.stream())
    ahead()
    Q.qvla_check_device(G.stream())
    assert (work == 0xA5).all()  # one launch
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    ahead()
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) * 1e6 > 4 * LIMIT_NS  # (else this shows nothing)
    Q.qvla_debug_set_hooks(LIMIT_NS, False)
    try:
        for _ in range(3):
            y = output()
            ahead()
            Q.qvla_fp4_linear(layer, x, 1, None, y, work, size, G.stream())
            Q.qvla_check_device(G.stream())  # no time-out
            assert torch.equal(y, want)
    finally:
        Q.qvla_debug_set_hooks(0, False)
    layer.close()
