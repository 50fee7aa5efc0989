"""Calls of the 4-bit operators that are under way at once: two threads with a stream each, and chains of calls that overwrite what
the calls before them read.  The same calls one at a time, with a synchronisation after each, say what has to come out, to the bit."""

import threading

import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G
from tests.test_gpu_fp4_gemm import Matrix, layer_of

pytestmark = pytest.mark.gpu


def draw(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16().to(G.DEV)


class Chain:
    """Norm with quantiser, product back to the width, linear in place, norm: every call reads what the one before wrote, and the
    linear's output lies where its input was."""

    def __init__(self, seed, fmt, m, k, h, had):
        self.fmt, self.m, self.k, self.had = fmt, m, k, had
        self.up, self.down = layer_of(Matrix(seed, h, k, fmt, k ** -0.5), "bf16"), layer_of(Matrix(seed + 1, k, h, fmt, h ** -0.5), "bf16")
        self.square = layer_of(Matrix(seed + 2, k, k, fmt, k ** -0.5), "bf16", had=had)
        self.norm = Q.BlockNorm(Q.NORM_RMS, Q.BF16, pre_weight=draw(seed, k), weight_offset=1.0)
        self.start, self.branch = draw(seed + 3, m, k), draw(seed + 4, m, k)
        self.r, self.y = torch.empty_like(self.start), torch.empty_like(self.start)
        self.wide = torch.empty(m, h, dtype=torch.bfloat16, device=G.DEV)
        self.codes = torch.empty(m, k // 2, dtype=torch.uint8, device=G.DEV)
        self.scales = torch.empty(Q.qvla_fp4_scale_bytes(fmt, m, k), dtype=torch.uint8, device=G.DEV)
        self.row = torch.empty(m, device=G.DEV)
        self.size = max(Q.qvla_fp4_linear_workspace_bytes(x, m) for x in (self.down, self.square))
        self.work = torch.empty(self.size, dtype=torch.uint8, device=G.DEV)

    def calls(self, st):
        m, k = self.m, self.k
        yield Q.qvla_block_norm_fp4(self.norm, self.r, Q.BF16, k, self.y, k, m, k, self.r, None, 1, self.fmt, None, self.codes, self.scales, self.row, st)
        yield Q.qvla_gemm_fp4(self.up, self.codes, self.scales, self.row, m, self.wide, st)
        yield Q.qvla_fp4_linear(self.down, self.wide, m, None, self.y, self.work, self.size, st)
        yield Q.qvla_fp4_linear(self.square, self.y, m, None, self.y, self.work, self.size, st)
        yield Q.qvla_block_norm(self.norm, self.r, Q.BF16, k, self.y, k, m, k, self.r, self.y, st)

    def run(self, turns, stream, apart=False):
        with torch.cuda.stream(stream):
            self.r.copy_(self.start)
            self.y.copy_(self.branch)
            for _ in range(turns):
                for _ in self.calls(stream):
                    if apart:
                        stream.synchronize()
            stream.synchronize()
        return self.r.clone(), self.y.clone()


SIZES = [(1, 1024, 2048, 1024), (16, 512, 1024, 64), (50, 1024, 512, 1), (130, 2048, 1024, 2048), (400, 512, 2048, 256)]


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("m,k,h,had", SIZES)
def test_a_chain_without_pauses(fmt, m, k, h, had):
    chain, stream = Chain(m, fmt, m, k, h, had), torch.cuda.Stream()
    want = chain.run(8, stream, apart=True)
    assert all(torch.isfinite(t.float()).all() for t in want)
    for _ in range(3):
        got = chain.run(8, stream)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    Q.qvla_check_device(G.stream())


@pytest.mark.parametrize("a,b", [((F.MX, *SIZES[0]), (F.NV, *SIZES[3])), ((F.NV, *SIZES[1]), (F.NV, *SIZES[4])), ((F.MX, *SIZES[4]), (F.MX, *SIZES[2])),
                                 ((F.NV, *SIZES[0]), (F.MX, *SIZES[0]))])
def test_two_threads(a, b):
    chains, streams = [Chain(7, *a), Chain(70, *b)], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = [c.run(20, s, apart=True) for c, s in zip(chains, streams)]
    got = [None, None]

    def work(i):
        got[i] = chains[i].run(20, streams[i])

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))
    Q.qvla_check_device(G.stream())
