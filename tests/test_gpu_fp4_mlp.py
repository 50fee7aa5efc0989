"""The 4-bit operators together as an MLP block: against the separate calls to the bit, and against the block in float64."""

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from paper_2605_28803_gb300.fp4_mlp import Fp4Mlp
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


class Setup:
    def __init__(self, fmt, dtype, rdtype, k, h, had_in, had_hidden, layer, cond, tokens, seed=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.rdtype, self.k, self.h, self.layer, self.cond, self.eps = dtype, rdtype, k, h, layer, cond, 1e-5
        code = Q.DTYPE_CODES[dtype]
        self.w_gu = (rng.standard_normal((2 * h, k)) / np.sqrt(k)).astype(np.float32)
        self.w_d = (rng.standard_normal((k, h)) / np.sqrt(h)).astype(np.float32)

        def pack(w, had):
            n, kk = w.shape
            wq, ws, row = np.empty((n, kk // 2), np.uint8), np.empty(Q.qvla_fp4_scale_bytes(fmt, n, kk), np.uint8), np.empty(n, np.float32)
            Q.qvla_fp4_pack_weights_host(w, Q.F32, n, kk, had_block=had, fmt=fmt, wq=wq, ws=ws, wscale=row)
            return wq, ws, row if fmt == F.NV else None

        self.gate_up = Q.qvla_fp4_layer_create_gated(h, k, had_in, fmt, code, code, *pack(self.w_gu, had_in))
        self.down = Q.qvla_fp4_layer_create(k, h, had_hidden, fmt, code, code, *pack(self.w_d, had_hidden))
        g = torch.Generator(device=G.DEV).manual_seed(seed)
        self.norms = []
        for _ in range(2):
            w = (torch.randn(k, generator=g, device=G.DEV) * 0.2).to(DT[dtype])
            mods = {}
            if cond:
                m = (torch.randn(-(-tokens // cond), 3 * k, generator=g, device=G.DEV) * 0.3).to(DT[dtype])
                mods = dict(gate=m[:, :k], scale=m[:, k: 2 * k], shift=m[:, 2 * k:], mod_tokens=cond)
            self.norms.append(Q.BlockNorm(Q.NORM_LAYER if layer else Q.NORM_RMS, code, eps=self.eps, weight_offset=1.0, pre_weight=w, **mods))
        self.block = Fp4Mlp(self.gate_up, self.down, *self.norms, tokens, Q.DTYPE_CODES[rdtype])
        self.g = g

    def inputs(self, m):
        r = (torch.randn(m, self.k, generator=self.g, device=G.DEV) * 2).to(DT[self.rdtype])
        y = torch.randn(m, self.k, generator=self.g, device=G.DEV).to(DT[self.dtype])
        return r, y

    def float64(self, r, y):
        r, y = r.double().cpu().numpy(), y.double().cpu().numpy()
        token = np.arange(r.shape[0]) // max(1, self.cond)

        def junction(r, y, plan):
            _, w, _, gate, scale, shift, _ = plan.tensors
            of = lambda t: t.double().cpu().numpy()[token]  # noqa: E731
            r = r + (y if gate is None else y * of(gate))
            h = F.norm(r, self.layer, self.eps) * (1 + w.double().cpu().numpy())
            return r, h if scale is None else h * (1 + of(scale)) + of(shift)

        r, h = junction(r, y, self.norms[0])
        a = h @ self.w_gu.astype(np.float64).T
        out = (F.gelu(a[:, : self.h]) * a[:, self.h:]) @ self.w_d.astype(np.float64).T
        return junction(r, out, self.norms[1])


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype,rdtype,k,h,had_in,had_hidden,layer,cond,m", [
    ("bf16", "bf16", 512, 1024, 512, 1024, False, 0, 1), ("f16", "f32", 256, 512, 64, 256, True, 50, 200), ("bf16", "f32", 1024, 4096, 1, 1, False, 0, 130)])
def test_block(fmt, dtype, rdtype, k, h, had_in, had_hidden, layer, cond, m):
    s = Setup(fmt, dtype, rdtype, k, h, had_in, had_hidden, layer, cond, m)
    r, y = s.inputs(m)
    want_r, want_h = s.float64(r, y)
    got_r = r.clone()
    got_h = s.block(got_r, y).clone()
    Q.qvla_check_device(G.stream())
    # every quantised matrix of the two products is off by 4-bit codes: half a step is 1/12 of a block's largest entry, in the
    # mean 10% of a Gaussian's entries' size, and a product of two such is 15% off; two of them in a row, the first through a
    # GELU times a second factor (twice the relative error): sqrt((2 * .15)^2 + .15^2) = .34 of the MLP's output
    first = r.double().cpu().numpy() + y.double().cpu().numpy() * (1 if not cond else s.norms[0].tensors[3].double().cpu().numpy()[np.arange(m) // cond])
    branch = np.linalg.norm(want_r - first)
    assert np.linalg.norm(got_r.double().cpu().numpy() - want_r) < 0.34 * branch + 2.0 ** -8 * np.linalg.norm(want_r)
    # and the separate calls give the same bits
    code, rcode, up, down, st = Q.DTYPE_CODES[dtype], Q.DTYPE_CODES[rdtype], s.gate_up, s.down, G.stream()
    r2, hh, hid, out, nxt = r.clone(), *(torch.empty(m, n, dtype=DT[dtype], device=G.DEV) for n in (k, h, k, k))
    Q.qvla_block_norm(s.norms[0], r2, rcode, k, y, k, m, k, r2, hh, st)
    work = torch.empty(max(Q.qvla_fp4_linear_workspace_bytes(up, m), Q.qvla_fp4_linear_workspace_bytes(down, m)), dtype=torch.uint8, device=G.DEV)
    Q.qvla_fp4_linear(up, hh, m, None, hid, work, work.numel(), st)
    Q.qvla_fp4_linear(down, hid, m, None, out, work, work.numel(), st)
    Q.qvla_block_norm(s.norms[1], r2, rcode, k, out, k, m, k, r2, nxt, st)
    Q.qvla_check_device(st)
    assert torch.equal(r2, got_r) and torch.equal(nxt, got_h)
    assert code == s.block.dt


def test_fewer_tokens_graphs_and_streams():
    s = Setup(F.NV, "bf16", "bf16", 256, 512, 256, 512, False, 0, 64)
    r, y = s.inputs(64)
    want = {}
    for m in (64, 9):
        rr = r[:m].clone()
        want[m] = s.block(rr, y[:m]).clone(), rr
    # the sums' order may depend on the number of tokens: last bits, and here and there a code beside a border
    for a, b in zip(want[9], want[64]):
        assert (a.float() - b[:9].float()).norm() < 0.02 * a.float().norm()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rr = r.clone()
        got = s.block(rr, y).clone()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[64][0]) and torch.equal(rr, want[64][1])
    # two graphs that share the block's buffers, replayed in turn
    torch.cuda.synchronize()
    graphs = []
    for m in (64, 9):
        rr, yy = r[:m].clone(), y[:m].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            n = s.block(rr, yy)
        graphs.append((g, rr, yy, n, m))
    for _ in range(2):
        for g, rr, _, n, m in graphs:
            rr.copy_(r[:m])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(n, want[m][0]) and torch.equal(rr, want[m][1])
    Q.qvla_check_device(G.stream())
