"""Residual, gate and norms between two blocks on the GPU, against float64.

The bound on r': two float32 roundings of a number of the terms' size, and half a step of the residual's type.  The bound on h:
the norm reads r' as stored, so its inputs are exact; a sum of K squares in float32, 32 to a thread and then a tree, is off by
at most 40 roundings, its square root by half as many: 24 2^-24, with the mean's error (40 2^-24 of the mean magnitude) added
where it is subtracted; five more roundings of the terms that are multiplied and added; half a step of the output's type."""

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2605_28803_gb300 import qvla as Q
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


class Case:
    def __init__(self, m, k, dtype, rdtype, layer=False, branch=True, post=False, weights=True, cond=0, index=False, alpha=1.0, offset=1.0, pad=0, seed=0):
        g = torch.Generator().manual_seed(m * 31 + k + seed)

        def draw(*shape, mean=0.0, spread=1.0, dt=dtype):
            return (torch.randn(*shape, generator=g) * spread + mean).to(DT[dt]).to(G.DEV)

        self.m, self.k, self.dtype, self.rdtype, self.layer, self.alpha, self.offset, self.eps = m, k, dtype, rdtype, layer, alpha, offset, 1e-5
        wide = draw(m, k + pad, spread=3.0, mean=0.5, dt=rdtype)
        wide[:, k:] = float("nan")
        self.r = wide[:, :k]
        self.y = None
        if branch:
            y = draw(m, k + 2 * pad, spread=2.0, mean=-0.3)
            y[:, k:] = float("nan")
            self.y = y[:, :k]
        self.post = post
        self.post_w = draw(k, spread=0.3) if post and weights else None
        self.pre_w = draw(k, spread=0.3) if weights else None
        self.pre_b = draw(k, spread=0.2) if weights and layer else None
        self.gate = self.scale = self.shift = self.index = None
        self.cond = cond
        if cond:
            n = -(-m // cond)
            mod = draw(n, 3 * k, spread=0.5)
            self.gate, self.scale, self.shift = mod[:, :k], mod[:, k: 2 * k], mod[:, 2 * k:]
            if index:
                self.index = torch.randint(0, n, (m,), generator=g, dtype=torch.int32).to(G.DEV)

    def plan(self):
        return Q.BlockNorm(Q.NORM_LAYER if self.layer else Q.NORM_RMS, Q.DTYPE_CODES[self.dtype], eps=self.eps, weight_offset=self.offset,
                           residual_scale=self.alpha, post_norm=self.post, post_weight=self.post_w, pre_weight=self.pre_w, pre_bias=self.pre_b,
                           gate=self.gate, scale=self.scale, shift=self.shift, mod_tokens=self.cond, mod_index=self.index)

    def run(self, r_out=True, h=True, stream=None, plan=None):
        out = torch.full((self.m + 1, self.r.stride(0)), 9.0, dtype=DT[self.rdtype], device=G.DEV) if r_out is True else r_out
        ho = torch.full((self.m + 1, self.k), 9.0, dtype=DT[self.dtype], device=G.DEV) if h else None
        Q.qvla_block_norm(plan or self.plan(), self.r, Q.DTYPE_CODES[self.rdtype], self.r.stride(0), self.y, 0 if self.y is None else self.y.stride(0), self.m,
                          self.k, out, ho, stream or G.stream())
        Q.qvla_check_device(stream or G.stream())
        if r_out is True:
            assert (out[self.m] == 9.0).all() and (out[:, self.k:] == 9.0).all()
        if h:
            assert (ho[self.m] == 9.0).all()
        return (out[: self.m, : self.k] if out is not None else None), (ho[: self.m] if h else None)

    def token(self):
        i = torch.arange(self.m, device=G.DEV) // self.cond if self.index is None else self.index.long()
        return i.cpu().numpy()

    def weight(self, w):
        return 1.0 if w is None else w.double().cpu().numpy() + self.offset

    def of(self, name):
        return getattr(self, name).double().cpu().numpy()[self.token()] if self.cond else (0.0 if name != "gate" else 1.0)

    def check_residual(self, got):
        r, off = self.alpha * self.r.double().cpu().numpy(), 0.0
        size = np.abs(r)
        if self.y is not None:
            u = self.y.double().cpu().numpy()
            off = np.zeros_like(u)
            if self.post:
                n = F.norm(u, self.layer, self.eps)
                off = norm_off(u, n, self.layer) * np.abs(self.weight(self.post_w)) + 4 * U * np.abs(n * self.weight(self.post_w))
                u = n * self.weight(self.post_w)
            u, off = u * self.of("gate"), off * np.abs(self.of("gate")) + 2 * U * np.abs(u * self.of("gate"))
            r, size = r + u, size + np.abs(u)
        off = off + 2 * U * size
        # (below 2^-14 float16 numbers are 2^-24 apart, so that a rounding is off by up to 2^-25 whatever the value's size)
        assert_within(got, r, off + HALF[self.rdtype] * (np.abs(r) + off) + (2.0 ** -25 if self.rdtype == "f16" else 1e-300))

    def check_h(self, got, residual):
        """`residual`: the one the kernel stored."""
        x = residual.double().cpu().numpy()
        n = F.norm(x, self.layer, self.eps)
        w = self.weight(self.pre_w)
        off = norm_off(x, n, self.layer)
        b = 0.0 if self.pre_b is None else self.pre_b.double().cpu().numpy()
        a, shift = n * w + b, self.of("shift")
        off = (off * np.abs(w) + 4 * U * (np.abs(n * w) + np.abs(b))) * np.abs(1 + self.of("scale"))
        want = a * (1 + self.of("scale")) + shift
        off = off + 3 * U * (np.abs(a) * (1 + np.abs(self.of("scale"))) + np.abs(shift))
        tiny = 2.0 ** -25 if self.dtype == "f16" else 0.0
        assert_within(got, want, off + HALF[self.dtype] * (np.abs(want) + off) + tiny)


def norm_off(x, n, layer, eps=1e-5):
    off = 28 * U * np.abs(n)
    if layer:  # the mean is off by 40 roundings of the mean magnitude, the difference by one more; the quotient passes that on
        d = x - x.mean(-1, keepdims=True)
        off = off + (40 * np.abs(x).mean(-1, keepdims=True) + np.abs(x)) * U / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return off


def assert_within(got, want, off):
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= off).all(), (np.abs(got - want) / off).max()


SHAPES = [(1, 8), (1, 1024), (3, 24), (5, 1000), (7, 1032), (50, 1024), (129, 256), (33, 2048), (2, 4104), (4, 8192), (1, 16384), (3, 16376), (700, 128), (300, 1152)]


@pytest.mark.parametrize("dtype,rdtype", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("m,k", SHAPES)
def test_everything_on(dtype, rdtype, layer, m, k):
    c = Case(m, k, dtype, rdtype, layer, post=m % 2 == 1, cond=max(1, m // 3), index=m % 3 == 0, alpha=1.0 if m % 2 else 0.5, pad=8 * (m % 4))
    r, h = c.run()
    c.check_residual(r)
    c.check_h(h, r)


@pytest.mark.parametrize("kw", [dict(branch=False), dict(branch=False, alpha=0.25), dict(weights=False), dict(weights=False, post=True), dict(layer=True, weights=False),
                                dict(post=True), dict(cond=4), dict(cond=4, branch=False), dict(offset=0.0), dict(alpha=-2.0)])
def test_parts_left_out(kw):
    c = Case(13, 520, "bf16", "bf16", **kw)
    r, h = c.run()
    c.check_residual(r)
    c.check_h(h, r)
    # the residual alone, the norm alone
    assert torch.equal(c.run(h=False)[0], r)
    if c.y is None and c.alpha == 1.0:
        assert torch.equal(c.run(r_out=None)[1], h)


@pytest.mark.parametrize("which", ["gate", "scale", "shift"])
def test_one_of_the_conditioning(which):
    c = Case(9, 256, "f16", "f32", cond=3)
    mod = getattr(c, which)
    c.gate = c.scale = c.shift = None
    setattr(c, which, mod)
    r, h = c.run()
    c.gate = mod if which == "gate" else torch.ones_like(mod)
    c.scale = mod if which == "scale" else torch.zeros_like(mod)
    c.shift = mod if which == "shift" else torch.zeros_like(mod)
    c.check_residual(r)
    c.check_h(h, r)


@pytest.mark.parametrize("rdtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k", [(5, 1024), (200, 2048), (3, 16384)])
def test_in_place(rdtype, m, k):
    c = Case(m, k, "bf16", rdtype, cond=m)
    r, h = c.run()
    before = c.r
    c.r = before.clone()
    _, h2 = c.run(r_out=c.r)
    assert torch.equal(c.r, r) and torch.equal(h2, h)


@pytest.mark.parametrize("quant", [False, True])
def test_an_index_out_of_range_skips_its_token(quant):
    c = Case(12, 256, "bf16", "bf16", cond=4, index=True)
    r, h = c.run()
    good = c.index.clone()
    c.index[3], c.index[7] = 3, -1  # of 3 rows
    plan = c.plan()
    out, ho = torch.full_like(r, 9.0), torch.full_like(h, 9.0)
    hq, hs, row = (torch.full((12, 128), 0x55, dtype=torch.uint8, device=G.DEV), torch.full((2048,), 0x55, dtype=torch.uint8, device=G.DEV),
                   torch.full((12,), 5.0, device=G.DEV))
    if quant:
        Q.qvla_block_norm_fp4(plan, c.r, Q.BF16, 256, c.y, 256, 12, 256, out, ho, 64, Q.NVFP4, None, hq, hs, row, G.stream())
    else:
        Q.qvla_block_norm(plan, c.r, Q.BF16, 256, c.y, 256, 12, 256, out, ho, G.stream())
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_check_device(G.stream())
    assert e.value.status == 1
    skipped = torch.zeros(12, dtype=torch.bool, device=G.DEV)
    skipped[3] = skipped[7] = True
    assert (out[skipped] == 9.0).all() and (ho[skipped] == 9.0).all()
    assert torch.equal(out[~skipped], r[~skipped]) and torch.allclose(ho[~skipped].float(), h[~skipped].float(), rtol=0.01, atol=0.01)
    if quant:
        scales = F.from_tiles(hs.cpu().numpy(), 12, 16)
        s = skipped.cpu().numpy()
        assert (hq[skipped] == 0x55).all() and (scales[s] == 0x55).all() and (row[skipped] == 5.0).all() and (row[~skipped] != 5.0).all()
    Q.qvla_check_device(G.stream())
    assert good is not None


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_stays_in_its_row(bad):
    c = Case(6, 512, "bf16", "bf16", post=True)
    r, h = c.run()
    c.y[2, 5] = bad
    r2, h2 = c.run()
    assert torch.isnan(h2[2]).all()
    keep = torch.arange(6, device=G.DEV) != 2
    assert torch.equal(r2[keep], r[keep]) and torch.equal(h2[keep], h[keep])


@pytest.mark.parametrize("layer", [False, True])
def test_constant_and_zero_rows(layer):
    c = Case(4, 768, "f16", "f16", layer, branch=False)
    c.r[0], c.r[1] = 0, 3.0
    r, h = c.run()
    c.check_h(h, r)


@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("dtype,rdtype", [("f16", "f16"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("m,k,had", [(1, 128, 1), (5, 384, 128), (50, 1024, 1024), (33, 2048, 2048), (129, 256, 64), (7, 1152, 16), (3, 4096, 4096), (2, 16384, 2048), (9, 2560, 512),
                                     (4, 1280, 256)])
def test_with_the_quantiser(fmt, dtype, rdtype, m, k, had):
    c = Case(m, k, dtype, rdtype, layer=m % 2 == 0, post=m % 3 == 0, cond=max(1, m // 2), pad=8 * (m % 3))
    out = torch.full((m, c.r.stride(0)), 9.0, dtype=DT[rdtype], device=G.DEV)
    h = torch.empty(m, k, dtype=DT[dtype], device=G.DEV)
    steps = [None] if fmt == F.MX else [None, torch.tensor([0.003], device=G.DEV)]
    for step in steps:
        results = []
        for ho in (h, None):
            hq = torch.full((m + 1, k // 2), 0x33, dtype=torch.uint8, device=G.DEV)
            hs = torch.full((Q.qvla_fp4_scale_bytes(fmt, m, k),), 0x33, dtype=torch.uint8, device=G.DEV)
            row = torch.full((m + 1,), 3.0, device=G.DEV)
            Q.qvla_block_norm_fp4(c.plan(), c.r, Q.DTYPE_CODES[rdtype], c.r.stride(0), c.y, c.y.stride(0), m, k, out, ho, had, fmt, step, hq, hs, row, G.stream())
            Q.qvla_check_device(G.stream())
            assert (hq[m] == 0x33).all() and row[m] == 3.0
            results.append((hq, hs, row))
        assert all(torch.equal(a, b) for a, b in zip(*results))
        c.check_residual(out[:, :k])
        c.check_h(h, out[:, :k])
        # the codes are those of h as it is stored
        want = torch.full_like(hq, 0x33), torch.full_like(hs, 0x33), torch.full_like(row, 3.0)
        Q.qvla_fp4_quantize_rows(h, Q.DTYPE_CODES[dtype], k, m, k, had, fmt, step, *want, G.stream())
        assert all(torch.equal(a, b) for a, b in zip(results[0], want))


def test_a_graph_and_another_stream():
    c = Case(50, 1024, "bf16", "bf16", layer=True, cond=50)
    side = torch.cuda.Stream()
    want = c.run()
    with torch.cuda.stream(side):
        got = c.run(stream=side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    plan, out, h = c.plan(), torch.empty_like(c.r), torch.empty(50, 1024, dtype=torch.bfloat16, device=G.DEV)
    call = lambda: Q.qvla_block_norm(plan, c.r, Q.BF16, 1024, c.y, 1024, 50, 1024, out, h, torch.cuda.current_stream())  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    c.y.mul_(0.5)
    c.gate.add_(0.25)
    graph.replay()
    torch.cuda.synchronize()
    c.check_residual(out)
    c.check_h(h, out)
