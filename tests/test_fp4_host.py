"""4-bit floating point and block norms without a GPU: the oracle's pins, weight packing to the bit, every refusal."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from oracle import qvla_oracle as O
from paper_2605_28803_gb300 import qvla as Q

BUF = torch.zeros(1 << 16, dtype=torch.uint8)
PTR = (BUF.data_ptr() + 255) // 256 * 256  # an aligned address; none of these calls gets as far as using it
INF, NAN = float("inf"), float("nan")


# ---- the oracle ---------------------------------------------------------------------------------------------------

def test_small_floats():
    assert list(F.E4M3[:10]) == [i / 512 for i in range(8)] + [1 / 64, 9 / 512] and F.E4M3[126] == 448 and F.E4M3[56] == 1
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(F.E4M3, t)


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.2501, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.01, 7), (99.0, 7)])
def test_ties_go_to_even_codes(x, code):
    assert F.nearest(np.array([x]), F.E2M1)[0] == code


def test_quantize_worked():
    # MX: the largest is 7 = 1.75 * 2^2, so e = 0, and 7 becomes 6; -1.25 is a tie between 1 and 1.5
    z = np.zeros((1, 32), np.float32)
    z[0, :4] = [7, -1.25, 0.75, 3.5]
    c, s, _ = F.quantize(z, F.MX)
    assert list(c[0, :4]) == [7, 10, 2, 6] and s[0, 0] == 127
    # NV: the row's largest, 2688, gives Delta 1 and the scale 448; a block whose largest is 6 gives the scale 1
    z = np.zeros((1, 32), np.float32)
    z[0, 0], z[0, 16], z[0, 17] = 2688, 6, -2.5
    c, s, d = F.quantize(z, F.NV)
    assert d[0] == 1 and list(s[0]) == [126, 56] and c[0, 0] == 7 and c[0, 16] == 7 and c[0, 17] == 12


def test_tiles():
    s = np.arange(200 * 8).reshape(200, 8).astype(np.uint8)
    t = F.to_tiles(s)
    for m, b in ((0, 0), (31, 3), (32, 0), (127, 5), (128, 4), (199, 7)):
        at = ((m // 128) * 2 + b // 4) * 512 + (m % 32) * 16 + (m // 32 % 4) * 4 + b % 4
        assert t[at] == s[m, b]
    assert np.array_equal(F.from_tiles(t, 200, 8), s)


# ---- packing --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [F.MX, F.NV])
@pytest.mark.parametrize("n,k,had,dtype", [(16, 128, 1, "f32"), (48, 384, 128, "bf16"), (144, 512, 16, "f16"), (16, 4096, 2048, "f32")])
def test_pack_matches_the_oracle(fmt, n, k, had, dtype):
    rng = np.random.default_rng(n + k)
    w = rng.standard_normal((n, k)).astype(np.float32) * np.float32(10.0) ** rng.integers(-30, 20, (n, 1)).astype(np.float32)
    w[0], w[1, : k // 2] = 0, 0
    if dtype != "f32":
        w = np.clip(w, -6e4, 6e4)
    t = torch.from_numpy(w).to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype])
    raw = t.view(torch.int16).numpy() if dtype != "f32" else t.numpy()
    wq, ws, row = np.full((n, k // 2), 99, np.uint8), np.full(Q.qvla_fp4_scale_bytes(fmt, n, k), 99, np.uint8), np.full(n, 9, np.float32)
    Q.qvla_fp4_pack_weights_host(np.ascontiguousarray(raw), Q.DTYPE_CODES[dtype], n, k, had_block=had, fmt=fmt, wq=wq, ws=ws,
                                 wscale=row if fmt == F.NV else None)
    z = t.double().numpy()
    if had > 1:  # float64 sums, then one float64 product, as the fold is defined
        z = (z.reshape(-1, had) @ O.sylvester_hadamard(had)).reshape(z.shape) * (1.0 / np.sqrt(had))
    codes, scale, delta = F.quantize(z.astype(np.float32), fmt)
    if had == 1:
        assert np.array_equal(wq, F.pack(codes)) and np.array_equal(ws, F.to_tiles(scale))
        if fmt == F.NV:
            assert np.array_equal(row, delta)
    else:  # sums of float32 numbers in float64 differ between two orders in last bits, and a value may cross a tie: hardly ever
        def unsigned_zeros(c):
            return np.where((c & 7) == 0, 0, c)

        assert (unsigned_zeros(F.unpack(wq)) != unsigned_zeros(codes)).mean() < 1e-3 and (ws != F.to_tiles(scale)).mean() < 1e-3
        if fmt == F.NV:
            assert np.allclose(row, delta, rtol=2e-7)


def test_pack_folds_the_permutation_and_rotation():
    rng = np.random.default_rng(3)
    n, k = 16, 128
    w, perm = rng.standard_normal((n, k)).astype(np.float32), rng.permutation(k).astype(np.int32)
    out = [(np.empty((n, k // 2), np.uint8), np.empty(Q.qvla_fp4_scale_bytes(F.NV, n, k), np.uint8), np.empty(n, np.float32)) for _ in range(2)]
    Q.qvla_fp4_pack_weights_host(w, Q.F32, n, k, perm=perm, wq=out[0][0], ws=out[0][1], wscale=out[0][2])
    Q.qvla_fp4_pack_weights_host(np.ascontiguousarray(w[:, perm]), Q.F32, n, k, wq=out[1][0], ws=out[1][1], wscale=out[1][2])
    assert all(np.array_equal(a, b) for a, b in zip(*out))
    rot = np.stack([np.linalg.qr(rng.standard_normal((32, 32)))[0] for _ in range(4)])
    Q.qvla_fp4_pack_weights_host(w, Q.F32, n, k, rot=rot, rot_block=32, wq=out[0][0], ws=out[0][1], wscale=out[0][2])
    z = np.concatenate([w[:, 32 * i: 32 * i + 32].astype(np.float64) @ rot[i] for i in range(4)], 1)
    got = F.values(F.unpack(out[0][0]), F.from_tiles(out[0][1], n, 8), F.NV) * out[0][2][:, None]
    # a code is half a step (1/4 of the value at most, 1 of 6 at the top) off, plus half an E4M3 step of a scale (1/16)
    assert np.abs(got - z).max() < 0.35 * np.abs(z).max()
    assert np.linalg.norm(got - z) < 0.15 * np.linalg.norm(z)


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_pack_refuses_weights_that_are_not_finite(bad):
    w = np.ones((16, 128), np.float32)
    w[5, 7] = bad
    b = np.empty(1 << 14, np.uint8)
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_fp4_pack_weights_host(w, Q.F32, 16, 128, wq=b, ws=b.copy(), wscale=np.empty(16, np.float32))
    assert e.value.status == 1


# ---- refusals ---------------------------------------------------------------------------------------------------------

def call(name, defaults, **kw):
    a = dict(defaults)
    assert set(kw) <= set(a)
    a.update(kw)
    return getattr(Q._lib, name)(*a.values())


QUANT = dict(x=PTR, xdt=Q.BF16, stride=256, M=4, K=256, had=64, fmt=Q.NVFP4, step=0, xq=PTR, xs=PTR, xscale=PTR, stream=None)
DEQUANT = dict(xq=PTR, xs=PTR, xscale=PTR, fmt=Q.NVFP4, M=4, K=256, out=PTR, odt=Q.F32, stream=None)
PACK = dict(W=PTR, wdt=Q.F32, N=16, K=128, rot=0, rot_block=0, perm=0, had=1, fmt=Q.NVFP4, wq=PTR, ws=PTR, wscale=PTR)


@pytest.mark.parametrize("kw,status", [
    (dict(xdt=3), 1), (dict(fmt=2), 1), (dict(fmt=-1), 1), (dict(M=-1), 1), (dict(M=(1 << 20) + 1), 1), (dict(K=0), 1), (dict(K=192), 1),
    (dict(K=16512, stride=16512, had=1), 2), (dict(had=3), 1), (dict(had=0), 1), (dict(had=512), 1), (dict(K=8192, stride=8192, had=8192), 2),
    (dict(stride=248), 1), (dict(stride=260), 1), (dict(stride=(1 << 31) + 8), 1), (dict(x=0), 1), (dict(x=PTR + 8), 1), (dict(xq=0), 1),
    (dict(xq=PTR + 4), 1), (dict(xs=0), 1), (dict(xs=PTR + 8), 1), (dict(xscale=0), 1), (dict(fmt=Q.MXFP4, step=PTR), 1)])
def test_quantize_refusals(kw, status):
    assert call("qvla_fp4_quantize_rows", QUANT, **kw) == status
    assert Q._lib.qvla_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(odt=3), 1), (dict(fmt=2), 1), (dict(M=-1), 1), (dict(K=64), 1), (dict(xq=0), 1), (dict(xs=0), 1), (dict(xscale=0), 1), (dict(out=0), 1),
    (dict(out=PTR + 8), 1)])
def test_dequantize_refusals(kw, status):
    assert call("qvla_fp4_dequantize_rows", DEQUANT, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(W=0), 1), (dict(wdt=3), 1), (dict(N=0), 1), (dict(N=24), 1), (dict(K=100), 1), (dict(had=256), 1), (dict(fmt=7), 1), (dict(wq=0), 1),
    (dict(ws=0), 1), (dict(wscale=0), 1), (dict(rot=PTR, rot_block=100), 1), (dict(rot=PTR, rot_block=0), 1), (dict(perm=PTR), 1)])
def test_pack_refusals(kw, status):
    assert call("qvla_fp4_pack_weights_host", PACK, **kw) == status


def test_scale_bytes():
    assert Q.qvla_fp4_scale_bytes(Q.NVFP4, 1, 128) == 1024 and Q.qvla_fp4_scale_bytes(Q.MXFP4, 129, 256) == 2048
    assert Q.qvla_fp4_scale_bytes(Q.NVFP4, 0, 128) == 0
    for bad in ((2, 1, 128), (1, -1, 128), (1, 1, 100), (1, 1, 0), (1, 1, 16512)):
        assert Q.qvla_fp4_scale_bytes(*bad) == 0


def layer_args(gated=False, **kw):
    n, k = (128, 128) if gated else (16, 128)
    rows = 2 * n if gated else n
    a = dict(N=n, K=k, had=1, fmt=Q.NVFP4, xdt=Q.BF16, ydt=Q.BF16, wq=np.zeros((rows, k // 2), np.uint8),
             ws=np.zeros(Q.qvla_fp4_scale_bytes(Q.NVFP4, rows, k), np.uint8), wscale=np.ones(rows, np.float32), bias=None)
    a.update(kw)
    return a


def one(n, at, value, dtype):
    x = np.zeros(n, dtype)
    x[at] = value
    return x


@pytest.mark.parametrize("kw,status", [
    (dict(N=0), 1), (dict(N=20), 1), (dict(K=64), 1), (dict(K=16512), 2), (dict(had=256), 1), (dict(fmt=2), 1), (dict(xdt=3), 1), (dict(ydt=Q.F32), 1),
    (dict(wq=None), 1), (dict(ws=None), 1), (dict(wscale=None), 1), (dict(fmt=Q.MXFP4), 1), (dict(wscale=one(16, 3, NAN, np.float32)), 1),
    (dict(wscale=one(16, 3, INF, np.float32)), 1), (dict(wscale=one(16, 3, -1, np.float32)), 1), (dict(ws=one(1024, 16 * 15 + 3, 0x7F, np.uint8)), 1),
    (dict(ws=one(1024, 0, 0x80, np.uint8)), 1), (dict(fmt=Q.MXFP4, wscale=None, ws=one(512, 1, 0xFF, np.uint8)), 1)])
def test_layer_refusals(kw, status):
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_fp4_layer_create(*layer_args(**kw).values())
    assert e.value.status == status


@pytest.mark.parametrize("n", [0, 16, 64, 192, -128])
def test_gated_layer_refusals(n):
    with pytest.raises(Q.QvlaError) as e:
        Q.qvla_fp4_layer_create_gated(*layer_args(True, N=n).values())
    assert e.value.status == 1


def test_a_null_layer_is_refused():
    assert Q._lib.qvla_gemm_fp4(None, PTR, PTR, PTR, 1, PTR, None) == 1
    assert Q._lib.qvla_fp4_linear(None, PTR, 1, None, PTR, PTR, 1 << 20, None) == 1
    assert Q._lib.qvla_fp4_linear_workspace_bytes(None, 1) == 0
    assert Q._lib.qvla_fp4_layer_destroy(None) == 0


def norm_struct(**kw):
    f = dict(kind=Q.NORM_RMS, eps=1e-6, weight_offset=1.0, residual_scale=1.0, post_norm=0, post_weight=None, pre_weight=PTR, pre_bias=None, gate=None,
             scale=None, shift=None, mod_stride=0, mod_rows=0, mod_tokens=0, mod_index=None)
    f.update(kw)
    return Q._NormStruct(*f.values())


NORM = dict(norm=None, dt=Q.BF16, r=PTR, rdt=Q.BF16, r_stride=256, y=PTR, y_stride=256, M=4, K=256, r_out=PTR, h=PTR)
MOD = dict(gate=PTR, mod_stride=256, mod_rows=2, mod_tokens=2)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("struct,kw,status", [
    (dict(kind=2), {}, 1), (dict(eps=0.0), {}, 1), (dict(eps=-1.0), {}, 1), (dict(eps=INF), {}, 1), (dict(eps=NAN), {}, 1), (dict(weight_offset=NAN), {}, 1),
    (dict(residual_scale=INF), {}, 1), (dict(post_weight=PTR), {}, 1), (dict(pre_weight=PTR + 8), {}, 1), (dict(pre_bias=PTR + 2), {}, 1),
    (dict(MOD, gate=PTR + 8), {}, 1), (dict(MOD, mod_stride=250), {}, 1), (dict(MOD, mod_stride=248), {}, 1), (dict(MOD, mod_rows=0), {}, 1),
    (dict(MOD, mod_rows=1), {}, 1), (dict(MOD, mod_tokens=0), {}, 1), ({}, dict(dt=Q.F32), 1), ({}, dict(rdt=Q.F16), 1), ({}, dict(rdt=4), 1),
    ({}, dict(M=-1), 1), ({}, dict(M=(1 << 20) + 1), 1), ({}, dict(K=0), 1), ({}, dict(K=252), 1), ({}, dict(K=16392, r_stride=16392, y_stride=16392), 2),
    ({}, dict(r=0), 1), ({}, dict(r=PTR + 8), 1), ({}, dict(r_stride=248), 1), ({}, dict(r_stride=257), 1), ({}, dict(y=PTR + 8), 1), ({}, dict(y_stride=0), 1),
    ({}, dict(r_out=PTR + 8), 1), ({}, dict(h=PTR + 8), 1), ({}, dict(r_out=0), 1), (dict(residual_scale=2.0), dict(y=0, r_out=0), 1)])
def test_norm_refusals(quant, struct, kw, status):
    s = norm_struct(**struct)
    a = dict(NORM, norm=ctypes.addressof(s))
    tail = dict(had=64, fmt=Q.NVFP4, step=None, hq=PTR, hs=PTR, hscale=PTR) if quant else {}
    assert call("qvla_block_norm_fp4" if quant else "qvla_block_norm", {**a, **tail, "stream": None}, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(K=248, r_stride=248, y_stride=248), 1), (dict(had=512), 1), (dict(had=5), 1), (dict(fmt=3), 1), (dict(hq=0), 1), (dict(hs=PTR + 8), 1), (dict(hscale=0), 1),
    (dict(fmt=Q.MXFP4, step=PTR), 1), (dict(K=8200, r_stride=8200, y_stride=8200), 1)])
def test_norm_quantizer_refusals(kw, status):
    s = norm_struct()
    base = dict(NORM, norm=ctypes.addressof(s), had=64, fmt=Q.NVFP4, step=None, hq=PTR, hs=PTR, hscale=PTR, stream=None)
    assert call("qvla_block_norm_fp4", base, **kw) == status


def test_nothing_to_write_is_refused_and_nothing_to_do_is_no_error():
    s = norm_struct()
    a = dict(NORM, norm=ctypes.addressof(s), stream=None)
    assert call("qvla_block_norm", a, y=0, r_out=0, h=0) == 1
    assert call("qvla_block_norm", a, norm=0) == 1
    assert call("qvla_block_norm", a, M=0, r=0, y=0, r_out=PTR) == 0
    assert call("qvla_fp4_quantize_rows", QUANT, M=0, x=0, xq=0, xs=0, xscale=0) == 0
    assert call("qvla_fp4_dequantize_rows", DEQUANT, M=0, xq=0, xs=0, xscale=0, out=0) == 0


def test_conditioning_of_unlike_shapes_is_refused():
    a, b = torch.zeros(2, 256), torch.zeros(3, 256)
    with pytest.raises(ValueError):
        Q.BlockNorm(Q.NORM_RMS, Q.F16, gate=a, scale=b)
    with pytest.raises(ValueError):
        Q.BlockNorm(Q.NORM_RMS, Q.F16, gate=a, shift=torch.zeros(2, 512)[:, :256])
    with pytest.raises(ValueError):
        Q.BlockNorm(Q.NORM_RMS, Q.F16, gate=a.T.contiguous().T)
