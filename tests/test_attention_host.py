"""Attention entry points without a GPU: every refusal, made before any device work, and the oracle's own pins."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2605_28803_gb300 import qvla as Q

BUF = torch.zeros(1 << 16, dtype=torch.uint8)
PTR = (BUF.data_ptr() + 255) // 256 * 256  # an aligned address; none of these calls gets as far as using it
INF, NAN = float("inf"), float("nan")


def prompt_args(**kw):
    a = dict(q=PTR, k=PTR, v=PTR, dt=Q.F16, heads=8, kv_heads=2, dim=64, qs=512, ks=128, vs=128, batch=1, cu_q=PTR, total_q=4,
             cu_k=PTR, total_k=4, scale=0.125, causal=1, o=PTR, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dt=Q.F32), 1), (dict(dt=9), 1), (dict(heads=0), 1), (dict(heads=9), 1), (dict(kv_heads=0), 1), (dict(heads=2048), 1),
    (dict(dim=96), 2), (dict(dim=512), 2), (dict(qs=511), 1), (dict(qs=504), 1), (dict(ks=120), 1), (dict(vs=0), 1),
    (dict(vs=-128), 1), (dict(qs=(1 << 31) + 8), 1), (dict(batch=-1), 1), (dict(batch=65536), 1), (dict(total_q=-1), 1),
    (dict(total_k=(1 << 24) + 1), 1), (dict(q=0), 1), (dict(k=0), 1), (dict(v=PTR + 2), 1), (dict(o=0), 1), (dict(o=PTR + 8), 1),
    (dict(cu_q=0), 1), (dict(cu_k=0), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=INF), 1), (dict(scale=NAN), 1)])
def test_prompt_refusals(kw, status):
    assert Q._lib.qvla_attention_prompt(*prompt_args(**kw)) == status
    assert Q._lib.qvla_last_error()


def test_nothing_to_do_is_no_error():
    assert Q._lib.qvla_attention_prompt(*prompt_args(batch=0, cu_q=0, cu_k=0)) == 0
    assert Q._lib.qvla_attention_prompt(*prompt_args(total_q=0, q=0, o=0)) == 0
    assert Q._lib.qvla_kv4_append(*append_args(total=0, k=0, v=0)) == 0
    assert Q._lib.qvla_kv4_gather(*gather_args(batch=0, cu=0, table=0)) == 0
    assert Q._lib.qvla_attention_kv4(*kv4_args(total_q=0)) == 0


def cache(**kw):
    f = dict(pool=PTR, num_pages=4, page_size=16, kv_heads=2, head_dim=64, rotate=1)
    f.update(kw)
    return Q._Kv4Struct(*f.values())


def address(c):
    return c if isinstance(c, int) else ctypes.addressof(GOOD if c is None else c)


def append_args(c=None, **kw):
    a = dict(c=address(c), k=PTR, v=PTR, dt=Q.BF16, ks=128, vs=128, batch=1,
             cu=PTR, total=4, table=PTR, max_pages=4, start=0, stream=None)
    a.update(kw)
    return list(a.values())


def gather_args(c=None, **kw):
    a = dict(c=address(c), batch=1, cu=PTR, total=4, table=PTR, max_pages=4,
             start=0, k=PTR, v=PTR, dt=Q.BF16, stream=None)
    a.update(kw)
    return list(a.values())


def kv4_args(c=None, **kw):
    a = dict(c=address(c), q=PTR, dt=Q.BF16, heads=8, qs=512, batch=1, cu=PTR,
             total_q=1, max_q=1, table=PTR, max_pages=4, kv_len=PTR, max_len=64, scale=0.125, causal=1, o=PTR, ws=0, ws_bytes=0,
             stream=None)
    a.update(kw)
    return list(a.values())


GOOD = cache()


@pytest.mark.parametrize("kw,status", [
    (dict(pool=0), 1), (dict(pool=PTR + 4), 1), (dict(num_pages=0), 1), (dict(page_size=8), 1), (dict(page_size=48), 1),
    (dict(page_size=512), 1), (dict(kv_heads=0), 1), (dict(kv_heads=3), 1), (dict(head_dim=80), 2)])
def test_cache_refusals(kw, status):
    c = cache(**kw)
    assert Q._lib.qvla_attention_kv4(*kv4_args(c)) == status
    if "kv_heads" not in kw or kw["kv_heads"] == 0:
        assert Q._lib.qvla_kv4_append(*append_args(c)) == status
        assert Q._lib.qvla_kv4_gather(*gather_args(c)) == status


@pytest.mark.parametrize("kw", [
    dict(c=0), dict(dt=Q.F32), dict(k=0), dict(v=PTR + 4), dict(ks=64), dict(vs=129), dict(batch=-1), dict(cu=0), dict(table=0),
    dict(max_pages=0), dict(total=-1), dict(total=(1 << 24) + 1)])
def test_append_refusals(kw):
    assert Q._lib.qvla_kv4_append(*append_args(**kw)) == 1
    kw = {k: v for k, v in kw.items() if k not in ("ks", "vs")}
    if kw:
        assert Q._lib.qvla_kv4_gather(*gather_args(**kw)) == 1


@pytest.mark.parametrize("kw", [
    dict(c=0), dict(q=0), dict(q=PTR + 8), dict(heads=7), dict(heads=0), dict(qs=448), dict(batch=70000), dict(cu=0), dict(table=0),
    dict(kv_len=0), dict(max_q=-1), dict(max_len=-1), dict(max_len=65), dict(scale=NAN), dict(scale=0.0), dict(o=0), dict(o=PTR + 2),
    dict(ws=PTR + 16, ws_bytes=4096), dict(ws=0, ws_bytes=256), dict(max_pages=0), dict(total_q=-2)])
def test_kv4_attention_refusals(kw):
    assert Q._lib.qvla_attention_kv4(*kv4_args(**kw)) == 1


def test_pool_bytes_and_the_binding():
    assert Q.qvla_kv4_pool_bytes(3, 64, 8, 128) == 3 * 64 * 8 * 136
    assert Q.qvla_kv4_pool_bytes(1 << 20, 256, 64, 256) == (1 << 20) * 256 * 64 * 264  # past 32 bits
    for bad in ((0, 64, 8, 128), (1, 24, 8, 128), (1, 64, 0, 128), (1, 64, 8, 100)):
        assert Q.qvla_kv4_pool_bytes(*bad) == 0
    with pytest.raises(ValueError):
        Q.Kv4Cache(torch.zeros(100, dtype=torch.uint8), 1, 16, 1, 64)
    assert Q.qvla_attention_kv4_workspace_bytes(0, 1, 64, 1, 1, 1, 1) == 0
    n = Q.qvla_attention_kv4_workspace_bytes(8, 1, 256, 1, 1, 1, 100000)
    assert n % 256 == 0


# ---- the oracle's own pins -----------------------------------------------------------------------------------------

def test_rotation_is_the_hadamard_matrix():
    rng = np.random.default_rng(1)
    for d in (64, 128, 256):
        x = rng.standard_normal((5, d))
        assert np.allclose(A.rotate_f32(x), x @ A.hadamard(d), atol=1e-5)
        assert np.allclose(A.hadamard(d) @ A.hadamard(d), np.eye(d))


def test_codes_worked_by_hand():
    c, d = A.quantize_heads(np.array([[7.0, 0.5, 1.5, -2.5, -7.0, 3.4, 0.0, 6.6]]), False)
    assert d[0] == 1.0 and c.tolist() == [[7, 0, 2, -2, -7, 3, 0, 7]]
    c, d = A.quantize_heads(np.zeros((1, 4)), False)
    assert d[0] == 0 and not c.any()
    c, d = A.quantize_heads(np.array([[1.0, np.nan], [np.inf, 1.0]]), False)
    assert np.isnan(d).all()
    codes = np.arange(-7, 8).astype(np.int8)[:14].reshape(1, 14)
    assert np.array_equal(A.unpack_nibbles(A.pack_nibbles(codes)), codes)
    assert A.pack_nibbles(np.array([[1, -1]], np.int8)).tolist() == [[0xF1]]


def test_read_back_is_the_rotation_of_code_times_scale():
    rng = np.random.default_rng(2)
    codes = rng.integers(-7, 8, (3, 2, 128)).astype(np.int8)
    scales = rng.uniform(0.1, 1.0, (3, 2)).astype(np.float32)
    want = (codes * scales[..., None].astype(np.float64)) @ A.hadamard(128)
    assert np.allclose(A.read_back(codes, scales, True), want, atol=1e-6)
    assert np.array_equal(A.read_back(codes, scales, False), codes.astype(np.float32) * scales[..., None])


def test_attention_worked_by_hand():
    q = np.zeros((2, 1, 2))
    k = np.ones((3, 1, 2))
    v = np.array([[[0.0, 3.0]], [[3.0, 3.0]], [[6.0, 9.0]]])
    o = A.attention(q, k, v, 1.0, True)[0]  # equal scores: means over the first 2, then 3 keys
    assert np.allclose(o[:, 0], [[1.5, 3.0], [3.0, 5.0]])
    q = np.array([[[1.0, 0.0]]])
    k = np.array([[[0.0, 5.0]], [[np.log(3.0), 5.0]]])
    assert np.allclose(A.attention(q, k, v[:2], 1.0, False)[0][0, 0], [2.25, 3.0])
    o = A.attention(np.ones((3, 2, 2)), np.ones((1, 1, 2)), v[:1], 1.0, True)[0]
    assert (o[:2] == 0).all() and (o[2] == [0.0, 3.0]).all()
