"""Binding of libqvla (include/qvla.h): the same entry points, argument marshalling only (by ctypes; the calls of the 4-bit
floating-point operators and norms by the compiled _calls).

Tensors are passed as raw pointers (``tensor.data_ptr()``) and streams as
``torch.cuda.Stream.cuda_stream``; every step of the computation runs in libqvla's kernels.
A non-zero status raises QvlaError with the library's message.  Importing this module loads
the in-tree libqvla.so and fails loudly if it has not been built; without _calls the calls that it
has fail loudly, and the others work.
"""

from __future__ import annotations

import ctypes
import os

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libqvla.so")

F16, BF16, F32 = 0, 1, 2
MXFP4, NVFP4 = 0, 1
NORM_RMS, NORM_LAYER = 0, 1
DTYPE_CODES = {"f16": F16, "bf16": BF16, "f32": F32}

STATUS = {0: "QVLA_OK", 1: "QVLA_ERR_INVALID_ARG", 2: "QVLA_ERR_UNSUPPORTED", 3: "QVLA_ERR_CUDA",
          4: "QVLA_ERR_OOM", 5: "QVLA_ERR_STEP_RANGE", 6: "QVLA_ERR_TIMEOUT"}

# every symbol include/*.h declares, with (restype, argtypes)
_P, _I, _S, _D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double
_L, _F = ctypes.c_int64, ctypes.c_float
SIGNATURES = {
    "qvla_last_error": (ctypes.c_char_p, []),
    "qvla_abi_version": (_I, []),
    "qvla_pack_weights_host": (_I, [_P, _I, _I, _I, _P, _I, _P, _I, _P, _P, _P]),
    "qvla_block_svd_rotation": (_I, [_P, _I, _I, _I, _I, _P, _P]),
    "qvla_gptq_pack_host": (_I, [_P, _I, _I, _I, _P, _I, _I, _P, _I, _P, _I, _I, _D, _P, _P, _P]),
    "qvla_layer_create": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, ctypes.POINTER(_P)]),
    "qvla_layer_create_gated": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, ctypes.POINTER(_P)]),
    "qvla_pack_weights": (_I, [_P, _I, _I, _I, _P, _I, _P, _I, _P, _I, _I, ctypes.POINTER(_P)]),
    "qvla_layer_destroy": (_I, [_P]),
    "qvla_set_step_scales": (_I, [_P, _P, _I]),
    "qvla_set_step_group_scales": (_I, [_P, _P, _I, _I]),
    "qvla_layer_scale_groups": (_I, [_P, _P, _P]),
    "qvla_layer_set_online_rotation": (_I, [_P, _P, _P, _I]),
    "qvla_online_rotate": (_I, [_P, _P, _I, _P, _P]),
    "qvla_rotated_absmax_groups": (_I, [_P, _I, _I, _I, _I, _P, _P]),
    "qvla_layer_info": (_I, [_P, _P, _P, _P, _P]),
    "qvla_rotate_quantize": (_I, [_P, _P, _I, _I, _P, _P, _P, _P]),
    "qvla_rotate_quantize_rows": (_I, [_P, _I, _I, _I, _I, _P, _P, _P, _P, _P]),
    "qvla_rotated_absmax": (_I, [_P, _I, _I, _I, _I, _P, _P]),
    "qvla_gemm_w4a4": (_I, [_P, _P, _P, _P, _I, _P, _P, _P]),
    "qvla_linear_workspace_bytes": (_S, [_P, _I]),
    "qvla_w4a4_linear": (_I, [_P, _P, _I, _I, _P, _P, _S, _P]),
    "qvla_linear_quantize": (_I, [_P, _P, _I, _I, _P, _S, _P]),
    "qvla_linear_gemm": (_I, [_P, _P, _S, _I, _P, _P]),
    "qvla_w4a4_linear_noalloc": (_I, [_P, _P, _I, _I, _P, _P]),
    "qvla_w4a4_linear_fused": (_I, [_P, _P, _I, _I, _P, _P]),
    "qvla_rotate_quantize_rows_a8": (_I, [_P, _I, _I, _I, _I, _P, _P, _P, _P, _P]),
    "qvla_w4a8_workspace_bytes": (_S, [_P, _I]),
    "qvla_w4a8_linear": (_I, [_P, _P, _I, _I, _P, _P, _S, _P]),
    "qvla_gemm_w4a8": (_I, [_P, _P, _P, _I, _P, _P, _P, _S, _P]),
    "qvla_check_device": (_I, [_P]),
    "qvla_debug_set_hooks": (_I, [ctypes.c_ulonglong, _I]),
    "qvla_debug_gemm_plan": (_I, [_I, _I, _I, _I, _I, _I, _P, _P]),
    "qvla_attention_prompt": (_I, [_P, _P, _P, _I, _I, _I, _I, _L, _L, _L, _I, _P, _I, _P, _I, _F, _I, _P, _P]),
    "qvla_kv4_pool_bytes": (_S, [_I, _I, _I, _I]),
    "qvla_kv4_append": (_I, [_P, _P, _P, _I, _L, _L, _I, _P, _I, _P, _I, _P, _P]),
    "qvla_kv4_gather": (_I, [_P, _I, _P, _I, _P, _I, _P, _P, _P, _I, _P]),
    "qvla_attention_kv4_workspace_bytes": (_S, [_I, _I, _I, _I, _I, _I, _I]),
    "qvla_attention_kv4": (_I, [_P, _P, _I, _I, _L, _I, _P, _I, _I, _P, _I, _P, _I, _F, _I, _P, _P, _S, _P]),
    "qvla_fp4_scale_bytes": (_S, [_I, _I, _I]),
    "qvla_fp4_quantize_rows": (_I, [_P, _I, _L, _I, _I, _I, _I, _P, _P, _P, _P, _P]),
    "qvla_fp4_dequantize_rows": (_I, [_P, _P, _P, _I, _I, _I, _P, _I, _P]),
    "qvla_fp4_pack_weights_host": (_I, [_P, _I, _I, _I, _P, _I, _P, _I, _I, _P, _P, _P]),
    "qvla_fp4_layer_create": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, ctypes.POINTER(_P)]),
    "qvla_fp4_layer_create_gated": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, ctypes.POINTER(_P)]),
    "qvla_fp4_layer_destroy": (_I, [_P]),
    "qvla_gemm_fp4": (_I, [_P, _P, _P, _P, _I, _P, _P]),
    "qvla_fp4_linear_workspace_bytes": (_S, [_P, _I]),
    "qvla_fp4_linear": (_I, [_P, _P, _I, _P, _P, _P, _S, _P]),
    "qvla_block_norm": (_I, [_P, _I, _P, _I, _L, _P, _L, _I, _I, _P, _P, _P]),
    "qvla_block_norm_fp4": (_I, [_P, _I, _P, _I, _L, _P, _L, _I, _I, _P, _P, _I, _I, _P, _P, _P, _P, _P]),
    "qvla_debug_gemm_plan_codes": (_I, [_I, _I, _I, _I, _I, _I, _I, _P, _P]),
}


class QvlaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


def load_library(path: str = _LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"libqvla.so is not built ({path}); run __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = load_library()

try:
    from . import _calls  # (linked against libqvla.so, whose absence is reported above)
except ImportError as error:  # built without CPython's headers, say: reported by the calls that it has
    _calls, _no_calls = None, str(error)


def lib() -> ctypes.CDLL:
    return _lib


def _check(status: int) -> None:
    if status != 0:
        raise QvlaError(status, _lib.qvla_last_error().decode())


def _ptr(t) -> int | None:
    """Raw address of a torch tensor / numpy array (None passes NULL)."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        return None
    return stream if isinstance(stream, int) else stream.cuda_stream


def qvla_abi_version() -> int:
    return _lib.qvla_abi_version()


def qvla_pack_weights_host(W: np.ndarray, wdt: int, N: int, K: int, rot=None, rot_block: int = 0, perm=None,
                           had_block: int = 1, wq=None, wscale=None, wsum=None) -> None:
    """Host-only fold + quantise + pack into caller-provided numpy buffers."""
    _check(_lib.qvla_pack_weights_host(_ptr(W), wdt, N, K, _ptr(rot), rot_block, _ptr(perm), had_block,
                                       _ptr(wq), _ptr(wscale), _ptr(wsum)))


def qvla_gptq_pack_host(W: np.ndarray, wdt: int, N: int, K: int, X: np.ndarray, xdt: int, n_cal: int, rot=None,
                        rot_block: int = 0, perm=None, had_block: int = 1, block: int = 128, damp: float = 0.01,
                        wq=None, wscale=None, wsum=None) -> None:
    """Host-only fold + GPTQ codes against calibration rows X + pack into caller-provided buffers."""
    _check(_lib.qvla_gptq_pack_host(_ptr(W), wdt, N, K, _ptr(X), xdt, n_cal, _ptr(rot), rot_block, _ptr(perm),
                                    had_block, block, float(damp), _ptr(wq), _ptr(wscale), _ptr(wsum)))


def qvla_block_svd_rotation(W: np.ndarray, wdt: int, N: int, K: int, block: int):
    """The zigzag permutation and block SVD factors chosen from the weights; returns
    (perm int32 [K], rot float64 [K/block, block, block])."""
    perm = np.empty(max(K, 1), dtype=np.int32)
    ok = block > 0 and K > 0 and K % block == 0
    rot = np.empty((K // block, block, block) if ok else (1,), dtype=np.float64)  # the library rejects bad shapes
    _check(_lib.qvla_block_svd_rotation(_ptr(np.ascontiguousarray(W)), wdt, N, K, block, _ptr(perm), _ptr(rot)))
    return perm, rot


class Layer:
    """Owner of a qvla_layer handle; ``close()`` (or garbage collection) destroys it."""

    def __init__(self, handle: int, N: int, K: int, had_block: int, xdt: int, ydt: int, gated: bool = False):
        self.handle, self.N, self.K, self.had_block, self.xdt, self.ydt = handle, N, K, had_block, xdt, ydt
        self.gated = gated  # N is the output width (H); the weight rows are 2H

    def close(self) -> None:
        if self.handle:
            _check(_lib.qvla_layer_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def qvla_layer_create(N: int, K: int, had_block: int, xdt: int, ydt: int, wq: np.ndarray, wscale: np.ndarray,
                      bias=None) -> Layer:
    h = ctypes.c_void_p()
    _check(_lib.qvla_layer_create(N, K, had_block, xdt, ydt, _ptr(wq), _ptr(wscale), _ptr(bias), ctypes.byref(h)))
    return Layer(h.value, N, K, had_block, xdt, ydt)


def qvla_layer_create_gated(H: int, K: int, had_block: int, xdt: int, ydt: int, wq_gate: np.ndarray,
                            wscale_gate: np.ndarray, wq_up: np.ndarray, wscale_up: np.ndarray, bias_gate=None,
                            bias_up=None) -> Layer:
    """Gate + up projections of a gated MLP as one layer whose output is h = gelu(gate) * up."""
    h = ctypes.c_void_p()
    _check(_lib.qvla_layer_create_gated(H, K, had_block, xdt, ydt, _ptr(wq_gate), _ptr(wscale_gate), _ptr(wq_up),
                                        _ptr(wscale_up), _ptr(bias_gate), _ptr(bias_up), ctypes.byref(h)))
    return Layer(h.value, H, K, had_block, xdt, ydt, gated=True)


def qvla_pack_weights(W: np.ndarray, wdt: int, N: int, K: int, rot=None, rot_block: int = 0, perm=None,
                      had_block: int = 1, bias=None, xdt: int = F16, ydt: int = F16) -> Layer:
    h = ctypes.c_void_p()
    _check(_lib.qvla_pack_weights(_ptr(W), wdt, N, K, _ptr(rot), rot_block, _ptr(perm), had_block, _ptr(bias),
                                  xdt, ydt, ctypes.byref(h)))
    return Layer(h.value, N, K, had_block, xdt, ydt)


def qvla_layer_destroy(layer: Layer) -> None:
    layer.close()


def qvla_set_step_scales(layer: Layer, scales: np.ndarray) -> None:
    scales = np.ascontiguousarray(scales, dtype=np.float32)
    _check(_lib.qvla_set_step_scales(layer.handle, _ptr(scales), int(scales.shape[0])))


def qvla_set_step_group_scales(layer: Layer, scales: np.ndarray) -> None:
    """Per-step, per-group table [T, G] (float32)."""
    arr = np.ascontiguousarray(scales, dtype=np.float32)
    if arr.ndim != 2:
        raise ValueError("scales must be [T, G]")
    _check(_lib.qvla_set_step_group_scales(layer.handle, _ptr(arr), arr.shape[0], arr.shape[1]))


def qvla_layer_set_online_rotation(layer: Layer, perm=None, rot=None, rot_block: int = 0) -> None:
    """Online x . P . BlockDiag(U_b) ahead of the layer's quantiser (perm int32 [K], rot float64
    [K/rot_block, rot_block, rot_block]); both None removes it."""
    p = None if perm is None else np.ascontiguousarray(perm, dtype=np.int32)
    r = None if rot is None else np.ascontiguousarray(rot, dtype=np.float64)
    _check(_lib.qvla_layer_set_online_rotation(layer.handle, _ptr(p), _ptr(r), int(rot_block)))


def qvla_online_rotate(layer: Layer, x, M: int, out, stream=None) -> None:
    _check(_lib.qvla_online_rotate(layer.handle, _ptr(x), M, _ptr(out), _stream(stream)))


def qvla_layer_scale_groups(layer: Layer):
    g, size = ctypes.c_int(), ctypes.c_int()
    _check(_lib.qvla_layer_scale_groups(layer.handle, ctypes.byref(g), ctypes.byref(size)))
    return g.value, size.value


def qvla_rotated_absmax_groups(x, xdt: int, M: int, K: int, had_block: int, absmax, stream=None) -> None:
    _check(_lib.qvla_rotated_absmax_groups(_ptr(x), xdt, M, K, had_block, _ptr(absmax), _stream(stream)))


def qvla_layer_info(layer: Layer):
    n, k, b, t = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(_lib.qvla_layer_info(layer.handle, ctypes.byref(n), ctypes.byref(k), ctypes.byref(b), ctypes.byref(t)))
    return n.value, k.value, b.value, t.value


def qvla_rotate_quantize(layer: Layer, x, M: int, step: int, xq, xscale, xsum=None, stream=None) -> None:
    _check(_lib.qvla_rotate_quantize(layer.handle, _ptr(x), M, step, _ptr(xq), _ptr(xscale), _ptr(xsum),
                                     _stream(stream)))


def qvla_rotate_quantize_rows(x, xdt: int, M: int, K: int, had_block: int, step_scale, xq, xscale, xsum=None,
                              stream=None) -> None:
    _check(_lib.qvla_rotate_quantize_rows(_ptr(x), xdt, M, K, had_block, _ptr(step_scale), _ptr(xq), _ptr(xscale),
                                          _ptr(xsum), _stream(stream)))


def qvla_rotated_absmax(x, xdt: int, M: int, K: int, had_block: int, absmax, stream=None) -> None:
    _check(_lib.qvla_rotated_absmax(_ptr(x), xdt, M, K, had_block, _ptr(absmax), _stream(stream)))


def qvla_gemm_w4a4(layer: Layer, xq, xscale, xsum, M: int, y, acc=None, stream=None) -> None:
    _check(_lib.qvla_gemm_w4a4(layer.handle, _ptr(xq), _ptr(xscale), _ptr(xsum), M, _ptr(y), _ptr(acc),
                               _stream(stream)))


def qvla_linear_workspace_bytes(layer: Layer, M: int) -> int:
    return int(_lib.qvla_linear_workspace_bytes(layer.handle, M))


def qvla_w4a4_linear(layer: Layer, x, M: int, step: int, y, workspace, workspace_bytes: int, stream=None) -> None:
    _check(_lib.qvla_w4a4_linear(layer.handle, _ptr(x), M, step, _ptr(y), _ptr(workspace), workspace_bytes,
                                 _stream(stream)))


def qvla_linear_quantize(layer: Layer, x, M: int, step: int, workspace, workspace_bytes: int, stream=None) -> None:
    _check(_lib.qvla_linear_quantize(layer.handle, _ptr(x), M, step, _ptr(workspace), workspace_bytes,
                                     _stream(stream)))


def qvla_linear_gemm(layer: Layer, workspace, workspace_bytes: int, M: int, y, stream=None) -> None:
    _check(_lib.qvla_linear_gemm(layer.handle, _ptr(workspace), workspace_bytes, M, _ptr(y), _stream(stream)))


NOALLOC_SCRATCH_BYTES = 8 << 20


def qvla_w4a4_linear_fused(layer: Layer, x, M: int, step: int, y, stream=None) -> None:
    """The one-launch linear (small batch, per-step scale); QvlaError status 2 where it does not apply."""
    _check(_lib.qvla_w4a4_linear_fused(layer.handle, _ptr(x), M, step, _ptr(y), _stream(stream)))


def qvla_w4a4_linear_noalloc(layer: Layer, x, M: int, step: int, y, stream=None) -> None:
    """qvla_w4a4_linear without a caller workspace: for callers that cannot allocate device
    memory while running; the library's fixed 8 MiB scratch takes the workspace's place."""
    _check(_lib.qvla_w4a4_linear_noalloc(layer.handle, _ptr(x), M, step, _ptr(y), _stream(stream)))


def qvla_rotate_quantize_rows_a8(x, xdt: int, M: int, K: int, had_block: int, step_scale, xq, xscale, xsum=None,
                                 stream=None) -> None:
    _check(_lib.qvla_rotate_quantize_rows_a8(_ptr(x), xdt, M, K, had_block, _ptr(step_scale), _ptr(xq),
                                             _ptr(xscale), _ptr(xsum), _stream(stream)))


def qvla_w4a8_workspace_bytes(layer: Layer, M: int) -> int:
    return int(_lib.qvla_w4a8_workspace_bytes(layer.handle, M))


def qvla_w4a8_linear(layer: Layer, x, M: int, step: int, y, workspace, workspace_bytes: int, stream=None) -> None:
    _check(_lib.qvla_w4a8_linear(layer.handle, _ptr(x), M, step, _ptr(y), _ptr(workspace), workspace_bytes,
                                 _stream(stream)))


def qvla_gemm_w4a8(layer: Layer, xq, xscale, M: int, y, acc, workspace, workspace_bytes: int, stream=None) -> None:
    _check(_lib.qvla_gemm_w4a8(layer.handle, _ptr(xq), _ptr(xscale), M, _ptr(y), _ptr(acc), _ptr(workspace),
                               workspace_bytes, _stream(stream)))


# The attention calls are short (a decoded token's takes a few microseconds): their wrappers take tensors only and call the
# library without the helpers above.

def qvla_attention_prompt(q, k, v, dt: int, heads: int, kv_heads: int, head_dim: int, q_stride: int, k_stride: int,
                          v_stride: int, batch: int, cu_q, total_q: int, cu_k, total_k: int, scale: float, causal: bool,
                          o, stream=None) -> None:
    """Softmax attention over packed prompts; strides in elements between tokens."""
    status = _lib.qvla_attention_prompt(q.data_ptr(), k.data_ptr(), v.data_ptr(), dt, heads, kv_heads, head_dim, q_stride,
                                        k_stride, v_stride, batch, cu_q.data_ptr(), total_q, cu_k.data_ptr(), total_k, scale,
                                        1 if causal else 0, o.data_ptr(), _stream(stream))
    if status:
        _check(status)


class _Kv4Struct(ctypes.Structure):
    _fields_ = [("pool", _P), ("num_pages", _I), ("page_size", _I), ("kv_heads", _I), ("head_dim", _I), ("rotate", _I)]


class Kv4Cache:
    """A 4-bit key/value cache (qvla_kv4_cache) over `pool`, a device buffer of qvla_kv4_pool_bytes(...) bytes that the
    caller owns and this object keeps alive."""

    __slots__ = ("pool", "struct", "ref")

    def __init__(self, pool, num_pages: int, page_size: int, kv_heads: int, head_dim: int, rotate: bool = True):
        if pool.nbytes < num_pages * page_size * kv_heads * (head_dim + 8):
            raise ValueError("the pool is smaller than qvla_kv4_pool_bytes(...)")
        self.pool = pool
        self.struct = _Kv4Struct(pool.data_ptr(), num_pages, page_size, kv_heads, head_dim, 1 if rotate else 0)
        self.ref = ctypes.addressof(self.struct)


def qvla_kv4_pool_bytes(num_pages: int, page_size: int, kv_heads: int, head_dim: int) -> int:
    return int(_lib.qvla_kv4_pool_bytes(num_pages, page_size, kv_heads, head_dim))


def qvla_kv4_append(cache: Kv4Cache, k, v, dt: int, k_stride: int, v_stride: int, batch: int, cu_new, total_new: int,
                    page_table, max_pages: int, start, stream=None) -> None:
    """Quantise new tokens into the cache; start None: every sequence begins at position 0."""
    status = _lib.qvla_kv4_append(cache.ref, k.data_ptr(), v.data_ptr(), dt, k_stride, v_stride, batch, cu_new.data_ptr(),
                                  total_new, page_table.data_ptr(), max_pages, None if start is None else start.data_ptr(),
                                  _stream(stream))
    if status:
        _check(status)


def qvla_kv4_gather(cache: Kv4Cache, batch: int, cu, total: int, page_table, max_pages: int, start, k, v, dt: int,
                    stream=None) -> None:
    """Read cached tokens back as values; start None: from position 0."""
    status = _lib.qvla_kv4_gather(cache.ref, batch, cu.data_ptr(), total, page_table.data_ptr(), max_pages,
                                  None if start is None else start.data_ptr(), k.data_ptr(), v.data_ptr(), dt, _stream(stream))
    if status:
        _check(status)


def qvla_attention_kv4_workspace_bytes(heads: int, kv_heads: int, head_dim: int, batch: int, total_q: int, max_q: int,
                                       max_len: int) -> int:
    return int(_lib.qvla_attention_kv4_workspace_bytes(heads, kv_heads, head_dim, batch, total_q, max_q, max_len))


def qvla_attention_kv4(cache: Kv4Cache, q, dt: int, heads: int, q_stride: int, batch: int, cu_q, total_q: int, max_q: int,
                       page_table, max_pages: int, kv_len, max_len: int, scale: float, causal: bool, o, workspace=None,
                       workspace_bytes: int = 0, stream=None) -> None:
    """Attention of a few query tokens of every sequence over its cached tokens."""
    status = _lib.qvla_attention_kv4(cache.ref, q.data_ptr(), dt, heads, q_stride, batch, cu_q.data_ptr(), total_q, max_q,
                                     page_table.data_ptr(), max_pages, kv_len.data_ptr(), max_len, scale, 1 if causal else 0,
                                     o.data_ptr(), None if workspace is None else workspace.data_ptr(), workspace_bytes,
                                     _stream(stream))
    if status:
        _check(status)


# 4-bit floating point and the norms around a block.  The calls of a step come compiled (csrc/calls.c), as they cost no more than
# their launch otherwise: what is optional is None or a tensor, a stream None, an address or a torch stream.
def _compiled(name: str):
    if _calls is not None:
        return getattr(_calls, name)

    def call(*args, **kwargs):
        raise ImportError(f"{name}() is a compiled call, and _calls cannot be imported ({_no_calls}): run __graft_entry__.build() with CPython's headers")

    call.__name__ = name
    return call


qvla_fp4_quantize_rows = _compiled("qvla_fp4_quantize_rows")
qvla_fp4_dequantize_rows = _compiled("qvla_fp4_dequantize_rows")
qvla_gemm_fp4 = _compiled("qvla_gemm_fp4")
qvla_fp4_linear = _compiled("qvla_fp4_linear")
qvla_block_norm = _compiled("qvla_block_norm")
qvla_block_norm_fp4 = _compiled("qvla_block_norm_fp4")


def qvla_fp4_scale_bytes(fmt: int, rows: int, K: int) -> int:
    return int(_lib.qvla_fp4_scale_bytes(fmt, rows, K))


def qvla_fp4_pack_weights_host(W: np.ndarray, wdt: int, N: int, K: int, rot=None, rot_block: int = 0, perm=None,
                               had_block: int = 1, fmt: int = NVFP4, wq=None, ws=None, wscale=None) -> None:
    """Host-only fold + quantise + pack into caller-provided numpy buffers."""
    _check(_lib.qvla_fp4_pack_weights_host(_ptr(W), wdt, N, K, _ptr(rot), rot_block, _ptr(perm), had_block, fmt, _ptr(wq), _ptr(ws),
                                           _ptr(wscale)))


class Fp4Layer:
    """Owner of a qvla_fp4_layer handle; ``close()`` (or garbage collection) destroys it."""

    def __init__(self, handle: int, N: int, K: int, had_block: int, fmt: int, xdt: int, ydt: int, gated: bool):
        self.handle, self.N, self.K, self.had_block, self.fmt, self.xdt, self.ydt = handle, N, K, had_block, fmt, xdt, ydt
        self.gated = gated  # N is the output width (H); the weight rows are 2H

    def close(self) -> None:
        if self.handle:
            _check(_lib.qvla_fp4_layer_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _fp4_layer(create, N, K, had_block, fmt, xdt, ydt, wq, ws, wscale, bias, gated):
    h = ctypes.c_void_p()
    _check(create(N, K, had_block, fmt, xdt, ydt, _ptr(wq), _ptr(ws), _ptr(wscale), _ptr(bias), ctypes.byref(h)))
    return Fp4Layer(h.value, N, K, had_block, fmt, xdt, ydt, gated)


def qvla_fp4_layer_create(N: int, K: int, had_block: int, fmt: int, xdt: int, ydt: int, wq: np.ndarray, ws: np.ndarray,
                          wscale=None, bias=None) -> Fp4Layer:
    return _fp4_layer(_lib.qvla_fp4_layer_create, N, K, had_block, fmt, xdt, ydt, wq, ws, wscale, bias, False)


def qvla_fp4_layer_create_gated(H: int, K: int, had_block: int, fmt: int, xdt: int, ydt: int, wq: np.ndarray, ws: np.ndarray,
                                wscale=None, bias=None) -> Fp4Layer:
    """Gate + up projections as one layer (arrays of H gate rows, then H up rows) whose output is gelu(gate) * up."""
    return _fp4_layer(_lib.qvla_fp4_layer_create_gated, H, K, had_block, fmt, xdt, ydt, wq, ws, wscale, bias, True)


def qvla_fp4_linear_workspace_bytes(layer: Fp4Layer, M: int) -> int:
    return int(_lib.qvla_fp4_linear_workspace_bytes(layer.handle, M))


class _NormStruct(ctypes.Structure):
    _fields_ = [("kind", _I), ("eps", _F), ("weight_offset", _F), ("residual_scale", _F), ("post_norm", _I),
                ("post_weight", _P), ("pre_weight", _P), ("pre_bias", _P), ("gate", _P), ("scale", _P), ("shift", _P),
                ("mod_stride", _L), ("mod_rows", _I), ("mod_tokens", _I), ("mod_index", _P)]


_NORM_DTYPES = {"torch.float16": F16, "torch.bfloat16": BF16}


class BlockNorm:
    """The norms, gate and modulation of one place between two blocks (qvla_block_norm_params), of type dt.  gate, scale and
    shift are 2-D tensors of the same rows and row stride (slices of one conditioning output, say) or None; token m takes row
    m // mod_tokens, or mod_index[m] (int32).  The tensors are kept alive and read at each call, whose K and M may not exceed
    ``width`` and ``tokens``, the channels and the indices that there are."""

    __slots__ = ("dt", "tensors", "struct", "ref", "width", "tokens")

    def __init__(self, kind: int, dt: int, eps: float = 1e-6, weight_offset: float = 0.0, residual_scale: float = 1.0,
                 post_norm: bool = False, post_weight=None, pre_weight=None, pre_bias=None, gate=None, scale=None, shift=None,
                 mod_tokens: int = 0, mod_index=None):
        mods = [t for t in (gate, scale, shift) if t is not None]
        if any(t.dim() != 2 or t.stride(1) != 1 or t.shape != mods[0].shape or t.stride(0) != mods[0].stride(0) for t in mods):
            raise ValueError("gate, scale and shift must be 2-D with the same rows, row stride and contiguous channels")
        vectors = [t for t in (post_weight, pre_weight, pre_bias) if t is not None]
        if any(t.dim() != 1 or not t.is_contiguous() for t in vectors):
            raise ValueError("the weights and the bias must be 1-D and contiguous")
        if any(_NORM_DTYPES.get(str(t.dtype)) != dt for t in vectors + mods):
            raise ValueError("weights, bias, gate, scale and shift must have the norm's type")
        if mod_index is not None and (mod_index.dim() != 1 or not mod_index.is_contiguous() or str(mod_index.dtype) != "torch.int32"):
            raise ValueError("mod_index must be 1-D, contiguous and int32")
        self.dt = dt
        self.width = min((t.shape[-1] for t in vectors + mods), default=(1 << 31) - 1)
        self.tokens = (1 << 31) - 1 if mod_index is None else mod_index.shape[0]
        self.tensors = (post_weight, pre_weight, pre_bias, gate, scale, shift, mod_index)
        rows = mods[0].shape[0] if mods else 0
        stride = (mods[0].stride(0) if rows > 1 else max(mods[0].stride(0), mods[0].shape[1])) if mods else 0
        self.struct = _NormStruct(kind, eps, weight_offset, residual_scale, 1 if post_norm else 0, _ptr(post_weight), _ptr(pre_weight),
                                  _ptr(pre_bias), _ptr(gate), _ptr(scale), _ptr(shift), stride, rows, mod_tokens, _ptr(mod_index))
        self.ref = ctypes.addressof(self.struct)


if _calls is not None:
    _calls.setup(_check, Fp4Layer, BlockNorm)


def qvla_check_device(stream=None) -> None:
    _check(_lib.qvla_check_device(_stream(stream)))


def qvla_debug_set_hooks(wait_limit_ns: int = 0, hold_gemm_loads: bool = False) -> None:
    """Test hooks (include/qvla_debug.h): the device wait limit (0 = default) and whether GEMM
    load warps hold back every copy."""
    _check(_lib.qvla_debug_set_hooks(int(wait_limit_ns), 1 if hold_gemm_loads else 0))


GEMM_SHAPES = ("single 128x128", "single 128x256", "pair 256x128", "pair 256x256") + tuple(
    f"tmem {32 * i}x256" for i in range(1, 7))


def qvla_debug_gemm_plan(M: int, K: int, N: int, gated: bool = False, num_sms: int = 152,
                         split_room: bool = True) -> tuple[str, int]:
    """The launch plan of qvla_w4a4_linear's GEMM (include/qvla_debug.h): (kernel and tile shape, work units
    per tile) for M > 128 tokens of an M x K -> N layer (N weight rows, 2H when gated).  Host only."""
    shape, parts = ctypes.c_int(-1), ctypes.c_int(0)
    _check(_lib.qvla_debug_gemm_plan(M, K, N, 1 if gated else 0, num_sms, 1 if split_room else 0,
                                     ctypes.addressof(shape), ctypes.addressof(parts)))
    return GEMM_SHAPES[shape.value], parts.value


def qvla_debug_gemm_plan_codes(codes: int, M: int, K: int, N: int, gated: bool = False, num_sms: int = 152,
                               split_room: bool = True) -> tuple[str, int]:
    """The same for packed 4-bit codes (0), qvla_w4a4_linear's activations (1) or 8-bit codes (2)."""
    shape, parts = ctypes.c_int(-1), ctypes.c_int(0)
    _check(_lib.qvla_debug_gemm_plan_codes(codes, M, K, N, 1 if gated else 0, num_sms, 1 if split_room else 0,
                                           ctypes.addressof(shape), ctypes.addressof(parts)))
    return GEMM_SHAPES[shape.value], parts.value
