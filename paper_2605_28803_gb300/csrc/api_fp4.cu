// The 4-bit floating-point and norm entry points of the C ABI (include/qvla.h): argument validation, layer objects, dispatch.
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/qvla.h"
#include "api_status.h"
#include "fp4.cuh"
#include "kernels.h"
#include "pack.h"

using qvla::aligned16;
using qvla::fail;

struct qvla_fp4_layer {
  int N = 0, K = 0, had_block = 1;  // N = weight rows (2H when gated)
  int fmt = 0, xdt = 0, ydt = 0, gated = 0, device = 0;
  uint8_t* wq = nullptr;    // device [N][K/2]; a gated layer's rows in turns of 16 gate rows and their 16 up rows
  uint8_t* ws = nullptr;    // device, scale tiles of the rows in that order, rows up to a multiple of 256
  float* wscale = nullptr;  // device [N] (ones for MX)
  float* bias = nullptr;    // device [N] (zeros without one)
  alignas(qvla::kFp4MapBytes) uint8_t maps[qvla::kFp4Maps * qvla::kFp4MapBytes] = {};  // tensor maps of wq and ws
};

namespace {

int ilog2_exact(int v) {
  if (v < 1 || (v & (v - 1))) return -1;
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

size_t round256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

qvla_status check_fmt(qvla_fp4_format fmt) {
  if (fmt != QVLA_MXFP4 && fmt != QVLA_NVFP4) return fail(QVLA_ERR_INVALID_ARG, "format %d must be MXFP4 or NVFP4", static_cast<int>(fmt));
  return QVLA_OK;
}

qvla_status check_rows(int M) {
  if (M < 0 || M > (1 << 20)) return fail(QVLA_ERR_INVALID_ARG, "M=%d outside [0, 2^20]", M);
  return QVLA_OK;
}

qvla_status check_k(int K, int had_block) {
  if (K <= 0 || K % 128 != 0) return fail(QVLA_ERR_INVALID_ARG, "K=%d must be a positive multiple of 128", K);
  if (K > 16384) return fail(QVLA_ERR_UNSUPPORTED, "K=%d exceeds 16384", K);
  if (ilog2_exact(had_block) < 0) return fail(QVLA_ERR_INVALID_ARG, "had_block=%d is not a power of two", had_block);
  if (had_block > 4096) return fail(QVLA_ERR_UNSUPPORTED, "had_block=%d exceeds 4096", had_block);
  if (K % had_block != 0) return fail(QVLA_ERR_INVALID_ARG, "K=%d is not a multiple of had_block=%d", K, had_block);
  return QVLA_OK;
}

qvla_status check_n(int N) {
  if (N <= 0 || N % 16 != 0 || N > (1 << 20)) return fail(QVLA_ERR_INVALID_ARG, "N=%d must be a positive multiple of 16 up to 2^20", N);
  return QVLA_OK;
}

// A matrix of M rows: its address and the distance of its rows.  Optional ones may be NULL.
qvla_status check_matrix(const char* name, const void* p, int M, int64_t stride, int K, bool optional = false) {
  if (optional && !p) return QVLA_OK;
  if (stride % 8 != 0 || stride < K || stride > (int64_t{1} << 31))
    return fail(QVLA_ERR_INVALID_ARG, "%s: a row stride of %lld elements must be a multiple of 8, at least %d and at most 2^31", name,
                static_cast<long long>(stride), K);
  if (M > 0 && (!p || !aligned16(p))) return fail(QVLA_ERR_INVALID_ARG, "%s must be a 16-byte aligned device pointer", name);
  return QVLA_OK;
}

qvla_status check_codes(int M, qvla_fp4_format fmt, const void* q, const void* s, const void* row) {
  if (M > 0 && (!q || !aligned16(q) || !s || !aligned16(s)))
    return fail(QVLA_ERR_INVALID_ARG, "codes and block scales must be 16-byte aligned device pointers");
  if (M > 0 && fmt == QVLA_NVFP4 && !row) return fail(QVLA_ERR_INVALID_ARG, "NVFP4 needs the rows' scales");
  return QVLA_OK;
}

qvla_status check_step(qvla_fp4_format fmt, const float* step_scale) {
  if (fmt == QVLA_MXFP4 && step_scale) return fail(QVLA_ERR_INVALID_ARG, "MXFP4 has no row scale that a step's could replace");
  return QVLA_OK;
}

qvla_status check_layer(const qvla_fp4_layer* L) {
  if (!L) return fail(QVLA_ERR_INVALID_ARG, "layer must not be NULL");
  int dev = 0;
  QVLA_CUDA(cudaGetDevice(&dev), "cudaGetDevice");
  if (dev != L->device)
    return fail(QVLA_ERR_INVALID_ARG, "the current device is %d but the layer lives on device %d", dev, L->device);
  return QVLA_OK;
}

qvla_status current_sms(int* sms) {
  int device = 0;
  QVLA_CUDA(cudaGetDevice(&device), "cudaGetDevice");
  *sms = qvla::num_sms(device);
  return QVLA_OK;
}

void set_quantizer(qvla::RowsArgs* a, int had_block, qvla_fp4_format fmt, const float* step_scale, uint8_t* xq, uint8_t* xs, float* xscale) {
  a->log_b = ilog2_exact(had_block);
  a->inv_sqrt_b = static_cast<float>(1.0 / std::sqrt(static_cast<double>(had_block)));
  a->fmt = static_cast<int>(fmt);
  a->step_scale = step_scale;
  a->codes = xq;
  a->scales = xs;
  a->row_scale = xscale;
}

qvla_status quantize(const void* x, int xdt, int64_t x_stride, int M, int K, int had_block, qvla_fp4_format fmt,
                     const float* step_scale, uint8_t* xq, uint8_t* xs, float* xscale, void* stream) {
  qvla::RowsArgs a = {};
  a.x = x;
  a.x_stride = x_stride;
  a.M = M;
  a.K = K;
  set_quantizer(&a, had_block, fmt, step_scale, xq, xs, xscale);
  a.stream = static_cast<cudaStream_t>(stream);
  if (qvla_status s = current_sms(&a.num_sms)) return s;
  QVLA_CUDA(xdt == QVLA_F16    ? qvla::launch_fp4_quantize_f16(a)
            : xdt == QVLA_BF16 ? qvla::launch_fp4_quantize_bf16(a)
                               : qvla::launch_fp4_quantize_f32(a),
            "fp4_quantize launch");
  return QVLA_OK;
}

qvla::Fp4GemmArgs product_args(const qvla_fp4_layer* L, const uint8_t* xq, const uint8_t* xs, const float* xscale, int M, void* y, void* stream) {
  return {xq, xs, L->fmt == QVLA_NVFP4 ? xscale : nullptr, L->wq, L->ws, L->maps, L->wscale, L->bias, L->fmt, L->ydt, L->gated,
          M, L->N, L->K, y, qvla::num_sms(L->device), static_cast<cudaStream_t>(stream)};
}

qvla_status multiply(const qvla_fp4_layer* L, const uint8_t* xq, const uint8_t* xs, const float* xscale, int M, void* y, void* stream) {
  const qvla::Fp4GemmArgs a = product_args(L, xq, xs, xscale, M, y, stream);
  QVLA_CUDA(qvla::launch_fp4_gemm(a), "gemm_fp4 launch");
  return QVLA_OK;
}

// The place in the device's order of weight row n as the caller gives it.
int device_row(int n, int N, int gated) {
  if (!gated) return n;
  const int h = N / 2, unit = n % h;
  return unit / 16 * 32 + (n >= h ? 16 : 0) + unit % 16;
}

qvla_status create(int N, int K, int had_block, qvla_fp4_format fmt, qvla_dtype xdt, qvla_dtype ydt, const uint8_t* wq, const uint8_t* ws,
                   const float* wscale, const float* bias, int gated, qvla_fp4_layer** out) {
  if (qvla_status s = check_fmt(fmt)) return s;
  if (qvla_status s = check_k(K, had_block)) return s;
  if (!wq || !ws || !out) return fail(QVLA_ERR_INVALID_ARG, "wq, ws and out must not be NULL");
  if ((fmt == QVLA_NVFP4) != (wscale != nullptr)) return fail(QVLA_ERR_INVALID_ARG, "wscale is for NVFP4, and NULL for MXFP4");
  if (xdt != QVLA_F16 && xdt != QVLA_BF16 && xdt != QVLA_F32) return fail(QVLA_ERR_INVALID_ARG, "bad activation dtype %d", static_cast<int>(xdt));
  if (ydt != QVLA_F16 && ydt != QVLA_BF16) return fail(QVLA_ERR_INVALID_ARG, "output dtype must be F16 or BF16");
  const int groups = K / (fmt == QVLA_MXFP4 ? 128 : 64);
  const size_t rb = static_cast<size_t>(K / 2), wbytes = static_cast<size_t>(N) * rb;
  const size_t sbytes = static_cast<size_t>((N + 255) / 256 * 2) * groups * 512;
  std::vector<uint8_t> codes, scales;
  std::vector<float> row, add;
  try {
    codes.resize(wbytes);
    scales.assign(sbytes, 0);
    row.assign(N, 1.0f);
    add.assign(N, 0.0f);
  } catch (const std::bad_alloc&) {
    return fail(QVLA_ERR_OOM, "host allocation failed");
  }
  const uint8_t worst = fmt == QVLA_MXFP4 ? 0xFE : 0x7E;  // the largest byte that is a number
  for (int n = 0; n < N; ++n) {
    const int d = device_row(n, N, gated);
    std::memcpy(codes.data() + d * rb, wq + n * rb, rb);
    for (int g = 0; g < groups; ++g) {
      const uint8_t* const from = ws + qvla::fp4::scale_offset(n, 4 * g, groups);
      for (int i = 0; i < 4; ++i)
        if (from[i] > worst) return fail(QVLA_ERR_INVALID_ARG, "the scale of row %d, block %d is not a non-negative number", n, 4 * g + i);
      std::memcpy(scales.data() + qvla::fp4::scale_offset(d, 4 * g, groups), from, 4);
    }
    if (wscale) {
      if (!(wscale[n] >= 0.0f) || std::isinf(wscale[n])) return fail(QVLA_ERR_INVALID_ARG, "wscale[%d] is not a finite non-negative float", n);
      row[d] = wscale[n];
    }
    if (bias) add[d] = bias[n];
  }
  auto* L = new (std::nothrow) qvla_fp4_layer();
  if (!L) return fail(QVLA_ERR_OOM, "host allocation failed");
  L->N = N;
  L->K = K;
  L->had_block = had_block;
  L->fmt = static_cast<int>(fmt);
  L->xdt = xdt;
  L->ydt = ydt;
  L->gated = gated;
  cudaError_t e = cudaGetDevice(&L->device);
  const size_t fbytes = static_cast<size_t>(N) * sizeof(float);
  if (e == cudaSuccess) e = cudaMalloc(&L->wq, wbytes);
  if (e == cudaSuccess) e = cudaMalloc(&L->ws, sbytes);
  if (e == cudaSuccess) e = cudaMalloc(&L->wscale, fbytes);
  if (e == cudaSuccess) e = cudaMalloc(&L->bias, fbytes);
  if (e == cudaSuccess) e = cudaMemcpy(L->wq, codes.data(), wbytes, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(L->ws, scales.data(), sbytes, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(L->wscale, row.data(), fbytes, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(L->bias, add.data(), fbytes, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = qvla::fp4_weight_maps(L->wq, L->ws, L->fmt, N, K, L->maps);
  if (e != cudaSuccess) {
    qvla_fp4_layer_destroy(L);
    return qvla::cuda_fail(e, "layer upload");
  }
  *out = L;
  return QVLA_OK;
}

qvla_status check_norm(const qvla_block_norm_params* n, qvla_dtype dt, const void* r, qvla_dtype rdt, int64_t r_stride, const void* y,
                       int64_t y_stride, int M, int K, void* r_out, void* h, bool quant, qvla::RowsArgs* a) {
  if (!n) return fail(QVLA_ERR_INVALID_ARG, "norm must not be NULL");
  if (n->kind != QVLA_NORM_RMS && n->kind != QVLA_NORM_LAYER) return fail(QVLA_ERR_INVALID_ARG, "norm kind %d", static_cast<int>(n->kind));
  if (!(n->eps > 0.0f) || std::isinf(n->eps)) return fail(QVLA_ERR_INVALID_ARG, "eps must be positive and finite");
  if (!std::isfinite(n->weight_offset) || !std::isfinite(n->residual_scale))
    return fail(QVLA_ERR_INVALID_ARG, "weight_offset and residual_scale must be finite");
  if (dt != QVLA_F16 && dt != QVLA_BF16) return fail(QVLA_ERR_INVALID_ARG, "dtype %d must be F16 or BF16", static_cast<int>(dt));
  if (rdt != dt && rdt != QVLA_F32) return fail(QVLA_ERR_INVALID_ARG, "the residual's dtype %d must be the branch's or F32", static_cast<int>(rdt));
  if (qvla_status s = check_rows(M)) return s;
  if (K <= 0 || K % 8 != 0) return fail(QVLA_ERR_INVALID_ARG, "K=%d must be a positive multiple of 8", K);
  if (K > 16384) return fail(QVLA_ERR_UNSUPPORTED, "K=%d exceeds 16384", K);
  if (qvla_status s = check_matrix("r", r, M, r_stride, K)) return s;
  if (qvla_status s = check_matrix("r_out", r_out, M, r_stride, K, true)) return s;
  if (qvla_status s = check_matrix("y", y, M, y_stride, K, true)) return s;
  if (h && !aligned16(h)) return fail(QVLA_ERR_INVALID_ARG, "h must be 16-byte aligned");
  if (h && h == y && y_stride != K && M > 1) return fail(QVLA_ERR_INVALID_ARG, "h is dense: it may be y only where y_stride is K=%d", K);
  if (!r_out && (y || n->residual_scale != 1.0f))
    return fail(QVLA_ERR_INVALID_ARG, "r_out may be NULL only without a branch and with residual_scale 1");
  if (!r_out && !h && !quant) return fail(QVLA_ERR_INVALID_ARG, "neither r_out nor h is given");
  if (!n->post_norm && n->post_weight) return fail(QVLA_ERR_INVALID_ARG, "post_weight without post_norm");
  for (const void* p : {n->post_weight, n->pre_weight, n->pre_bias, n->gate, n->scale, n->shift})
    if (p && !aligned16(p)) return fail(QVLA_ERR_INVALID_ARG, "weights, bias, gate, scale and shift must be 16-byte aligned");
  if (n->gate || n->scale || n->shift) {
    if (n->mod_stride % 8 != 0 || n->mod_stride < K) return fail(QVLA_ERR_INVALID_ARG, "mod_stride must be a multiple of 8 and at least K=%d", K);
    if (n->mod_rows < 1) return fail(QVLA_ERR_INVALID_ARG, "mod_rows=%d must be positive", n->mod_rows);
    if (!n->mod_index) {
      if (n->mod_tokens < 1) return fail(QVLA_ERR_INVALID_ARG, "mod_tokens=%d must be positive", n->mod_tokens);
      if (M > 0 && (M - 1) / n->mod_tokens >= n->mod_rows)
        return fail(QVLA_ERR_INVALID_ARG, "%d tokens by %d need more than %d rows", M, n->mod_tokens, n->mod_rows);
    }
  }
  a->x = r;
  a->xdt = static_cast<int>(rdt);
  a->dt = static_cast<int>(dt);
  a->x_stride = r_stride;
  a->M = M;
  a->K = K;
  a->norm = {n->kind == QVLA_NORM_LAYER, n->eps, n->weight_offset, n->residual_scale, n->post_norm, n->post_weight, n->pre_weight,
             n->pre_bias, n->gate, n->scale, n->shift, n->mod_stride, n->mod_rows, n->mod_tokens, n->mod_index};
  a->y = y;
  a->y_stride = y_stride;
  a->residual_out = r_out;
  a->h = h;
  return QVLA_OK;
}

qvla_status launch_norm(qvla::RowsArgs* a, void* stream) {
  a->stream = static_cast<cudaStream_t>(stream);
  if (qvla_status s = current_sms(&a->num_sms)) return s;
  QVLA_CUDA(a->dt == QVLA_F16 ? qvla::launch_norm_f16(*a) : qvla::launch_norm_bf16(*a), "block_norm launch");
  return QVLA_OK;
}

}  // namespace

extern "C" {

size_t qvla_fp4_scale_bytes(qvla_fp4_format fmt, int rows, int K) {
  if ((fmt != QVLA_MXFP4 && fmt != QVLA_NVFP4) || rows < 0 || rows > (1 << 20) || K <= 0 || K % 128 != 0 || K > 16384) return 0;
  return static_cast<size_t>((rows + 127) / 128) * (K / (fmt == QVLA_MXFP4 ? 128 : 64)) * 512;
}

qvla_status qvla_fp4_quantize_rows(const void* x, qvla_dtype xdt, int64_t x_stride, int M, int K, int had_block,
                                   qvla_fp4_format fmt, const float* step_scale, uint8_t* xq, uint8_t* xs, float* xscale,
                                   void* stream) {
  qvla::clear_error();
  if (xdt != QVLA_F16 && xdt != QVLA_BF16 && xdt != QVLA_F32) return fail(QVLA_ERR_INVALID_ARG, "bad dtype %d", static_cast<int>(xdt));
  if (qvla_status s = check_fmt(fmt)) return s;
  if (qvla_status s = check_rows(M)) return s;
  if (qvla_status s = check_k(K, had_block)) return s;
  if (qvla_status s = check_matrix("x", x, M, x_stride, K)) return s;
  if (qvla_status s = check_codes(M, fmt, xq, xs, xscale)) return s;
  if (qvla_status s = check_step(fmt, step_scale)) return s;
  if (M == 0) return QVLA_OK;
  return quantize(x, xdt, x_stride, M, K, had_block, fmt, step_scale, xq, xs, xscale, stream);
}

qvla_status qvla_fp4_dequantize_rows(const uint8_t* xq, const uint8_t* xs, const float* xscale, qvla_fp4_format fmt, int M, int K,
                                     void* out, qvla_dtype odt, void* stream) {
  qvla::clear_error();
  if (odt != QVLA_F16 && odt != QVLA_BF16 && odt != QVLA_F32) return fail(QVLA_ERR_INVALID_ARG, "bad dtype %d", static_cast<int>(odt));
  if (qvla_status s = check_fmt(fmt)) return s;
  if (qvla_status s = check_rows(M)) return s;
  if (qvla_status s = check_k(K, 1)) return s;
  if (qvla_status s = check_codes(M, fmt, xq, xs, xscale)) return s;
  if (M > 0 && (!out || !aligned16(out))) return fail(QVLA_ERR_INVALID_ARG, "out must be a 16-byte aligned device pointer");
  if (M == 0) return QVLA_OK;
  QVLA_CUDA(qvla::launch_fp4_dequantize(xq, xs, xscale, static_cast<int>(fmt), M, K, out, static_cast<int>(odt), static_cast<cudaStream_t>(stream)),
            "fp4_dequantize launch");
  return QVLA_OK;
}

qvla_status qvla_fp4_pack_weights_host(const void* W, qvla_dtype wdt, int N, int K, const double* rot, int rot_block,
                                       const int32_t* perm, int had_block, qvla_fp4_format fmt, uint8_t* wq, uint8_t* ws,
                                       float* wscale) {
  qvla::clear_error();
  if (qvla_status s = check_fmt(fmt)) return s;
  if (!W || !wq || !ws || (fmt == QVLA_NVFP4 && !wscale)) return fail(QVLA_ERR_INVALID_ARG, "W, wq, ws and (for NVFP4) wscale must not be NULL");
  if (wdt != QVLA_F16 && wdt != QVLA_BF16 && wdt != QVLA_F32) return fail(QVLA_ERR_INVALID_ARG, "bad weight dtype %d", static_cast<int>(wdt));
  if (qvla_status s = check_k(K, had_block)) return s;
  if (qvla_status s = check_n(N)) return s;
  if (rot && (rot_block <= 0 || K % rot_block != 0)) return fail(QVLA_ERR_INVALID_ARG, "rot_block=%d must divide K=%d", rot_block, K);
  try {
    if (perm) {
      std::vector<char> seen(K, 0);
      for (int k = 0; k < K; ++k) {
        if (perm[k] < 0 || perm[k] >= K || seen[perm[k]]) return fail(QVLA_ERR_INVALID_ARG, "perm is not a permutation of [0, K)");
        seen[perm[k]] = 1;
      }
    }
    if (!qvla::fp4_pack_weights_host_impl(W, static_cast<int>(wdt), N, K, rot, rot_block, perm, had_block, static_cast<int>(fmt), wq, ws, wscale))
      return fail(QVLA_ERR_INVALID_ARG, "a folded weight is not finite");
  } catch (const std::bad_alloc&) {
    return fail(QVLA_ERR_OOM, "host allocation failed");
  }
  return QVLA_OK;
}

qvla_status qvla_fp4_layer_create(int N, int K, int had_block, qvla_fp4_format fmt, qvla_dtype xdt, qvla_dtype ydt, const uint8_t* wq,
                                  const uint8_t* ws, const float* wscale, const float* bias, qvla_fp4_layer** out) {
  qvla::clear_error();
  if (qvla_status s = check_n(N)) return s;
  return create(N, K, had_block, fmt, xdt, ydt, wq, ws, wscale, bias, 0, out);
}

qvla_status qvla_fp4_layer_create_gated(int H, int K, int had_block, qvla_fp4_format fmt, qvla_dtype xdt, qvla_dtype ydt,
                                        const uint8_t* wq, const uint8_t* ws, const float* wscale, const float* bias,
                                        qvla_fp4_layer** out) {
  qvla::clear_error();
  if (H <= 0 || H % 128 != 0 || H > (1 << 19)) return fail(QVLA_ERR_INVALID_ARG, "H=%d must be a positive multiple of 128 up to 2^19", H);
  return create(2 * H, K, had_block, fmt, xdt, ydt, wq, ws, wscale, bias, 1, out);
}

qvla_status qvla_fp4_layer_destroy(qvla_fp4_layer* layer) {
  qvla::clear_error();
  if (!layer) return QVLA_OK;
  int dev = 0;
  const bool other = cudaGetDevice(&dev) == cudaSuccess && dev != layer->device;
  if (other) cudaSetDevice(layer->device);
  cudaDeviceSynchronize();
  cudaFree(layer->wq);
  cudaFree(layer->ws);
  cudaFree(layer->wscale);
  cudaFree(layer->bias);
  if (other) cudaSetDevice(dev);
  delete layer;
  return QVLA_OK;
}

qvla_status qvla_gemm_fp4(const qvla_fp4_layer* layer, const uint8_t* xq, const uint8_t* xs, const float* xscale, int M, void* y,
                          void* stream) {
  qvla::clear_error();
  if (!layer) return fail(QVLA_ERR_INVALID_ARG, "layer must not be NULL");
  if (qvla_status s = check_rows(M)) return s;
  if (qvla_status s = check_codes(M, static_cast<qvla_fp4_format>(layer->fmt), xq, xs, xscale)) return s;
  if (M > 0 && (!y || !aligned16(y))) return fail(QVLA_ERR_INVALID_ARG, "y must be a 16-byte aligned device pointer");
  if (M == 0) return QVLA_OK;
  if (qvla_status s = check_layer(layer)) return s;
  return multiply(layer, xq, xs, xscale, M, y, stream);
}

size_t qvla_fp4_linear_workspace_bytes(const qvla_fp4_layer* layer, int M) {
  if (!layer || M < 0 || M > (1 << 20)) return 0;
  return round256(static_cast<size_t>(M) * (layer->K / 2)) + round256(qvla_fp4_scale_bytes(static_cast<qvla_fp4_format>(layer->fmt), M, layer->K)) +
         round256(static_cast<size_t>(M) * sizeof(float));
}

qvla_status qvla_fp4_linear(const qvla_fp4_layer* layer, const void* x, int M, const float* step_scale, void* y, void* workspace,
                            size_t workspace_bytes, void* stream) {
  qvla::clear_error();
  if (!layer) return fail(QVLA_ERR_INVALID_ARG, "layer must not be NULL");
  const qvla_fp4_format fmt = static_cast<qvla_fp4_format>(layer->fmt);
  if (qvla_status s = check_rows(M)) return s;
  if (qvla_status s = check_matrix("x", x, M, layer->K, layer->K)) return s;
  if (qvla_status s = check_step(fmt, step_scale)) return s;
  if (M > 0 && (!y || !aligned16(y))) return fail(QVLA_ERR_INVALID_ARG, "y must be a 16-byte aligned device pointer");
  if (M > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))) return fail(QVLA_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  if (workspace_bytes < qvla_fp4_linear_workspace_bytes(layer, M))
    return fail(QVLA_ERR_INVALID_ARG, "the workspace has %zu bytes, the call needs %zu", workspace_bytes, qvla_fp4_linear_workspace_bytes(layer, M));
  if (M == 0) return QVLA_OK;
  if (qvla_status s = check_layer(layer)) return s;
  uint8_t* const xq = static_cast<uint8_t*>(workspace);
  uint8_t* const xs = xq + round256(static_cast<size_t>(M) * (layer->K / 2));
  float* const xscale = reinterpret_cast<float*>(xs + round256(qvla_fp4_scale_bytes(fmt, M, layer->K)));
  // In one launch a CTA may write y while others still read x.
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y);
  const uintptr_t x1 = x0 + static_cast<size_t>(M) * layer->K * 2, y1 = y0 + static_cast<size_t>(M) * (layer->gated ? layer->N / 2 : layer->N) * 2;
  if (layer->xdt == layer->ydt && (x1 <= y0 || y1 <= x0)) {
    bool taken = false;
    QVLA_CUDA(qvla::launch_fp4_token(product_args(layer, xq, xs, xscale, M, y, stream), x, ilog2_exact(layer->had_block),
                                     static_cast<float>(1.0 / std::sqrt(static_cast<double>(layer->had_block))), step_scale, &taken),
              "fp4_linear launch");
    if (taken) return QVLA_OK;
  }
  if (qvla_status s = quantize(x, layer->xdt, layer->K, M, layer->K, layer->had_block, fmt, step_scale, xq, xs, xscale, stream)) return s;
  return multiply(layer, xq, xs, xscale, M, y, stream);
}

qvla_status qvla_block_norm(const qvla_block_norm_params* norm, qvla_dtype dt, const void* r, qvla_dtype rdt, int64_t r_stride, const void* y,
                            int64_t y_stride, int M, int K, void* r_out, void* h, void* stream) {
  qvla::clear_error();
  qvla::RowsArgs a = {};
  if (qvla_status s = check_norm(norm, dt, r, rdt, r_stride, y, y_stride, M, K, r_out, h, false, &a)) return s;
  if (M == 0) return QVLA_OK;
  return launch_norm(&a, stream);
}

qvla_status qvla_block_norm_fp4(const qvla_block_norm_params* norm, qvla_dtype dt, const void* r, qvla_dtype rdt, int64_t r_stride,
                                const void* y, int64_t y_stride, int M, int K, void* r_out, void* h, int had_block,
                                qvla_fp4_format fmt, const float* step_scale, uint8_t* hq, uint8_t* hs, float* hscale, void* stream) {
  qvla::clear_error();
  qvla::RowsArgs a = {};
  if (qvla_status s = check_norm(norm, dt, r, rdt, r_stride, y, y_stride, M, K, r_out, h, true, &a)) return s;
  if (qvla_status s = check_fmt(fmt)) return s;
  if (qvla_status s = check_k(K, had_block)) return s;
  if (qvla_status s = check_codes(M, fmt, hq, hs, hscale)) return s;
  if (qvla_status s = check_step(fmt, step_scale)) return s;
  if (M == 0) return QVLA_OK;
  set_quantizer(&a, had_block, fmt, step_scale, hq, hs, hscale);
  return launch_norm(&a, stream);
}

}  // extern "C"
