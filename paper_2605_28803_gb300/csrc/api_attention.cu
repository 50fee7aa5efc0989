// The attention entry points of the C ABI (include/qvla.h): argument validation and dispatch.
#include <cuda_runtime.h>

#include <cmath>

#include "../../include/qvla.h"
#include "api_status.h"
#include "kernels.h"

using qvla::aligned16;
using qvla::fail;

namespace {

constexpr int kMaxTokens = 1 << 24;
constexpr int kMaxLength = 1 << 30;  // of a cached sequence
constexpr int kMaxHeads = 1024;
constexpr int64_t kMaxRows = 0x7fffffff - 16;  // query heads of a call (rows of its tiles are numbered in 32 bits, the last tile's past them)

qvla_status check_heads(qvla_dtype dt, int heads, int kv_heads, int head_dim) {
  if (dt != QVLA_F16 && dt != QVLA_BF16) return fail(QVLA_ERR_INVALID_ARG, "dtype %d must be F16 or BF16", static_cast<int>(dt));
  if (heads < 1 || heads > kMaxHeads || kv_heads < 1 || heads % kv_heads != 0)
    return fail(QVLA_ERR_INVALID_ARG, "heads=%d (1 to %d) must be a multiple of kv_heads=%d", heads, kMaxHeads, kv_heads);
  if (head_dim != 64 && head_dim != 128 && head_dim != 256)
    return fail(QVLA_ERR_UNSUPPORTED, "head_dim=%d must be 64, 128 or 256", head_dim);
  return QVLA_OK;
}

qvla_status check_tokens(const char* name, const void* p, int total, int64_t stride, int width) {
  if (total < 0 || total > kMaxTokens) return fail(QVLA_ERR_INVALID_ARG, "%s: %d tokens outside [0, 2^24]", name, total);
  if (stride % 8 != 0 || stride < width || stride > (int64_t{1} << 31))
    return fail(QVLA_ERR_INVALID_ARG, "%s: a token stride of %lld elements must be a multiple of 8, at least %d and at most 2^31",
                name, static_cast<long long>(stride), width);
  if (total > 0 && (!p || !aligned16(p))) return fail(QVLA_ERR_INVALID_ARG, "%s must be a 16-byte aligned device pointer", name);
  return QVLA_OK;
}

qvla_status check_scale(float scale) {
  if (!(scale > 0.0f) || std::isinf(scale)) return fail(QVLA_ERR_INVALID_ARG, "scale must be positive and finite");
  return QVLA_OK;
}

int log_page(int page_size) {
  for (int l = 4; l <= 8; ++l)
    if (page_size == 1 << l) return l;
  return -1;
}

// The cache's geometry; `heads` is the queries' (kv_heads itself for a call without queries).
qvla_status check_cache(const qvla_kv4_cache* c, qvla_dtype dt, int heads, qvla::Kv4Pool* pool) {
  if (!c) return fail(QVLA_ERR_INVALID_ARG, "cache must not be NULL");
  if (qvla_status s = check_heads(dt, heads < 0 ? c->kv_heads : heads, c->kv_heads, c->head_dim)) return s;
  const int lp = log_page(c->page_size);
  if (lp < 0) return fail(QVLA_ERR_INVALID_ARG, "page_size=%d must be 16, 32, 64, 128 or 256", c->page_size);
  if (c->num_pages < 1) return fail(QVLA_ERR_INVALID_ARG, "num_pages=%d must be positive", c->num_pages);
  if (!c->pool || !aligned16(c->pool)) return fail(QVLA_ERR_INVALID_ARG, "the pool must be a 16-byte aligned device pointer");
  *pool = {static_cast<uint8_t*>(c->pool), c->num_pages, lp, c->kv_heads, c->head_dim, c->rotate ? 1 : 0};
  return QVLA_OK;
}

qvla_status check_batch(int batch, const void* cu, const void* table, int max_pages) {
  if (batch < 0 || batch > 65535) return fail(QVLA_ERR_INVALID_ARG, "batch=%d outside [0, 65535]", batch);
  if (batch > 0 && (!cu || !table)) return fail(QVLA_ERR_INVALID_ARG, "offsets and page_table must not be NULL");
  if (max_pages < 1) return fail(QVLA_ERR_INVALID_ARG, "max_pages=%d must be positive", max_pages);
  return QVLA_OK;
}

// No sequence has more queries than the call.
int queries_at_most(int max_q, int total_q) { return max_q < total_q ? max_q : total_q; }

qvla_status current_sms(int* sms) {
  int device = 0;
  QVLA_CUDA(cudaGetDevice(&device), "cudaGetDevice");
  *sms = qvla::num_sms(device);
  return QVLA_OK;
}

}  // namespace

extern "C" {

qvla_status qvla_attention_prompt(const void* q, const void* k, const void* v, qvla_dtype dt, int heads, int kv_heads,
                                  int head_dim, int64_t q_stride, int64_t k_stride, int64_t v_stride, int batch,
                                  const int32_t* cu_q, int total_q, const int32_t* cu_k, int total_k, float scale,
                                  int causal, void* o, void* stream) {
  qvla::clear_error();
  if (qvla_status s = check_heads(dt, heads, kv_heads, head_dim)) return s;
  if (qvla_status s = check_tokens("q", q, total_q, q_stride, heads * head_dim)) return s;
  if (qvla_status s = check_tokens("k", k, total_k, k_stride, kv_heads * head_dim)) return s;
  if (qvla_status s = check_tokens("v", v, total_k, v_stride, kv_heads * head_dim)) return s;
  if (qvla_status s = check_tokens("o", o, total_q, heads * head_dim, heads * head_dim)) return s;
  if (batch < 0 || batch > 65535) return fail(QVLA_ERR_INVALID_ARG, "batch=%d outside [0, 65535]", batch);
  if (batch > 0 && (!cu_q || !cu_k)) return fail(QVLA_ERR_INVALID_ARG, "cu_q and cu_k must not be NULL");
  if (qvla_status s = check_scale(scale)) return s;
  if (batch == 0 || total_q == 0) return QVLA_OK;
  qvla::PromptArgs a = {q, k, v, static_cast<int>(dt), heads, kv_heads, head_dim, q_stride, k_stride, v_stride, batch,
                        cu_q, cu_k, total_q, total_k, scale, causal ? 1 : 0, o, 0, static_cast<cudaStream_t>(stream)};
  if (qvla_status s = current_sms(&a.num_sms)) return s;
  QVLA_CUDA(qvla::launch_attention_prompt(a), "attention_prompt launch");
  return QVLA_OK;
}

size_t qvla_kv4_pool_bytes(int num_pages, int page_size, int kv_heads, int head_dim) {
  if (num_pages < 1 || log_page(page_size) < 0 || kv_heads < 1 || kv_heads > kMaxHeads ||
      (head_dim != 64 && head_dim != 128 && head_dim != 256))
    return 0;
  return static_cast<size_t>(num_pages) * kv_heads * page_size * (head_dim + 8);
}

qvla_status qvla_kv4_append(const qvla_kv4_cache* cache, const void* k, const void* v, qvla_dtype dt, int64_t k_stride,
                            int64_t v_stride, int batch, const int32_t* cu_new, int total_new,
                            const int32_t* page_table, int max_pages, const int32_t* start, void* stream) {
  qvla::clear_error();
  qvla::Kv4Pool pool;
  if (qvla_status s = check_cache(cache, dt, -1, &pool)) return s;
  const int width = pool.kv_heads * pool.head_dim;
  if (qvla_status s = check_tokens("k", k, total_new, k_stride, width)) return s;
  if (qvla_status s = check_tokens("v", v, total_new, v_stride, width)) return s;
  if (qvla_status s = check_batch(batch, cu_new, page_table, max_pages)) return s;
  if (batch == 0 || total_new == 0) return QVLA_OK;
  qvla::Kv4RowsArgs a = {pool, const_cast<void*>(k), const_cast<void*>(v), k_stride, v_stride, static_cast<int>(dt), batch,
                         cu_new, total_new, page_table, max_pages, start, 0, static_cast<cudaStream_t>(stream)};
  if (qvla_status s = current_sms(&a.num_sms)) return s;
  QVLA_CUDA(qvla::launch_kv4_append(a), "kv4_append launch");
  return QVLA_OK;
}

qvla_status qvla_kv4_gather(const qvla_kv4_cache* cache, int batch, const int32_t* cu, int total,
                            const int32_t* page_table, int max_pages, const int32_t* start, void* k, void* v,
                            qvla_dtype dt, void* stream) {
  qvla::clear_error();
  qvla::Kv4Pool pool;
  if (qvla_status s = check_cache(cache, dt, -1, &pool)) return s;
  const int width = pool.kv_heads * pool.head_dim;
  if (qvla_status s = check_tokens("k", k, total, width, width)) return s;
  if (qvla_status s = check_tokens("v", v, total, width, width)) return s;
  if (qvla_status s = check_batch(batch, cu, page_table, max_pages)) return s;
  if (batch == 0 || total == 0) return QVLA_OK;
  qvla::Kv4RowsArgs a = {pool, k, v, width, width, static_cast<int>(dt), batch, cu, total, page_table, max_pages, start, 0,
                         static_cast<cudaStream_t>(stream)};
  if (qvla_status s = current_sms(&a.num_sms)) return s;
  QVLA_CUDA(qvla::launch_kv4_gather(a), "kv4_gather launch");
  return QVLA_OK;
}

size_t qvla_attention_kv4_workspace_bytes(int heads, int kv_heads, int head_dim, int batch, int total_q, int max_q,
                                          int max_len) {
  if (heads < 1 || heads > kMaxHeads || kv_heads < 1 || heads % kv_heads != 0 ||
      (head_dim != 64 && head_dim != 128 && head_dim != 256) || batch < 1 || batch > 65535 || total_q < 1 ||
      total_q > kMaxTokens || max_q < 1 || max_q > kMaxTokens || max_len < 1 || max_len > kMaxLength ||
      static_cast<int64_t>(total_q) * heads > kMaxRows)
    return 0;
  qvla::Kv4AttentionArgs a = {};
  a.pool.kv_heads = kv_heads;
  a.pool.head_dim = head_dim;
  a.heads = heads;
  a.batch = batch;
  a.total_q = total_q;
  a.max_q = queries_at_most(max_q, total_q);
  a.max_len = max_len;
  if (current_sms(&a.num_sms) != QVLA_OK) {
    qvla::clear_error();
    a.num_sms = 152;
  }
  return qvla::attention_kv4_workspace(a);
}

qvla_status qvla_attention_kv4(const qvla_kv4_cache* cache, const void* q, qvla_dtype dt, int heads, int64_t q_stride,
                               int batch, const int32_t* cu_q, int total_q, int max_q, const int32_t* page_table,
                               int max_pages, const int32_t* kv_len, int max_len, float scale, int causal, void* o,
                               void* workspace, size_t workspace_bytes, void* stream) {
  qvla::clear_error();
  qvla::Kv4Pool pool;
  if (qvla_status s = check_cache(cache, dt, heads, &pool)) return s;
  const int width = heads * pool.head_dim;
  if (qvla_status s = check_tokens("q", q, total_q, q_stride, width)) return s;
  if (qvla_status s = check_tokens("o", o, total_q, width, width)) return s;
  if (qvla_status s = check_batch(batch, cu_q, page_table, max_pages)) return s;
  if (batch > 0 && !kv_len) return fail(QVLA_ERR_INVALID_ARG, "kv_len must not be NULL");
  if (max_q < 0 || max_q > kMaxTokens || max_len < 0 || max_len > kMaxLength)
    return fail(QVLA_ERR_INVALID_ARG, "max_q=%d outside [0, 2^24] or max_len=%d outside [0, 2^30]", max_q, max_len);
  if (static_cast<int64_t>(max_len) > (static_cast<int64_t>(max_pages) << pool.log_page))
    return fail(QVLA_ERR_INVALID_ARG, "max_len=%d exceeds the %d pages of a sequence's table", max_len, max_pages);
  if (static_cast<int64_t>(total_q) * heads > kMaxRows)
    return fail(QVLA_ERR_UNSUPPORTED, "%d tokens of %d heads are more rows than 2^31 - 17", total_q, heads);
  if (qvla_status s = check_scale(scale)) return s;
  if (workspace_bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)))
    return fail(QVLA_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  if (batch == 0 || total_q == 0 || max_q == 0) return QVLA_OK;
  qvla::Kv4AttentionArgs a = {pool, q, static_cast<int>(dt), heads, q_stride, batch, cu_q, total_q, queries_at_most(max_q, total_q), page_table,
                              max_pages, kv_len, max_len, scale, causal ? 1 : 0, o, workspace, workspace_bytes, 0,
                              static_cast<cudaStream_t>(stream)};
  if (qvla_status s = current_sms(&a.num_sms)) return s;
  QVLA_CUDA(qvla::launch_attention_kv4(a), "attention_kv4 launch");
  return QVLA_OK;
}

}  // extern "C"
