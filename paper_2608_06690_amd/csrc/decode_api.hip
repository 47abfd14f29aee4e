// C ABI of a decoding step's operators (paged cache, attention over it, sampling): argument validation (host
// only, before any launch) and dispatch to the kernel launchers. No exception crosses this boundary; no device
// memory is allocated.
#include <cmath>

#include "pmpe_internal.h"

using namespace pmpe;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

pmpe_status launched(hipError_t e) { return e == hipSuccess ? PMPE_OK : PMPE_ERR_LAUNCH; }

constexpr int32_t kMaxHeads = 1024;

pmpe_status check_cache(const pmpe_cache_desc* c) {
  if (!c) return PMPE_ERR_NULL;
  if (c->act_dtype != PMPE_BF16 && c->act_dtype != PMPE_F32) return PMPE_ERR_DTYPE;
  if (c->cache_dtype != c->act_dtype && !(c->act_dtype == PMPE_BF16 && c->cache_dtype == PMPE_FP8_E4M3)) return PMPE_ERR_DTYPE;
  if (c->n_pages < 1 || c->max_pages < 1) return PMPE_ERR_SHAPE;
  if (c->page_size < 16 || c->page_size > 1024 || c->page_size % 16 != 0) return PMPE_ERR_SHAPE;
  if (c->head_dim < 32 || c->head_dim > 256 || c->head_dim % 32 != 0) return PMPE_ERR_SHAPE;
  if (c->n_kv_heads < 1 || c->n_kv_heads > kMaxHeads) return PMPE_ERR_SHAPE;
  if ((int64_t)c->n_kv_heads * c->page_size * c->head_dim >= ((int64_t)1 << 31)) return PMPE_ERR_SHAPE;
  if ((int64_t)c->max_pages * c->page_size >= ((int64_t)1 << 30)) return PMPE_ERR_SHAPE;
  return PMPE_OK;
}

// tokens that are `stride` elements of the activation type apart, each of `row` elements
pmpe_status check_stride(const pmpe_cache_desc* c, int64_t stride, int64_t row) {
  const int64_t el = c->act_dtype == PMPE_BF16 ? 2 : 4;
  if (stride < row || stride > ((int64_t)1 << 40)) return PMPE_ERR_SHAPE;
  return stride * el % 16 != 0 ? PMPE_ERR_ALIGN : PMPE_OK;
}

pmpe_status check_values(const pmpe_cache_desc* c, const int32_t* table, const void* k, const void* v, const uint8_t* ks,
                         const uint8_t* vs) {
  if (!table || !k || !v) return PMPE_ERR_NULL;
  if (c->cache_dtype == PMPE_FP8_E4M3 ? !ks || !vs : ks || vs) return PMPE_ERR_NULL;
  return aligned16(k) && aligned16(v) && aligned16(ks) && aligned16(vs) ? PMPE_OK : PMPE_ERR_ALIGN;
}

CacheArgs cache_args(const pmpe_cache_desc* c, int32_t R, const int32_t* table, const uint32_t* tag, const uint32_t* words,
                     const void* k, const void* v, const uint8_t* ks, const uint8_t* vs, uint32_t* dev_status) {
  return CacheArgs{R, c->n_pages, c->page_size, c->n_kv_heads, c->head_dim, c->max_pages, c->act_dtype == PMPE_BF16,
                   c->cache_dtype == PMPE_FP8_E4M3, table, tag, words, const_cast<void*>(k), const_cast<void*>(v),
                   const_cast<uint8_t*>(ks), const_cast<uint8_t*>(vs), dev_status};
}

pmpe_status check_batch(const pmpe_cache_desc* c, int32_t T, int32_t R) {
  const pmpe_status st = check_cache(c);
  if (st != PMPE_OK) return st;
  return T < 0 || T > PMPE_MAX_TOKENS || R < 0 || R > PMPE_MAX_REQUESTS ? PMPE_ERR_SHAPE : PMPE_OK;
}

}  // namespace

extern "C" {

pmpe_status pmpe_kv_write(const pmpe_cache_desc* c, int32_t T, int32_t R, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, const int32_t* req_offset,
                          const int32_t* seq_len, const int32_t* block_table, const uint32_t* page_tag,
                          const uint32_t* policy_word, void* k_cache, void* v_cache, uint8_t* k_scale,
                          uint8_t* v_scale, uint32_t* dev_status, pmpe_stream_t stream) {
  pmpe_status st = check_batch(c, T, R);
  if (st != PMPE_OK || T == 0 || R == 0) return st;
  if (!k || !v || !req_offset || !seq_len) return PMPE_ERR_NULL;
  st = check_values(c, block_table, k_cache, v_cache, k_scale, v_scale);
  const int64_t row = (int64_t)c->n_kv_heads * c->head_dim;
  if (st == PMPE_OK) st = check_stride(c, k_stride, row);
  if (st == PMPE_OK) st = check_stride(c, v_stride, row);
  if (st != PMPE_OK) return st;
  if (!aligned16(k) || !aligned16(v)) return PMPE_ERR_ALIGN;
  KvRowsArgs a{cache_args(c, R, block_table, page_tag, policy_word, k_cache, v_cache, k_scale, v_scale, dev_status), T,
               const_cast<void*>(k), const_cast<void*>(v), k_stride, v_stride, req_offset, seq_len};
  return launched(launch_kv_write(a, (hipStream_t)stream));
}

pmpe_status pmpe_kv_read(const pmpe_cache_desc* c, int32_t T, int32_t R, void* k, void* v,
                         const int32_t* req_offset, const int32_t* first, const int32_t* block_table,
                         const uint32_t* page_tag, const uint32_t* policy_word, const void* k_cache,
                         const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale,
                         uint32_t* dev_status, pmpe_stream_t stream) {
  pmpe_status st = check_batch(c, T, R);
  if (st != PMPE_OK || T == 0 || R == 0) return st;
  if (!k || !v || !req_offset) return PMPE_ERR_NULL;
  st = check_values(c, block_table, k_cache, v_cache, k_scale, v_scale);
  if (st != PMPE_OK) return st;
  if (!aligned16(k) || !aligned16(v)) return PMPE_ERR_ALIGN;
  const int64_t row = (int64_t)c->n_kv_heads * c->head_dim;
  KvRowsArgs a{cache_args(c, R, block_table, page_tag, policy_word, k_cache, v_cache, k_scale, v_scale, dev_status), T,
               k, v, row, row, req_offset, first};
  return launched(launch_kv_read(a, (hipStream_t)stream));
}

size_t pmpe_attn_decode_workspace_bytes(const pmpe_cache_desc* c, int32_t R, int32_t n_heads) {
  if (check_batch(c, 0, R) != PMPE_OK || n_heads < 1 || n_heads > kMaxHeads || n_heads % c->n_kv_heads != 0) return 0;
  return attn_decode_workspace(R, n_heads, c);
}

pmpe_status pmpe_attn_decode(const pmpe_cache_desc* c, int32_t R, int32_t n_heads, const void* q,
                             int64_t q_stride, const int32_t* seq_first, const int32_t* seq_len,
                             const int32_t* block_table, const uint32_t* page_tag,
                             const uint32_t* policy_word, const void* k_cache, const void* v_cache,
                             const uint8_t* k_scale, const uint8_t* v_scale, float scale, void* out,
                             float* lse, uint32_t* dev_status, void* ws, size_t ws_bytes,
                             pmpe_stream_t stream) {
  pmpe_status st = check_batch(c, 0, R);
  if (st != PMPE_OK) return st;
  if (n_heads < 1 || n_heads > kMaxHeads || n_heads % c->n_kv_heads != 0 || !std::isfinite(scale)) return PMPE_ERR_SHAPE;
  if (R == 0) return PMPE_OK;
  if (!q || !seq_len || !out) return PMPE_ERR_NULL;
  st = check_values(c, block_table, k_cache, v_cache, k_scale, v_scale);
  if (st == PMPE_OK) st = check_stride(c, q_stride, (int64_t)n_heads * c->head_dim);
  if (st != PMPE_OK) return st;
  if (!aligned16(q) || !aligned16(out)) return PMPE_ERR_ALIGN;
  const size_t need = attn_decode_workspace(R, n_heads, c);
  if (need > 0) {
    if (!ws || ws_bytes < need) return PMPE_ERR_WORKSPACE;
    if (!aligned16(ws)) return PMPE_ERR_ALIGN;
  }
  AttnArgs a{cache_args(c, R, block_table, page_tag, policy_word, k_cache, v_cache, k_scale, v_scale, dev_status), n_heads, q,
             q_stride, seq_first, seq_len, scale, out, lse, (float*)ws};
  return launched(launch_attn_decode(a, (hipStream_t)stream));
}

size_t pmpe_sample_workspace_bytes(int32_t B, int32_t V) {
  if (B < 1 || B > PMPE_MAX_REQUESTS || V < 1 || V > PMPE_MAX_VOCAB) return 0;
  return sample_workspace(B, V);
}

pmpe_status pmpe_sample(int32_t B, int32_t V, const void* logits, int32_t logits_dtype, int64_t stride,
                        const float* temperature, const int32_t* top_k, const float* top_p,
                        const float* min_p, const float* u, int32_t* token, float* prob, int32_t* kept,
                        void* ws, size_t ws_bytes, pmpe_stream_t stream) {
  if (B < 0 || B > PMPE_MAX_REQUESTS || V < 1 || V > PMPE_MAX_VOCAB) return PMPE_ERR_SHAPE;
  if (stride < V || stride > ((int64_t)1 << 40)) return PMPE_ERR_SHAPE;
  if (logits_dtype != PMPE_F32 && logits_dtype != PMPE_BF16) return PMPE_ERR_DTYPE;
  if (B == 0) return PMPE_OK;
  if (!logits || !u || !token) return PMPE_ERR_NULL;
  if (((uintptr_t)logits & (logits_dtype == PMPE_BF16 ? 1u : 3u)) != 0) return PMPE_ERR_ALIGN;
  const void* al[] = {temperature, top_k, top_p, min_p, u, token, prob, kept};
  for (const void* p : al)
    if (((uintptr_t)p & 3u) != 0) return PMPE_ERR_ALIGN;
  const size_t need = sample_workspace(B, V);
  if (need > 0) {
    if (!ws || ws_bytes < need) return PMPE_ERR_WORKSPACE;
    if (!aligned16(ws)) return PMPE_ERR_ALIGN;
  }
  SampleArgs a{B, V, logits_dtype == PMPE_BF16, logits, stride, temperature, top_k, top_p, min_p, u, token, prob, kept, ws};
  return launched(launch_sample(a, (hipStream_t)stream));
}

}  // extern "C"
