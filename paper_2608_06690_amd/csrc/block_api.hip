// C ABI of the operators around the layer: argument validation (host only, before any launch)
// and dispatch to the kernel launchers. No exception crosses this boundary; no device memory is allocated.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "pmpe_internal.h"

using namespace pmpe;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

pmpe_status launched(hipError_t e) { return e == hipSuccess ? PMPE_OK : PMPE_ERR_LAUNCH; }

bool float_type(int32_t t) { return t == PMPE_F32 || t == PMPE_BF16; }

constexpr int32_t kNormMaxH = 16384;

pmpe_status check_rows(int32_t T, int32_t H) {
  return T < 0 || T > PMPE_MAX_TOKENS || H < 1 || H > kNormMaxH ? PMPE_ERR_SHAPE : PMPE_OK;
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

// the descriptor of the 8-bit experts: the bf16 path's checks, with the weight type read as bf16
pmpe_status check_mx(const pmpe_layer_desc* d, int32_t T) {
  if (!d) return PMPE_ERR_NULL;
  if (d->act_dtype != PMPE_BF16 || d->w_dtype != PMPE_FP8_E4M3) return PMPE_ERR_DTYPE;
  pmpe_layer_desc db = *d;
  db.w_dtype = PMPE_BF16;
  const pmpe_status st = pmpe_check_desc(&db, T);
  if (st != PMPE_OK) return st;
  return d->n_shared != 0 || d->inter % 128 != 0 ? PMPE_ERR_SHAPE : PMPE_OK;
}

// sizes, types and pointers of a list of gradients
pmpe_status check_grads(const void* const* grads, const uint64_t* n, const int32_t* dtype, int32_t count) {
  if (count < 0 || count > PMPE_MAX_GRADS) return PMPE_ERR_SHAPE;
  if (count > 0 && (!grads || !n || !dtype)) return PMPE_ERR_NULL;
  for (int32_t i = 0; i < count; ++i) {
    if (!float_type(dtype[i])) return PMPE_ERR_DTYPE;
    if (n[i] >= ((uint64_t)1 << 43)) return PMPE_ERR_SHAPE;
    if (n[i] > 0 && !grads[i]) return PMPE_ERR_NULL;
    if (((uintptr_t)grads[i] & (dtype[i] == PMPE_BF16 ? 1u : 3u)) != 0) return PMPE_ERR_ALIGN;
  }
  return PMPE_OK;
}

// Whether an output shares memory with another output, or with a gradient that is not its own. (Lists
// side by side in memory, the usual ones, are seen to be apart in one pass.)
bool outputs_overlap(const void* const* grads, const void* const* outs, const uint64_t* n, const int32_t* dtype, int32_t count) {
  const auto bytes = [&](int32_t i) { return n[i] * (dtype[i] == PMPE_BF16 ? 2 : 4); };
  bool ascending = true, in_place = true;
  uintptr_t end = 0, o0 = UINTPTR_MAX, g0 = UINTPTR_MAX, g1 = 0, o1 = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (n[i] == 0) continue;
    const uintptr_t o = (uintptr_t)outs[i], g = (uintptr_t)grads[i];
    ascending = ascending && o >= end;
    in_place = in_place && o == g;
    end = o + bytes(i);
    o0 = std::min(o0, o);
    o1 = std::max(o1, end);
    g0 = std::min(g0, g);
    g1 = std::max(g1, g + bytes(i));
  }
  if (ascending && (in_place || o1 <= g0 || g1 <= o0)) return false;
  std::unique_ptr<int32_t[]> at(new (std::nothrow) int32_t[(size_t)count]);
  if (!at) return true;
  int32_t m = 0;
  for (int32_t i = 0; i < count; ++i)
    if (n[i] > 0) at[m++] = i;
  std::sort(at.get(), at.get() + m, [&](int32_t a, int32_t b) { return (uintptr_t)outs[a] < (uintptr_t)outs[b]; });
  for (int32_t j = 1; j < m; ++j)
    if ((uintptr_t)outs[at[j - 1]] + bytes(at[j - 1]) > (uintptr_t)outs[at[j]]) return true;
  for (int32_t i = 0; i < count; ++i) {  // the outputs lie apart: those around gradient i
    if (n[i] == 0) continue;
    const uintptr_t g = (uintptr_t)grads[i], e = g + bytes(i);
    int32_t j = (int32_t)(std::upper_bound(at.get(), at.get() + m, g, [&](uintptr_t v, int32_t a) { return v < (uintptr_t)outs[a]; }) - at.get());
    for (j = j > 0 ? j - 1 : 0; j < m && (uintptr_t)outs[at[j]] < e; ++j)
      if ((uintptr_t)outs[at[j]] + bytes(at[j]) > g && !(at[j] == i && (uintptr_t)outs[i] == g)) return true;
  }
  return false;
}

}  // namespace

namespace pmpe {

pmpe_status check_rule(const pmpe_layer_desc* d, const pmpe_score_rule* r) {
  if (!r) return PMPE_ERR_NULL;
  if (r->score != PMPE_SCORE_SOFTMAX && r->score != PMPE_SCORE_SIGMOID) return PMPE_ERR_SHAPE;
  if (r->group_top != 1 && r->group_top != 2) return PMPE_ERR_SHAPE;
  if (!std::isfinite(r->scale)) return PMPE_ERR_SHAPE;
  const int32_t pool[2][3] = {{d->n_pub, r->n_group_pub, r->topk_group_pub}, {d->n_priv, r->n_group_priv, r->topk_group_priv}};
  for (const auto& p : pool) {
    if (p[1] < 1 || p[1] > PMPE_MAX_GROUPS || p[2] < 1 || p[2] > p[1]) return PMPE_ERR_SHAPE;
    if (p[0] % p[1] != 0 || (p[0] > 0 && (int64_t)p[2] * (p[0] / p[1]) < d->top_k)) return PMPE_ERR_SHAPE;
    if (d->route_mode == PMPE_ROUTE_SOFT && p[1] != 1) return PMPE_ERR_SHAPE;
  }
  return PMPE_OK;
}

SelectArgs select_args(const pmpe_layer_desc* d, const pmpe_score_rule* r, int T) {
  SelectArgs a{};
  a.T = T;
  a.n_pub = d->n_pub;
  a.n_priv = d->n_priv;
  a.k = d->top_k;
  a.sigmoid = r->score == PMPE_SCORE_SIGMOID;
  a.renorm = d->gate_mode == PMPE_GATE_RENORM_TOPK;
  a.soft = d->route_mode == PMPE_ROUTE_SOFT;
  a.groups_pub = r->n_group_pub;
  a.keep_pub = r->topk_group_pub;
  a.groups_priv = r->n_group_priv;
  a.keep_priv = r->topk_group_priv;
  a.group_top = r->group_top;
  a.scale = r->scale;
  a.zstride = d->n_pub + d->n_priv;
  a.zsplit = 1;
  return a;
}

}  // namespace pmpe

extern "C" {

pmpe_status pmpe_rmsnorm(int32_t T, int32_t H, int32_t dtype, const void* x, const void* residual,
                         const void* weight, int32_t w_dtype, float eps, void* sum_out, void* out,
                         uint8_t* out_q, uint8_t* out_scale, float* rstd, pmpe_stream_t stream) {
  const pmpe_status st = check_rows(T, H);
  if (st != PMPE_OK) return st;
  if (!float_type(dtype) || !float_type(w_dtype)) return PMPE_ERR_DTYPE;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return PMPE_ERR_SHAPE;
  if (out_q && H % 32 != 0) return PMPE_ERR_SHAPE;
  if (T == 0) return PMPE_OK;  // (arrays without elements may be NULL)
  if (!x || !weight || (!out && !out_q) || (out_q != nullptr) != (out_scale != nullptr) ||
      (residual != nullptr) != (sum_out != nullptr))
    return PMPE_ERR_NULL;
  const void* al[] = {x, residual, weight, sum_out, out, out_q};
  for (const void* p : al)
    if (p && !aligned16(p)) return PMPE_ERR_ALIGN;
  NormArgs a{T, H, dtype == PMPE_BF16, w_dtype == PMPE_BF16, eps, x, residual, weight, sum_out, out, out_q,
             out_scale, rstd};
  return launched(launch_rmsnorm(a, (hipStream_t)stream));
}

size_t pmpe_rmsnorm_backward_workspace_bytes(int32_t T, int32_t H) {
  if (check_rows(T, H) != PMPE_OK || T == 0) return 0;
  return (size_t)rmsnorm_bwd_parts(T, H) * H * 4;
}

pmpe_status pmpe_rmsnorm_backward(int32_t T, int32_t H, int32_t dtype, const void* dy,
                                  int32_t dy_dtype, const void* dres, const void* r,
                                  const void* weight, int32_t w_dtype, const float* rstd, void* dx,
                                  float* dweight, void* ws, size_t ws_bytes, pmpe_stream_t stream) {
  const pmpe_status st = check_rows(T, H);
  if (st != PMPE_OK) return st;
  if (!float_type(dtype) || !float_type(w_dtype)) return PMPE_ERR_DTYPE;
  if (dy_dtype != PMPE_F32 && dy_dtype != dtype) return PMPE_ERR_DTYPE;
  if (T > 0 && (!dy || !r || !weight || !rstd || !dx)) return PMPE_ERR_NULL;
  const void* al[] = {dy, dres, r, weight, dx, dweight};
  for (const void* p : al)
    if (p && !aligned16(p)) return PMPE_ERR_ALIGN;
  const size_t need = pmpe_rmsnorm_backward_workspace_bytes(T, H);
  if (dweight && need > 0) {
    if (!ws || ws_bytes < need) return PMPE_ERR_WORKSPACE;
    if (!aligned16(ws)) return PMPE_ERR_ALIGN;
  }
  if (T == 0 && !dweight) return PMPE_OK;
  NormBwdArgs a{T, H, dtype == PMPE_BF16, dy_dtype == PMPE_F32, w_dtype == PMPE_BF16, dy, dres, r, weight, rstd,
                dx, dweight, dweight ? (float*)ws : nullptr};
  return launched(launch_rmsnorm_bwd(a, (hipStream_t)stream));
}

pmpe_status pmpe_select(const pmpe_layer_desc* d, const pmpe_score_rule* rule, int32_t T,
                        const void* logits, int32_t logits_dtype, const float* select_bias,
                        const uint32_t* policy_word, int32_t* topk_idx, float* topk_gate,
                        float* topk_logit, uint8_t* allow, float* margin, pmpe_stream_t stream) {
  pmpe_status st = pmpe_check_desc(d, T);
  if (st == PMPE_OK) st = check_rule(d, rule);
  if (st != PMPE_OK) return st;
  if (!float_type(logits_dtype)) return PMPE_ERR_DTYPE;
  if (T == 0) return PMPE_OK;
  if (!logits || !topk_idx || !topk_gate || !allow) return PMPE_ERR_NULL;
  SelectArgs a = select_args(d, rule, T);
  a.z = logits;
  a.z_bf16 = logits_dtype == PMPE_BF16;
  a.select_bias = select_bias;
  a.words = policy_word;
  a.topk_idx = topk_idx;
  a.topk_gate = topk_gate;
  a.topk_logit = topk_logit;
  a.allow = allow;
  a.margin = margin;
  return launched(launch_select(a, (hipStream_t)stream));
}

pmpe_status pmpe_select_backward(const pmpe_layer_desc* d, const pmpe_score_rule* rule, int32_t T,
                                 const void* logits, int32_t logits_dtype, const int32_t* topk_idx,
                                 const float* dgate, float* dlogits, pmpe_stream_t stream) {
  pmpe_status st = pmpe_check_desc(d, T);
  if (st == PMPE_OK) st = check_rule(d, rule);
  if (st != PMPE_OK) return st;
  if (!float_type(logits_dtype)) return PMPE_ERR_DTYPE;
  if (T == 0) return PMPE_OK;
  if (!logits || !topk_idx || !dgate || !dlogits) return PMPE_ERR_NULL;
  SelectBwdArgs a{select_args(d, rule, T), dgate, dlogits};
  a.f.z = logits;
  a.f.z_bf16 = logits_dtype == PMPE_BF16;
  a.f.topk_idx = const_cast<int32_t*>(topk_idx);
  return launched(launch_select_bwd(a, (hipStream_t)stream));
}

size_t pmpe_grad_norm_workspace_bytes(const uint64_t* n, int32_t count) {
  if (count < 0 || count > PMPE_MAX_GRADS || (count > 0 && !n)) return 0;
  uint64_t pieces = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (n[i] >= ((uint64_t)1 << 43)) return 0;
    pieces += (n[i] + GRAD_PIECE - 1) / GRAD_PIECE;
  }
  return (size_t)(pieces / GRAD_LIST + 1) * GRAD_BLOCKS * sizeof(double);
}

pmpe_status pmpe_grad_norm(const void* const* grads, const uint64_t* n, const int32_t* dtype,
                           int32_t count, double max_norm, float* norm, void* ws, size_t ws_bytes,
                           pmpe_stream_t stream) {
  const pmpe_status st = check_grads(grads, n, dtype, count);
  if (st != PMPE_OK) return st;
  if (!(max_norm > 0.0)) return PMPE_ERR_SHAPE;
  if (!norm) return PMPE_ERR_NULL;
  if (((uintptr_t)norm & 3u) != 0) return PMPE_ERR_ALIGN;
  if (!ws || ws_bytes < pmpe_grad_norm_workspace_bytes(n, count)) return PMPE_ERR_WORKSPACE;
  if (!aligned16(ws)) return PMPE_ERR_ALIGN;
  return launched(launch_grad_norm(GradListArgs{grads, nullptr, n, dtype, count}, max_norm, norm, (double*)ws,
                                   (hipStream_t)stream));
}

pmpe_status pmpe_clip_grads(const void* const* grads, void* const* outs, const uint64_t* n,
                            const int32_t* dtype, int32_t count, const float* norm,
                            pmpe_stream_t stream) {
  const pmpe_status st = check_grads(grads, n, dtype, count);
  if (st != PMPE_OK) return st;
  if (!norm) return PMPE_ERR_NULL;
  if (((uintptr_t)norm & 3u) != 0) return PMPE_ERR_ALIGN;
  for (int32_t i = 0; outs && i < count; ++i) {
    if (n[i] == 0) continue;
    if (!outs[i]) return PMPE_ERR_NULL;
    if (((uintptr_t)outs[i] & (dtype[i] == PMPE_BF16 ? 1u : 3u)) != 0) return PMPE_ERR_ALIGN;
  }
  if (outputs_overlap(grads, outs ? outs : grads, n, dtype, count)) return PMPE_ERR_SHAPE;
  return launched(launch_clip_grads(GradListArgs{grads, outs, n, dtype, count}, norm, (hipStream_t)stream));
}

size_t pmpe_expert_ffn_mx_workspace_bytes(const pmpe_layer_desc* d, int32_t T) {
  if (check_mx(d, T) != PMPE_OK) return 0;
  const size_t n = (size_t)T * d->top_k * d->inter;
  return round_up(n) + round_up(n / 32);
}

pmpe_status pmpe_expert_ffn_mx(const pmpe_layer_desc* d, int32_t T, const uint8_t* xq,
                               const uint8_t* xs, const int32_t* expert_count,
                               const int32_t* expert_offset, const int32_t* row_token,
                               const void* w13_pub, const void* w2_pub, const void* w13_priv,
                               const void* w2_priv, const float* w13s_pub, const float* w2s_pub,
                               const float* w13s_priv, const float* w2s_priv, void* y_perm,
                               uint32_t* audit_token_rows, uint32_t* audit_priv_calls,
                               uint32_t* dev_status, void* ws, size_t ws_bytes,
                               pmpe_stream_t stream) {
  const pmpe_status st = check_mx(d, T);
  if (st != PMPE_OK) return st;
  if (T == 0) return PMPE_OK;
  if (!xq || !xs || !expert_count || !expert_offset || !row_token || !w13_pub || !w2_pub || !w13s_pub || !w2s_pub ||
      !y_perm || !audit_token_rows)
    return PMPE_ERR_NULL;
  if ((w13_priv != nullptr) != (w13s_priv != nullptr) || (w2_priv != nullptr) != (w2s_priv != nullptr))
    return PMPE_ERR_NULL;
  const void* al[] = {xq, xs, w13_pub, w2_pub, w13_priv, w2_priv, y_perm};
  for (const void* p : al)
    if (p && !aligned16(p)) return PMPE_ERR_ALIGN;
  if (!ws || ws_bytes < pmpe_expert_ffn_mx_workspace_bytes(d, T)) return PMPE_ERR_WORKSPACE;
  if (!aligned16(ws)) return PMPE_ERR_ALIGN;
  uint8_t* hq = (uint8_t*)ws;
  MxFfnArgs a{T, d->hidden, d->inter, d->n_pub, d->n_priv, d->top_k, xq, xs, expert_count, expert_offset, row_token,
              w13_pub, w2_pub, w13_priv, w2_priv, w13s_pub, w2s_pub, w13s_priv, w2s_priv, y_perm,
              audit_token_rows, audit_priv_calls, dev_status, hq, hq + round_up((size_t)T * d->top_k * d->inter)};
  return launched(launch_expert_ffn_mx(a, (hipStream_t)stream));
}

}  // extern "C"
