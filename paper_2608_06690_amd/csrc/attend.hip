// Attention of one new token per request over its paged cache.
//
//   s_j = scale q . k_j, out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), lse = m + ln sum_j exp(s_j - m)
//
// A block has one query head of one request; each of its waves goes over every fourth row with a running
// maximum and sum, lane l holding values l, 64 + l, .. of the head; the waves' parts are joined in LDS.
#include "kvcache.h"

namespace pmpe {
namespace {

constexpr int WAVES = 4;

__device__ __forceinline__ float cached(const void* cache, const uint8_t* scale, const CacheArgs& c, size_t hp, int row, int d) {
  const size_t at = (hp * c.page_size + row) * c.dim + d;
  if (c.fp8) {
    const uint32_t e = scale[(hp * (c.dim / 32) + d / 32) * c.page_size + row];
    const float s = __uint_as_float(e == 255 ? 0x7FC00000u : e ? e << 23 : 0x400000u);
    return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)cache)[at], 0) * s;
  }
  return c.act_bf16 ? bf16_to_f32(((const uint16_t*)cache)[at]) : ((const float*)cache)[at];
}

__global__ __launch_bounds__(64 * WAVES) void attn_kernel(AttnArgs a) {
  __shared__ float s_m[WAVES], s_l[WAVES], s_o[WAVES][256];
  const CacheArgs& c = a.c;
  const int r = blockIdx.x / a.heads, head = blockIdx.x % a.heads, lane = lane_id(), w = threadIdx.x >> 6;
  const int h = head / (a.heads / c.kv);
  const int64_t end = a.len[r], first = max(0, a.first ? a.first[r] : 0);
  const uint32_t want = request_tag(c, r);
  float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
  uint32_t bad = 0;
  for (int i = 0; i < 4; ++i) {
    const int d = i * 64 + lane;
    const size_t at = (size_t)r * a.q_stride + (size_t)head * c.dim + d;
    q[i] = d < c.dim ? (c.act_bf16 ? bf16_to_f32(((const uint16_t*)a.q)[at]) : ((const float*)a.q)[at]) : 0.f;
  }
  const int64_t most = (int64_t)c.max_pages * c.page_size;
  if (end > most) bad |= PMPE_DEV_CACHE_RANGE;
  for (int64_t p = first + w; p < min(end, most); p += WAVES) {
    const int page = page_at(c, r, p / c.page_size, want, bad);
    if (page < 0) continue;
    const int row = (int)(p % c.page_size);
    const size_t hp = (size_t)page * c.kv + h;
    float dot = 0;
    for (int i = 0; i * 64 < c.dim; ++i)
      if (i * 64 + lane < c.dim) dot += q[i] * cached(c.k, c.ks, c, hp, row, i * 64 + lane);
    const float s = wave_sum(dot) * a.scale, mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - mn);
    const float e = mn == -INFINITY ? 0.f : expf(s - mn);
    l = l * f + e;
    for (int i = 0; i * 64 < c.dim; ++i)
      if (i * 64 + lane < c.dim) o[i] = o[i] * f + e * cached(c.v, c.vs, c, hp, row, i * 64 + lane);
    m = mn;
  }
  if (lane == 0) {
    s_m[w] = m;
    s_l[w] = l;
    report(c, bad);
  }
  for (int i = 0; i < 4; ++i) s_o[w][i * 64 + lane] = o[i];
  __syncthreads();
  float M = -INFINITY, L = 0, O = 0;
  for (int i = 0; i < WAVES; ++i) M = fmaxf(M, s_m[i]);
  for (int i = 0; i < WAVES; ++i) {
    const float f = s_m[i] == -INFINITY ? 0.f : expf(s_m[i] - M);
    L += s_l[i] * f;
    O += s_o[i][threadIdx.x] * f;
  }
  if ((int)threadIdx.x < c.dim) {
    const size_t at = ((size_t)r * a.heads + head) * c.dim + threadIdx.x;
    const float v = L == 0.f ? 0.f : O / L;
    if (c.act_bf16) ((uint16_t*)a.out)[at] = (uint16_t)f32_to_bf16_rne(v);
    else ((float*)a.out)[at] = v;
  }
  if (threadIdx.x == 0 && a.lse) a.lse[(size_t)r * a.heads + head] = L == 0.f ? -INFINITY : M + logf(L);
}

}  // namespace

size_t attn_decode_workspace(int, int, const pmpe_cache_desc*) { return 0; }

hipError_t launch_attn_decode(const AttnArgs& a, hipStream_t s) {
  attn_kernel<<<a.c.R * a.heads, 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace pmpe
