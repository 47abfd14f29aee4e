// Routing by scores: top-k of a token's permitted pool by score plus a balance bias, inside the
// best groups of experts, and the gradient of the gates.
//
//   s = sigmoid(z), or softmax(z) over the pool;  u = s + select_bias
//   a group's rank: the sum of its best one or two u; the best `keep` groups stay
//   the k largest u of the experts that stay win, ties to the lower id
//   gates: scale s, or scale s / sum of the winners' s (softmax: the softmax of the winners' z)
//
// One wave per token, expert i of the pool in register i / 64 of lane i % 64. Scores and u are fp64:
// the choice is that of 64-bit arithmetic, whatever two fp32 roundings would make of a near tie, and
// costs little here (fp64 runs at the rate of scalar fp32, and v_max_f64 makes a wave maximum of
// 64-bit keys six DPP steps of three instructions). The k winners are k wave maxima; a sort of
// the pool takes more for k up to 16.
#include <cfloat>

#include "pmpe_internal.h"

namespace pmpe {
namespace {

constexpr int SEL_WAVES = 4;

// max(v, v of the lane that the DPP control names); lanes without one keep v
template <int CTRL>
__device__ __forceinline__ double dpp_max(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const int lo = (int)(uint32_t)u, hi = (int)(u >> 32);
  const uint32_t l2 = (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xF, 0xF, false);
  const uint32_t h2 = (uint32_t)__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xF, 0xF, false);
  return fmax(v, __longlong_as_double((long long)(((uint64_t)h2 << 32) | l2)));
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
// Maximum over the wave: shifts by 1, 2, 4, 8 in each row of 16 lanes, then the row ends of rows 0
// and 2 into rows 1 and 3, and of row 1 into rows 2 and 3; lane 63 has it.
__device__ __forceinline__ double wave_max(double v) {
  v = dpp_max<0x111>(v);
  v = dpp_max<0x112>(v);
  v = dpp_max<0x114>(v);
  v = dpp_max<0x118>(v);
  v = dpp_max<0x142>(v);
  v = dpp_max<0x143>(v);
  return read_lane(v, 63);
}
__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// The pool of a token: columns [first, first + n) of the experts, its groups.
struct Pool {
  int first, n, groups, keep;
};
__device__ __forceinline__ Pool pool_of(const SelectArgs& a, int tau) {
  if (a.soft) return {0, a.n_pub + a.n_priv, 1, 1};
  return tau ? Pool{a.n_pub, a.n_priv, a.groups_priv, a.keep_priv} : Pool{0, a.n_pub, a.groups_pub, a.keep_pub};
}
// Logit of expert i of the pool: the caller's [T, E] array, or the router's partial sums of the
// token's pool, added in order.
__device__ __forceinline__ float logit(const SelectArgs& a, int t, const Pool& p, int i) {
  if (a.z_bf16) return bf16_to_f32(((const uint16_t*)a.z)[(size_t)t * a.zstride + p.first + i]);
  const float* z = (const float*)a.z + (size_t)t * a.zstride + (a.zpool ? 0 : p.first) + i;
  float v = z[0];
  for (int q = 1; q < a.zsplit; ++q) v += z[(size_t)q * a.T * a.zstride];
  return v;
}
// A masked logit (-inf) or NaN has score 0 and ranks behind every other; +inf counts as the
// largest finite value.
__device__ __forceinline__ bool live_logit(float z) { return z > -INFINITY; }
__device__ __forceinline__ double sigmoid64(float z) {
  const double e = exp(-fabs((double)z));
  return (z < 0.f ? e : 1.0) / (1.0 + e);
}

// NPL registers of experts per lane; tau and the pool are the wave's own.
template <int NPL>
__device__ void select_token(const SelectArgs& a, int t, int tau, const Pool& p, double* s_u) {
  const int lane = lane_id(), k = a.k;
  double u[NPL];
  double top = -INFINITY, den = 1.0;
  if (a.sigmoid) {
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const int i = r * 64 + lane;
      u[r] = -INFINITY;
      if (i < p.n) {
        const float z = logit(a, t, p, i);
        u[r] = live_logit(z) ? sigmoid64(z) : -DBL_MAX;
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const int i = r * 64 + lane;
      u[r] = -INFINITY;
      if (i < p.n) {
        const float z = logit(a, t, p, i);
        u[r] = live_logit(z) ? (double)fminf(z, FLT_MAX) : -DBL_MAX;
      }
      top = fmax(top, u[r]);
    }
    top = wave_max(top);
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      if (u[r] > -DBL_MAX) {
        u[r] = exp(u[r] - top);
        sum += u[r];
      }
    }
    den = wave_add(sum);
#pragma unroll
    for (int r = 0; r < NPL; ++r)
      if (u[r] > -DBL_MAX) u[r] /= den;
  }
  // -DBL_MAX: a masked expert, behind every other; -INFINITY: none, or out of the running
  if (a.select_bias) {
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const int i = r * 64 + lane;
      if (i < p.n && u[r] > -DBL_MAX) {
        u[r] += (double)a.select_bias[p.first + i];
        if (!(u[r] > -DBL_MAX)) u[r] = -DBL_MAX;  // a bias of -inf or NaN
      }
    }
  }
  if (p.keep < p.groups) {
    // lanes g * per .. g * per + per - 1 find the best two u of group g
    const int gs = p.n / p.groups;
    int per = 64;
    while (per * p.groups > 64) per >>= 1;
#pragma unroll
    for (int r = 0; r < NPL; ++r) s_u[r * 64 + lane] = u[r];
    __builtin_amdgcn_s_waitcnt(0xc07f);  // the wave's LDS writes are done before its reads
    __builtin_amdgcn_wave_barrier();
    const int g = lane / per;
    double b0 = -INFINITY, b1 = -INFINITY;
    if (g < p.groups)
      for (int i = lane % per; i < gs; i += per) {
        const double v = s_u[g * gs + i];
        b1 = fmax(b1, fmin(b0, v));
        b0 = fmax(b0, v);
      }
    for (int off = 1; off < per; off <<= 1) {
      const double o0 = __shfl_xor(b0, off, 64), o1 = __shfl_xor(b1, off, 64);
      b1 = fmax(fmin(b0, o0), fmax(b1, o1));
      b0 = fmax(b0, o0);
    }
    // masked experts add nothing; a group of masked ones only ranks behind the others
    if (a.group_top == 2 && b1 > -DBL_MAX) b0 += b1;
    int rank = 0;
    for (int q = 0; q < p.groups; ++q) {
      const double v = read_lane(b0, q * per);
      rank += (v > b0 || (v == b0 && q < g)) ? 1 : 0;
    }
    const uint64_t kept = __ballot(g < p.groups && rank < p.keep);
    const float inv = 1.0f / (float)gs;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const int i = r * 64 + lane;
      const int gi = (int)(((float)i + 0.5f) * inv);  // i / gs (i < 512)
      if (i >= p.n || !((kept >> (gi * per)) & 1)) u[r] = -INFINITY;
    }
  }
  // k winners, lane j keeping the j-th, and (for the margin) the u of the last and of the next
  int mine = 0;
  double last = 0.0;
  for (int j = 0; j < k; ++j) {
    double m = u[0];
#pragma unroll
    for (int r = 1; r < NPL; ++r) m = fmax(m, u[r]);
    m = wave_max(m);
    int id = -1;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const uint64_t at = __ballot(u[r] == m);
      if (id < 0 && at) id = r * 64 + __builtin_ctzll(at);
    }
#pragma unroll
    for (int r = 0; r < NPL; ++r)
      if (r * 64 + lane == id) u[r] = -INFINITY;
    if (lane == j) mine = id;
    last = m;
  }
  // gates from the winners' own logits
  const float z = lane < k ? logit(a, t, p, mine) : -INFINITY;
  const bool live = live_logit(z);
  double s = 0.0;
  if (a.sigmoid) {
    if (live) s = sigmoid64(z);
    if (a.renorm) s /= wave_add(s) + 1e-20;
  } else {
    const double zd = live ? (double)fminf(z, FLT_MAX) : -DBL_MAX;
    if (a.renorm) {
      top = wave_max(zd);
      s = live ? exp(zd - top) : 0.0;
      const double sum = wave_add(s);
      if (sum > 0.0) s /= sum;
    } else if (live) {
      s = exp(zd - top) / den;
    }
  }
  int pos = 0;
  for (int q = 0; q < k; ++q) pos += __builtin_amdgcn_readlane(mine, q) < mine ? 1 : 0;
  if (lane < k) {
    const size_t o = (size_t)t * k + pos;
    a.topk_idx[o] = p.first + mine;
    a.topk_gate[o] = (float)(s * (double)a.scale);
    if (a.topk_logit) a.topk_logit[o] = z;
  }
  if (a.margin) {
    double m = u[0];
#pragma unroll
    for (int r = 1; r < NPL; ++r) m = fmax(m, u[r]);
    m = wave_max(m);
    // no other expert left, or only masked ones: +inf (0 between two masked ones)
    if (lane == 0) a.margin[t] = m == last ? 0.f : m <= -DBL_MAX ? INFINITY : (float)(last - m);
  }
  if (lane == 0) a.allow[t] = (uint8_t)tau;
}

__global__ __launch_bounds__(64 * SEL_WAVES) void select_kernel(SelectArgs a) {
  __shared__ double s_u[SEL_WAVES][2 * PMPE_MAX_POOL];
  const int w = threadIdx.x >> 6, t = blockIdx.x * SEL_WAVES + w;
  if (t >= a.T) return;  // wave-uniform; no block barrier follows
  int tau = (a.words != nullptr && a.words[t] == PMPE_POLICY_ALLOW) ? 1 : 0;
  if (tau && a.no_private) {
    tau = 0;
    if (a.dev_status && lane_id() == 0) atomicOr(a.dev_status, PMPE_DEV_PRIV_ROUTER_MISSING);
  }
  tau = __builtin_amdgcn_readfirstlane(tau);
  const Pool p = pool_of(a, tau);
  if (p.n <= 64)
    select_token<1>(a, t, tau, p, s_u[w]);
  else if (p.n <= 128)
    select_token<2>(a, t, tau, p, s_u[w]);
  else if (p.n <= 256)
    select_token<4>(a, t, tau, p, s_u[w]);
  else
    select_token<8>(a, t, tau, p, s_u[w]);
}

// Gradient of the logits, one wave per token: the whole row of dlogits is written, zero outside the
// token's pool (the one that its first selected expert lies in). An id that lies outside it is
// passed over.
template <int NPL>
__device__ void select_bwd_token(const SelectBwdArgs& a, int t, const Pool& p) {
  const SelectArgs& f = a.f;
  const int lane = lane_id(), k = f.k;
  const int id = lane < k ? f.topk_idx[(size_t)t * k + lane] - p.first : -1;
  const bool in = id >= 0 && id < p.n;
  const float z = in ? logit(f, t, p, id) : -INFINITY;
  const bool live = live_logit(z);
  const float dg = in ? a.dgate[(size_t)t * k + lane] : 0.f;
  float top = 0.f, den = 1.f, mean = 0.f, dz = 0.f;
  float v[NPL];
#pragma unroll
  for (int r = 0; r < NPL; ++r) v[r] = 0.f;
  if (f.sigmoid) {
    const float e = live ? expf(-fabsf(z)) : 0.f;
    const float s = live ? (z < 0.f ? e : 1.f) / (1.f + e) : 0.f;
    float ds = f.scale * dg;
    if (f.renorm) {
      const float inv = 1.f / (wave_sum(s) + 1e-20f);
      ds = f.scale * inv * (dg - wave_sum(s * dg) * inv);
    }
    dz = live ? ds * e / ((1.f + e) * (1.f + e)) : 0.f;
  } else if (f.renorm) {
    const float zc = live ? fminf(z, FLT_MAX) : -FLT_MAX;
    top = zc;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float s = live ? expf(zc - top) : 0.f;
    den = wave_sum(s);
    const float pr = den > 0.f ? s / den : 0.f;
    dz = f.scale * pr * (dg - wave_sum(pr * dg));
  } else {
    // dense over the pool: p_e (dg_e - sum over the selected of p dg)
    top = -FLT_MAX;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      const int i = r * 64 + lane;
      v[r] = i < p.n ? logit(f, t, p, i) : -INFINITY;
      if (live_logit(v[r])) top = fmaxf(top, fminf(v[r], FLT_MAX));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      v[r] = live_logit(v[r]) ? expf(fminf(v[r], FLT_MAX) - top) : 0.f;
      sum += v[r];
    }
    den = wave_sum(sum);
    const float inv = den > 0.f ? 1.f / den : 0.f;
    const float pr = live ? expf(fminf(z, FLT_MAX) - top) * inv : 0.f;
    mean = wave_sum(pr * dg);
#pragma unroll
    for (int r = 0; r < NPL; ++r) v[r] *= -f.scale * inv * mean;
    dz = f.scale * pr * dg;
  }
  // the selected experts' own part, to the lanes that hold them
  for (int j = 0; j < k; ++j) {
    const int idj = __builtin_amdgcn_readlane(id, j);
    const float dj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(dz), j));
#pragma unroll
    for (int r = 0; r < NPL; ++r)
      if (r * 64 + lane == idj) v[r] += dj;
  }
  const int E = f.n_pub + f.n_priv;
  float* o = a.dlogits + (size_t)t * E;
#pragma unroll
  for (int r = 0; r < NPL; ++r) {
    const int i = r * 64 + lane;
    if (i < p.n) o[p.first + i] = v[r];
  }
  for (int i = lane; i < E - p.n; i += 64) o[i < p.first ? i : i + p.n] = 0.f;
}

__global__ __launch_bounds__(64 * SEL_WAVES) void select_bwd_kernel(SelectBwdArgs a) {
  const int t = blockIdx.x * SEL_WAVES + (threadIdx.x >> 6);
  if (t >= a.f.T) return;  // wave-uniform
  const Pool p = pool_of(a.f, __builtin_amdgcn_readfirstlane(a.f.topk_idx[(size_t)t * a.f.k] >= a.f.n_pub ? 1 : 0));
  if (p.n <= 64)
    select_bwd_token<1>(a, t, p);
  else if (p.n <= 128)
    select_bwd_token<2>(a, t, p);
  else if (p.n <= 256)
    select_bwd_token<4>(a, t, p);
  else
    select_bwd_token<8>(a, t, p);
}

}  // namespace

hipError_t launch_select(const SelectArgs& a, hipStream_t s) {
  select_kernel<<<(a.T + SEL_WAVES - 1) / SEL_WAVES, 64 * SEL_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_select_bwd(const SelectBwdArgs& a, hipStream_t s) {
  select_bwd_kernel<<<(a.f.T + SEL_WAVES - 1) / SEL_WAVES, 64 * SEL_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace pmpe
