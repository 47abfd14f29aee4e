// Routing by scores: top-k of a token's permitted pool by score plus a balance bias, inside the
// best groups of experts, and the gradient of the gates.
//
//   s = sigmoid(z), or softmax(z) over the pool;  u = s + select_bias
//   a group's rank: its best u, or the sum of its best two, (s + s) + (bias + bias); the best `keep` stay
//   the k largest u of the experts that stay win, ties to the lower id
//   gates: scale s, or scale s / sum of the winners' s (softmax: the softmax of the winners' z)
//
// One wave per token, expert i of the pool in register i / 64 of lane i % 64. Scores and u are fp64:
// the choice is that of 64-bit arithmetic, whatever two fp32 roundings would make of a near tie
// (fp64 runs at the rate of scalar fp32). u becomes a 64-bit key of the same order, of which a round
// compares the upper word (20 bits of mantissa) by six DPP maxima; only when experts tie there
// does it look at the lower word. The k winners are k such rounds: a sort of the pool takes more for
// k up to 16. Bound by the vector instructions of a token (556 at 256 experts in 8 groups, k 8: half of
// them the scores in 64 bits): 16384 such tokens take 22 us, of which their issue is 16; 16.8 MB of
// logits alone would take 4. (Of them the test for ranks that are as good as equal takes 1, with a balance
// bias.) 32 us with fp64 maxima, library exponentials and winners gathered by lane moves; 26 with the rows'
// loads behind one another.
#include <cfloat>

#include "exp64.h"
#include "pmpe_internal.h"

namespace pmpe {
namespace {

constexpr int SEL_WAVES = 4;

// op(v, v of the lane that the DPP control names), where lanes without one take `none`
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, 0xF, 0xF, false);
}
// Maximum over the wave: shifts by 1, 2, 4, 8 in each row of 16 lanes, then the row ends of rows 0
// and 2 into rows 1 and 3, and of row 1 into rows 2 and 3; lane 63 has it.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, dpp<0x111>(v, 0));
  v = max(v, dpp<0x112>(v, 0));
  v = max(v, dpp<0x114>(v, 0));
  v = max(v, dpp<0x118>(v, 0));
  v = max(v, dpp<0x142>(v, 0));
  v = max(v, dpp<0x143>(v, 0));
  return __builtin_amdgcn_readlane(v, 63);
}
template <int CTRL>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint64_t o = ((uint64_t)dpp<CTRL>((uint32_t)(u >> 32), 0) << 32) | dpp<CTRL>((uint32_t)u, 0);
  return v + __longlong_as_double((long long)o);
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
// Sums of the first 16 lanes and of the wave, by the same steps.
__device__ __forceinline__ double row_add(double v) {
  return dpp_add<0x118>(dpp_add<0x114>(dpp_add<0x112>(dpp_add<0x111>(v))));
}
__device__ __forceinline__ double wave_add(double v) { return read_lane(dpp_add<0x143>(dpp_add<0x142>(row_add(v))), 63); }
__device__ __forceinline__ double first_row_add(double v) { return read_lane(row_add(v), 15); }

// 1 / d for d in [1, 2], to about one step: the hardware's reciprocal and two Newton steps.
__device__ __forceinline__ double rcp64(double d) {
  double r = __builtin_amdgcn_rcp(d);
  r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
  return __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
}

// Keys of the order of u, as two words. A masked expert (u = -DBL_MAX) has MASKED_HI and 0, every other live
// one more; below it lie experts out of the running (u = -inf) and winners of earlier rounds (0).
constexpr uint32_t MASKED_HI = 0x00100000u;
__device__ __forceinline__ uint64_t key_of(double u) {
  const uint64_t b = (uint64_t)__double_as_longlong(u);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double u_of(uint64_t key) {
  return __longlong_as_double((long long)(key ^ ((key >> 63) ? 0x8000000000000000ull : ~0ull)));
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
// Those of experts lane, 64 + lane, .. of the pool (-inf past its end), all loads of them in flight at once.
template <int NPL>
__device__ __forceinline__ void logits(const SelectArgs& a, int t, const Pool& p, float (&v)[NPL]) {
  const int lane = lane_id();
  if (a.z_bf16) {
    const uint16_t* z = (const uint16_t*)a.z + (size_t)t * a.zstride + p.first;
#pragma unroll
    for (int r = 0; r < NPL; ++r) v[r] = r * 64 + lane < p.n ? bf16_to_f32(z[r * 64 + lane]) : -INFINITY;
    return;
  }
  const float* z = (const float*)a.z + (size_t)t * a.zstride + (a.zpool ? 0 : p.first);
#pragma unroll
  for (int r = 0; r < NPL; ++r) v[r] = r * 64 + lane < p.n ? z[r * 64 + lane] : -INFINITY;
  for (int q = 1; q < a.zsplit; ++q) {
    z += (size_t)a.T * a.zstride;
#pragma unroll
    for (int r = 0; r < NPL; ++r) v[r] += r * 64 + lane < p.n ? z[r * 64 + lane] : 0.f;
  }
}
// A masked logit (-inf) or NaN has score 0 and ranks behind every other; +inf counts as the
// largest finite value.
__device__ __forceinline__ bool live_logit(float z) { return z > -INFINITY; }
// For z >= 0 the complement of that of -z: the two then add up to 1 in fp64 as well (the complement is off by
// 2^-54 at most, the sum of the two by less than half a step from 1).
__device__ __forceinline__ double sigmoid64(float z) {
#pragma clang fp contract(off)
  const double e = exp64(-fabs((double)z));
  const double q = e * rcp64(1.0 + e);
  return z < 0.f ? q : 1.0 - q;
}

// LDS of a wave: u of the pool for the groups' ranks, then the winners' ids and logits.
union SelectLds {
  double u[2 * PMPE_MAX_POOL];
  struct {
    int id[PMPE_MAX_TOPK];
    float z[PMPE_MAX_TOPK];
  } win;
};
// The wave's LDS writes are done, and no later access moves ahead of them.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// Ranks of the groups where two of them are as good as equal: a rank is (s + s) + (bias + bias), so that
// equal sums have equal bits wherever the biases lie, and the u of two experts are each rounded. One lane per
// group; u in LDS, where the experts of the groups that do not stay become -inf. Only where few values of logits and
// biases occur (one lane walks a group: the 16384 tokens take 44 us if all of them come here).
__device__ __forceinline__ void near_ranks(const SelectArgs& a, int t, const Pool& p, float top, double inv, SelectLds& lds) {
#pragma clang fp contract(off)
  const int gs = p.n / p.groups, g = lane_id();
  double* u = lds.u + g * gs;
  double r = -INFINITY;
  if (g < p.groups) {
    int i0 = 0, i1 = -1;
    for (int i = 1; i < gs; ++i) {
      if (u[i] > u[i0]) {
        i1 = i0;
        i0 = i;
      } else if (i1 < 0 || u[i] > u[i1]) {
        i1 = i;
      }
    }
    r = u[i0];
    if (i1 >= 0 && u[i1] > -DBL_MAX) {
      auto score = [&](int i) {
        const float z = logit(a, t, p, g * gs + i);
        return a.sigmoid ? sigmoid64(z) : exp64((double)fminf(z, FLT_MAX) - (double)top) * inv;
      };
      const float* bias = a.select_bias + p.first + g * gs;
      r = (score(i0) + score(i1)) + ((double)bias[i0] + (double)bias[i1]);
    }
  }
  int rank = 0;
  for (int q = 0; q < p.groups; ++q) {
    const double v = read_lane(r, q);
    rank += (v > r || (v == r && q < g)) ? 1 : 0;
  }
  if (g < p.groups && rank >= p.keep)
    for (int i = 0; i < gs; ++i) u[i] = -INFINITY;
}

// NPL registers of experts per lane; tau and the pool are the wave's own.
template <int NPL>
__device__ void select_token(const SelectArgs& a, int t, int tau, const Pool& p, SelectLds& lds) {
  const int lane = lane_id(), k = a.k;
  float z[NPL], bias[NPL];
  double u[NPL];
  bool live[NPL];
  logits<NPL>(a, t, p, z);
  if (a.select_bias) {
#pragma unroll
    for (int r = 0; r < NPL; ++r) bias[r] = r * 64 + lane < p.n ? a.select_bias[p.first + r * 64 + lane] : 0.f;
  } else {
#pragma unroll
    for (int r = 0; r < NPL; ++r) bias[r] = 0.f;
  }
#pragma unroll
  for (int r = 0; r < NPL; ++r) live[r] = live_logit(z[r]);
  float top = -INFINITY;
  double inv = 1.0;
  if (a.sigmoid) {
#pragma unroll
    for (int r = 0; r < NPL; ++r) u[r] = sigmoid64(z[r]);
  } else {
#pragma unroll
    for (int r = 0; r < NPL; ++r)
      if (live[r]) top = fmaxf(top, fminf(z[r], FLT_MAX));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __uint_as_float(xor_lanes(__float_as_uint(top), off)));
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      u[r] = live[r] ? exp64((double)fminf(z[r], FLT_MAX) - (double)top) : 0.0;
      sum += u[r];
    }
    inv = 1.0 / fmax(wave_add(sum), DBL_MIN);
#pragma unroll
    for (int r = 0; r < NPL; ++r) u[r] *= inv;
  }
#pragma unroll
  for (int r = 0; r < NPL; ++r) {
    u[r] += (double)bias[r];
    if (!live[r] || !(u[r] > -DBL_MAX)) u[r] = -DBL_MAX;  // masked (also by a bias of -inf or NaN)
    if (r * 64 + lane >= p.n) u[r] = -INFINITY;
  }
  if (p.keep < p.groups) {
    // lanes g * per .. g * per + per - 1 find the best two u of group g
    const int gs = p.n / p.groups;
    int per = 64;
    while (per * p.groups > 64) per >>= 1;
#pragma unroll
    for (int r = 0; r < NPL; ++r) lds.u[r * 64 + lane] = u[r];
    wave_lds_fence();
    const int g = lane / per;
    double b0 = -INFINITY, b1 = -INFINITY;
    if (g < p.groups)
      for (int i = lane % per; i < gs; i += per) {
        const double v = lds.u[g * gs + i];
        b1 = fmax(b1, fmin(b0, v));
        b0 = fmax(b0, v);
      }
    auto merge = [&](int off) {
      const uint64_t x = (uint64_t)__double_as_longlong(b0), y = (uint64_t)__double_as_longlong(b1);
      const double o0 = __longlong_as_double((long long)(((uint64_t)xor_lanes((uint32_t)(x >> 32), off) << 32) | xor_lanes((uint32_t)x, off)));
      const double o1 = __longlong_as_double((long long)(((uint64_t)xor_lanes((uint32_t)(y >> 32), off) << 32) | xor_lanes((uint32_t)y, off)));
      b1 = fmax(fmin(b0, o0), fmax(b1, o1));
      b0 = fmax(b0, o0);
    };
    if (per > 1) merge(1);
    if (per > 2) merge(2);
    if (per > 4) merge(4);
    if (per > 8) merge(8);
    if (per > 16) merge(16);
    if (per > 32) merge(32);
    // masked experts add nothing; a group of masked ones only ranks behind the others
    const bool two = a.group_top == 2 && b1 > -DBL_MAX;
    const double room = 0x1p-48 * (fabs(b0) + (two ? fabs(b1) : 0.0) + 1.0);
    const double u0 = b0, u1 = b1;
    if (two) b0 += b1;
    int rank = 0;
    for (int q = 0; q < p.groups; ++q) {
      const double v = read_lane(b0, q * per);
      rank += (v > b0 || (v == b0 && q < g)) ? 1 : 0;
    }
    // A sum of two u is off by less than an eighth of `room`, as is near_ranks' own: where a group that stays and the
    // first that does not, or one that does not and the last that stays, lie nearer to one another (and are not the
    // same two u), theirs decides.
    bool near = false;
    if (a.select_bias && a.group_top == 2) {
      const bool in = g < p.groups, stays = rank < p.keep;
      const int last = __builtin_ctzll(__ballot(in && rank == p.keep - 1)), next = __builtin_ctzll(__ballot(in && rank == p.keep));
      const double vl = read_lane(b0, last), vn = read_lane(b0, next);
      near = in && fmin(b0, vn) > -DBL_MAX && (stays ? b0 - vn : vl - b0) <= room;
      if (__ballot(near) != 0) {
        const double l0 = read_lane(u0, last), l1 = read_lane(u1, last), n0 = read_lane(u0, next), n1 = read_lane(u1, next);
        near = __ballot(near && (u0 != (stays ? n0 : l0) || u1 != (stays ? n1 : l1))) != 0;
      } else {
        near = false;
      }
    }
    if (near)
      near_ranks(a, t, p, top, inv, lds);
    else if (g < p.groups && rank >= p.keep)  // the experts of the other groups are out of the running
      for (int i = lane % per; i < gs; i += per) lds.u[g * gs + i] = -INFINITY;
    wave_lds_fence();
#pragma unroll
    for (int r = 0; r < NPL; ++r) u[r] = lds.u[r * 64 + lane];
    wave_lds_fence();  // they have been read: the winners go where u was
  }
  uint32_t hi[NPL], lo[NPL];
#pragma unroll
  for (int r = 0; r < NPL; ++r) {
    const uint64_t key = key_of(u[r]);
    hi[r] = (uint32_t)(key >> 32);
    lo[r] = (uint32_t)key;
  }
  // The winner of a round: the lowest id of the largest key. Its upper word becomes 0, which no other has.
  uint32_t last_hi = 0, last_lo = 0;
  auto round = [&](bool take) {
    uint32_t m = hi[0];
#pragma unroll
    for (int r = 1; r < NPL; ++r) m = max(m, hi[r]);
    last_hi = wave_max(m);
    uint64_t at[NPL];
    int cnt = 0;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      at[r] = __ballot(hi[r] == last_hi);
      cnt += __popcll(at[r]);
    }
    if (cnt > 1 || !take) {  // a tie in the upper word (or the whole key is asked for)
      m = 0;
#pragma unroll
      for (int r = 0; r < NPL; ++r) m = max(m, hi[r] == last_hi ? lo[r] : 0u);
      last_lo = wave_max(m);
#pragma unroll
      for (int r = 0; r < NPL; ++r) at[r] = __ballot(hi[r] == last_hi && lo[r] == last_lo);
    }
    if (!take) return;
    bool found = false;
#pragma unroll
    for (int r = 0; r < NPL; ++r) {
      if (!found && at[r] != 0) {  // (wave-uniform)
        const int l = __builtin_ctzll(at[r]);
        if (lane == l) hi[r] = 0;
        found = true;
      }
    }
  };
  for (int j = 0; j < k - 1; ++j) round(true);
  uint64_t last = 0;
  if (a.margin) {
    round(false);
    last = ((uint64_t)last_hi << 32) | last_lo;
  }
  round(true);
  // the winners in ascending order to lanes 0 .. k - 1
  int before = 0;
#pragma unroll
  for (int r = 0; r < NPL; ++r) {
    const uint64_t win = __ballot(hi[r] == 0);
    if (hi[r] == 0) {
      const int pos = before + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(win >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)win, 0));
      lds.win.id[pos] = r * 64 + lane;
      lds.win.z[pos] = z[r];
    }
    before += __popcll(win);
  }
  wave_lds_fence();
  const float zw = lane < k ? lds.win.z[lane] : -INFINITY;
  const bool lw = live_logit(zw);
  double s = 0.0;
  if (a.sigmoid) {
    if (lw) s = sigmoid64(zw);
    if (a.renorm) s /= first_row_add(s) + 1e-20;
  } else {
    const float zc = lw ? fminf(zw, FLT_MAX) : -FLT_MAX;
    if (a.renorm) {
      top = zc;
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __uint_as_float(xor_lanes(__float_as_uint(top), off)));
      s = lw ? exp64((double)zc - (double)top) : 0.0;
      s /= fmax(first_row_add(s), DBL_MIN);
    } else if (lw) {
      s = exp64((double)zc - (double)top) * inv;
    }
  }
  if (lane < k) {
    const size_t o = (size_t)t * k + lane;
    a.topk_idx[o] = p.first + lds.win.id[lane];
    a.topk_gate[o] = (float)(s * (double)a.scale);
    if (a.topk_logit) a.topk_logit[o] = zw;
  }
  if (a.margin) {
    round(false);
    const uint64_t next = ((uint64_t)last_hi << 32) | last_lo;
    // no other expert left, or only masked ones: +inf (0 between equal ones, two masked ones too)
    if (lane == 0) a.margin[t] = next == last ? 0.f : next <= (uint64_t)MASKED_HI << 32 ? INFINITY : (float)(u_of(last) - u_of(next));
  }
  if (lane == 0) a.allow[t] = (uint8_t)tau;
}

// WIDE: a pool of more than 256 experts. (Its registers in the same kernel cost the narrower pools 6 %.)
template <bool WIDE>
__global__ __launch_bounds__(64 * SEL_WAVES) void select_kernel(SelectArgs a) {
  __shared__ SelectLds s_lds[SEL_WAVES];
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
    select_token<1>(a, t, tau, p, s_lds[w]);
  else if (p.n <= 128)
    select_token<2>(a, t, tau, p, s_lds[w]);
  else
    select_token<WIDE ? 8 : 4>(a, t, tau, p, s_lds[w]);
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
    logits<NPL>(f, t, p, v);
#pragma unroll
    for (int r = 0; r < NPL; ++r)
      if (live_logit(v[r])) top = fmaxf(top, fminf(v[r], FLT_MAX));
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
  const int grid = (a.T + SEL_WAVES - 1) / SEL_WAVES;
  if ((a.soft ? a.n_pub + a.n_priv : max(a.n_pub, a.n_priv)) > 256)
    select_kernel<true><<<grid, 64 * SEL_WAVES, 0, s>>>(a);
  else
    select_kernel<false><<<grid, 64 * SEL_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_select_bwd(const SelectBwdArgs& a, hipStream_t s) {
  select_bwd_kernel<<<(a.f.T + SEL_WAVES - 1) / SEL_WAVES, 64 * SEL_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace pmpe
