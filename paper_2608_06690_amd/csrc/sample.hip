// One token per row of logits: temperature, top-k, top-p, min-p, and a draw by a given uniform number.
//
// The order of a row is (logit descending, id ascending); every cut leaves a leading part of it, and the
// draw is its first token whose cumulated mass exceeds u times the whole. Each of them is "the first place where
// the count, or the mass, up to it crosses a threshold": found bit by bit, first of the logit (as an unsigned
// key of the same order), then among the tokens of that logit of the id. A block has a row.
#include "pmpe_internal.h"

namespace pmpe {
namespace {

constexpr int THREADS = 1024;

__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float z_of(uint32_t k) { return __uint_as_float((k >> 31) ? k ^ 0x80000000u : ~k); }

struct Sum {
  double mass;
  int count;
};
__device__ Sum block_sum(Sum v) {
  __shared__ Sum s[THREADS / 64];
  for (int off = 32; off > 0; off >>= 1) {
    v.mass += __shfl_xor(v.mass, off, 64);
    v.count += __shfl_xor(v.count, off, 64);
  }
  __syncthreads();
  if (lane_id() == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  Sum t{0, 0};
  for (int w = 0; w < THREADS / 64; ++w) {
    t.mass += s[w].mass;
    t.count += s[w].count;
  }
  return t;
}

struct Row {
  const SampleArgs& a;
  int b;
  double inv, top;  // 1 / temperature, largest logit
  __device__ float z(int i) const {
    const size_t at = (size_t)b * a.stride + i;
    float v = a.bf16 ? bf16_to_f32(((const uint16_t*)a.z)[at]) : ((const float*)a.z)[at];
    v = v > -INFINITY ? fminf(v, 3.402823466e38f) : -INFINITY;
    return v == 0.f ? 0.f : v;  // (-0 is 0)
  }
  __device__ double mass(float v) const { return exp(((double)v - top) * inv); }
  // Sum over the tokens up to (key, id) of the order.
  __device__ Sum upto(uint32_t key, int id) const {
    Sum s{0, 0};
    for (int i = threadIdx.x; i < a.V; i += THREADS) {
      const float v = z(i);
      const uint32_t k = key_of(v);
      if (v > -INFINITY && (k > key || (k == key && i <= id))) {
        s.mass += mass(v);
        s.count += 1;
      }
    }
    return block_sum(s);
  }
  struct Place {
    uint32_t key;
    int id;
    Sum sum;  // up to and with it
  };
  template <class F>
  __device__ Place cross(F crossed) const {
    uint32_t key = 0;
    for (uint32_t bit = 1u << 31; bit; bit >>= 1)
      if (crossed(upto(key | bit, a.V))) key |= bit;
    int lo = -1, hi = a.V - 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (crossed(upto(key, mid))) hi = mid;
      else lo = mid;
    }
    return Place{key, hi, upto(key, hi)};
  }
};

__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
  const int b = blockIdx.x;
  Row row{a, b, 1.0, 0.0};
  const float t = a.temperature ? a.temperature[b] : 1.f;
  const bool greedy = !(t > 0.f);
  int k = greedy ? 1 : a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.f, least = a.min_p ? a.min_p[b] : 0.f;
  const Row::Place one = row.cross([](Sum s) { return s.count >= 1; });
  if (one.sum.count == 0) {
    if (threadIdx.x == 0) {
      a.token[b] = -1;
      if (a.prob) a.prob[b] = 0.f;
      if (a.kept) a.kept[b] = 0;
    }
    return;
  }
  row.inv = greedy ? 1.0 : 1.0 / (double)t;
  row.top = (double)z_of(one.key);
  Sum all = row.upto(0, a.V);
  if (k > 0 && k < all.count) all = row.cross([=](Sum s) { return s.count >= k; }).sum;
  if (p < 1.f) {
    const double want = (double)fmaxf(p, 0.f) * all.mass;
    all = row.cross([=](Sum s) { return s.count >= 1 && s.mass >= want; }).sum;
  }
  if (least > 0.f) {
    const double low = log(fmin((double)least, 1.0));
    Sum s{0, 0};
    for (int i = threadIdx.x; i < a.V; i += THREADS) {
      const float v = row.z(i);
      if (v > -INFINITY && ((double)v - row.top) * row.inv >= low) {
        s.mass += row.mass(v);
        s.count += 1;
      }
    }
    s = block_sum(s);
    if (s.count < all.count) all = s;
  }
  float u = a.u[b];
  u = u > 0.f ? u : 0.f;
  const double want = (double)u * all.mass;
  const int last = all.count;
  const Row::Place at = row.cross([=](Sum s) { return s.mass > want || s.count >= last; });
  if (threadIdx.x == 0) {
    a.token[b] = at.id;
    if (a.prob) a.prob[b] = (float)(row.mass(z_of(at.key)) / all.mass);
    if (a.kept) a.kept[b] = all.count;
  }
}

}  // namespace

size_t sample_workspace(int, int) { return 0; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  sample_kernel<<<a.B, THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace pmpe
