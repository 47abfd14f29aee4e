// Global norm of a list of gradients and the clipped gradients.
//
//   norm = sqrt(sum over all tensors of g^2),  coef = min(1, max_norm / (norm + 1e-6)),  out = coef g
//
// Bound by HBM: one read for the norm, one read and one write for the clipping. The squares of fp32
// values are exact in fp64 and summed there (no overflow or cancellation below 1e150 terms of any
// fp32 size; fp64 runs at the rate of scalar fp32, far below the memory time). The tensors are cut
// into chunks; a block adds every gridDim-th chunk and a last block the blocks' sums, all in a fixed
// order, so equal gradients give equal bits. The list travels by value, GRAD_LIST tensors to a launch.
#include <algorithm>

#include "pmpe_internal.h"

namespace pmpe {
namespace {

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));  // a gradient may start at any element
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

constexpr int GR_THREADS = 256;
constexpr int GR_CHUNK = 8192;  // elements: four vectors of 8 per thread

struct GradTable {
  const void* src[GRAD_LIST];
  void* dst[GRAD_LIST];
  uint64_t n[GRAD_LIST];
  uint32_t first[GRAD_LIST + 1];  // first chunk of each tensor, and the number of chunks
  uint8_t bf16[GRAD_LIST];
};

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
// sum over the block's threads, in thread 0 (s: one double per wave)
template <int THREADS>
__device__ __forceinline__ double block_add(double v, double* s) {
  v = wave_add(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < THREADS / 64; ++w) v += s[w];
  return v;
}

// last tensor whose first chunk is at or before c
__device__ __forceinline__ int tensor_of(const GradTable& t, int count, uint32_t c) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const void* p, uint64_t e0, uint64_t n) {
  double acc[4] = {0, 0, 0, 0};
  if (e0 + GR_CHUNK <= n) {
    float v[GR_CHUNK / GR_THREADS];
#pragma unroll
    for (int j = 0; j < GR_CHUNK / GR_THREADS / 8; ++j) {
      const uint64_t i = e0 + (uint64_t)(j * GR_THREADS + threadIdx.x) * 8;
      if constexpr (BF16) {
        const u32x4 q = *(const u32x4_a2*)((const uint16_t*)p + i);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          v[8 * j + 2 * h] = bf16_to_f32(q[h] & 0xFFFFu);
          v[8 * j + 2 * h + 1] = bf16_to_f32(q[h] >> 16);
        }
      } else {
        const f32x4 a = *(const f32x4_a4*)((const float*)p + i), b = *(const f32x4_a4*)((const float*)p + i + 4);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          v[8 * j + h] = a[h];
          v[8 * j + 4 + h] = b[h];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < GR_CHUNK / GR_THREADS; ++j) acc[j & 3] += (double)v[j] * (double)v[j];
  } else {
    for (uint64_t i = e0 + threadIdx.x; i < n; i += GR_THREADS) {
      const double x = BF16 ? bf16_to_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
      acc[0] += x * x;
    }
  }
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

__global__ __launch_bounds__(GR_THREADS) void grad_squares_kernel(GradTable t, int count, double* part) {
  __shared__ double s[GR_THREADS / 64];
  double acc = 0.0;
  const uint32_t chunks = t.first[count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = tensor_of(t, count, c);
    const uint64_t e0 = (uint64_t)(c - t.first[i]) * GR_CHUNK;
    acc += t.bf16[i] ? chunk_squares<true>(t.src[i], e0, t.n[i]) : chunk_squares<false>(t.src[i], e0, t.n[i]);
  }
  acc = block_add<GR_THREADS>(acc, s);
  if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

__global__ __launch_bounds__(1024) void grad_total_kernel(const double* part, int parts, double max_norm, float* norm) {
  __shared__ double s[16];
  double acc = 0.0;
  for (int i = threadIdx.x; i < parts; i += 1024) acc += part[i];
  acc = block_add<1024>(acc, s);
  if (threadIdx.x == 0) {
    const double total = sqrt(acc), coef = max_norm / (total + 1e-6);
    norm[0] = (float)total;
    norm[1] = coef > 1.0 ? 1.0f : (float)coef;  // (NaN stays)
  }
}

template <bool BF16>
__device__ __forceinline__ void chunk_scale(const void* p, void* o, uint64_t e0, uint64_t n, float coef) {
  const uint64_t end = e0 + GR_CHUNK < n ? e0 + GR_CHUNK : n;
  if (e0 + GR_CHUNK <= n) {
    constexpr int V = GR_CHUNK / GR_THREADS / 8;
    if constexpr (BF16) {
      u32x4 q[V];
#pragma unroll
      for (int j = 0; j < V; ++j) q[j] = *(const u32x4_a2*)((const uint16_t*)p + e0 + (j * GR_THREADS + threadIdx.x) * 8);
#pragma unroll
      for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int h = 0; h < 4; ++h) q[j][h] = pack_bf16x2(bf16_to_f32(q[j][h] & 0xFFFFu) * coef, bf16_to_f32(q[j][h] >> 16) * coef);
        *(u32x4_a2*)((uint16_t*)o + e0 + (j * GR_THREADS + threadIdx.x) * 8) = q[j];
      }
    } else {
      f32x4 q[2 * V];
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) q[j] = *(const f32x4_a4*)((const float*)p + e0 + (j * GR_THREADS + threadIdx.x) * 4);
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) *(f32x4_a4*)((float*)o + e0 + (j * GR_THREADS + threadIdx.x) * 4) = q[j] * coef;
    }
  } else {
    for (uint64_t i = e0 + threadIdx.x; i < end; i += GR_THREADS) {
      if constexpr (BF16)
        ((uint16_t*)o)[i] = (uint16_t)f32_to_bf16_rne(bf16_to_f32(((const uint16_t*)p)[i]) * coef);
      else
        ((float*)o)[i] = ((const float*)p)[i] * coef;
    }
  }
}

__global__ __launch_bounds__(GR_THREADS) void grad_scale_kernel(GradTable t, int count, const float* norm) {
  const float coef = norm[1];
  const uint32_t chunks = t.first[count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = tensor_of(t, count, c);
    if (coef == 1.0f && t.dst[i] == t.src[i]) continue;  // in place and inside the bound: nothing changes
    const uint64_t e0 = (uint64_t)(c - t.first[i]) * GR_CHUNK;
    if (t.bf16[i])
      chunk_scale<true>(t.src[i], t.dst[i], e0, t.n[i], coef);
    else
      chunk_scale<false>(t.src[i], t.dst[i], e0, t.n[i], coef);
  }
}

// The next tensors of the list that have elements, from *at on: up to GRAD_LIST of them and 2^31 chunks.
int fill(const GradListArgs& a, int* at, GradTable* t) {
  int m = 0;
  uint64_t chunks = 0;
  for (; *at < a.count && m < GRAD_LIST; ++*at) {
    const int i = *at;
    if (a.n[i] == 0) continue;
    const uint64_t c = (a.n[i] + GR_CHUNK - 1) / GR_CHUNK;
    if (m > 0 && chunks + c > GRAD_MAX_CHUNKS) break;
    t->src[m] = a.src[i];
    t->dst[m] = a.dst ? a.dst[i] : const_cast<void*>(a.src[i]);
    t->n[m] = a.n[i];
    t->bf16[m] = a.dtype[i] == PMPE_BF16;
    t->first[m] = (uint32_t)chunks;
    chunks += c;
    ++m;
  }
  t->first[m] = (uint32_t)chunks;
  return m;
}

}  // namespace

hipError_t launch_grad_norm(const GradListArgs& a, double max_norm, float* norm, double* part, hipStream_t s) {
  int at = 0, parts = 0;
  while (at < a.count) {
    GradTable t;
    const int m = fill(a, &at, &t);
    if (m == 0) break;
    const int grid = (int)std::min<uint32_t>(t.first[m], GRAD_BLOCKS);
    grad_squares_kernel<<<grid, GR_THREADS, 0, s>>>(t, m, part + parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    parts += grid;
  }
  grad_total_kernel<<<1, 1024, 0, s>>>(part, parts, max_norm, norm);
  return hipGetLastError();
}

hipError_t launch_clip_grads(const GradListArgs& a, const float* norm, hipStream_t s) {
  int at = 0;
  while (at < a.count) {
    GradTable t;
    const int m = fill(a, &at, &t);
    if (m == 0) break;
    const int grid = (int)std::min<uint32_t>(t.first[m], 16384);
    grad_scale_kernel<<<grid, GR_THREADS, 0, s>>>(t, m, norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pmpe
