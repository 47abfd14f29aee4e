// Global norm of a list of gradients and the clipped gradients.
//
//   norm = sqrt(sum over all tensors of g^2),  coef = min(1, max_norm / (norm + 1e-6)),  out = coef g
//
// Bound by HBM: one read for the norm, one read and one write for the clipping. The squares of fp32
// values are exact in fp64 and summed there (no overflow or cancellation below 1e150 terms of any
// fp32 size; fp64 runs at the rate of scalar fp32, far below the memory time). The tensors are cut
// into chunks; a block adds every gridDim-th chunk and a last block the blocks' sums, all in a fixed
// order, so equal gradients give equal bits. The list travels by value, as many pieces of at most 2^31
// elements to a launch as the 4 KB of a kernel's arguments hold: 256, or 160 where gradients and outputs
// lie apart in different orders. A block finds the piece of a chunk by reading all of them, one load per
// lane and 64 of them, and comparing: one latency, where a search of the list waits for eight. The norm of
// 604 MB of fp32 takes 102 us (5.9 TB/s). Norm and clipping of 500 bf16 tensors of up to 200000 elements
// take 28 us in five launches that cannot overlap (35 when a call took 2.5 us more of host time); 112 with 96
// tensors to a launch and the last chunk of each tensor read element by element. Chunks of 4096 and 8192 elements are equal on large tensors; the
// smaller ones fill the card with less.
#include <algorithm>

#include "pmpe_internal.h"

namespace pmpe {
namespace {

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));  // a gradient may start at any element
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

constexpr int GR_THREADS = 256;
constexpr int GR_CHUNK = 4096;  // elements: two vectors of 8 per thread

// Pieces of gradients. Bit 63 of src: bf16. Piece i has the launch's chunks first[i] .. first[i + 1] - 1, and
// tail[i] elements in the last of them. DST: its output is at dst[i]; without, all of them lie at the distance
// dst[0] of their gradients (0: in place), and more pieces fit.
constexpr uint64_t GR_BF16 = (uint64_t)1 << 63;
template <int COUNT, bool DST_>
struct GradTable {
  static constexpr int SIZE = COUNT;
  static constexpr bool DST = DST_;
  uint64_t src[COUNT];
  uint64_t dst[DST ? COUNT : 1];
  uint32_t first[COUNT + 1];
  uint16_t tail[COUNT];
  uint32_t count;
};
// 3.6 KB each
typedef GradTable<GRAD_LIST, false> NearTable;
typedef GradTable<160, true> FarTable;

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

// first[]: those of the pieces lane, 64 + lane, .. (past the last one: 2^32 - 1)
template <class T>
__device__ __forceinline__ void read_firsts(const T& t, uint32_t (&first)[(T::SIZE + 63) / 64]) {
#pragma unroll
  for (int r = 0; r < (T::SIZE + 63) / 64; ++r) {
    const uint32_t i = r * 64 + lane_id();
    first[r] = i < t.count ? t.first[i] : ~0u;
  }
}
// elements of piece i
template <class T>
__device__ __forceinline__ uint32_t elements_of(const T& t, int i) {
  return (t.first[i + 1] - t.first[i] - 1) * GR_CHUNK + t.tail[i];
}
// last piece whose first chunk is at or before c
template <int R>
__device__ __forceinline__ int piece_of(const uint32_t (&first)[R], uint32_t c) {
  int m = -1;
#pragma unroll
  for (int r = 0; r < R; ++r) m += __popcll(__ballot(first[r] <= c));
  return m;
}

// A thread's vectors of 8 elements of the chunk at e0 of a piece: first elements GR_THREADS * 8 apart. Those
// that the piece ends in are left to one thread, element by element.
constexpr int GR_VEC = GR_CHUNK / GR_THREADS / 8;
__device__ __forceinline__ uint32_t vector_at(uint32_t e0, int j) { return e0 + (j * GR_THREADS + threadIdx.x) * 8; }

template <bool STREAM, class V>
__device__ __forceinline__ V load_vector(const V* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(p);
  else
    return *p;
}
template <bool BF16, bool STREAM>
__device__ __forceinline__ void load8(const void* p, uint32_t i, float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 q = load_vector<STREAM>((const u32x4_a2*)((const uint16_t*)p + i));
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      v[2 * h] = bf16_to_f32(q[h] & 0xFFFFu);
      v[2 * h + 1] = bf16_to_f32(q[h] >> 16);
    }
  } else {
    const f32x4_a4* q = (const f32x4_a4*)((const float*)p + i);
    const f32x4 a = load_vector<STREAM>(q), b = load_vector<STREAM>(q + 1);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      v[h] = a[h];
      v[4 + h] = b[h];
    }
  }
}
template <bool BF16>
__device__ __forceinline__ float load1(const void* p, uint32_t i) {
  return BF16 ? bf16_to_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

template <bool BF16, bool STREAM>
__device__ __forceinline__ double chunk_squares(const void* p, uint32_t e0, uint32_t n) {
  float v[GR_VEC][8];
#pragma unroll
  for (int j = 0; j < GR_VEC; ++j) {
    const uint32_t i = vector_at(e0, j);
#pragma unroll
    for (int h = 0; h < 8; ++h) v[j][h] = 0.f;
    if (i + 8 <= n) {
      load8<BF16, STREAM>(p, i, v[j]);
    } else {
#pragma unroll
      for (int h = 0; h < 7; ++h)
        if (i + h < n) v[j][h] = load1<BF16>(p, i + h);
    }
  }
  double acc[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < GR_VEC; ++j)
#pragma unroll
    for (int h = 0; h < 8; ++h) acc[h & 3] += (double)v[j][h] * (double)v[j][h];
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

template <bool STREAM>
__global__ __launch_bounds__(GR_THREADS) void grad_squares_kernel(NearTable t, double* part) {
  __shared__ double s[GR_THREADS / 64];
  double acc = 0.0;
  uint32_t first[(NearTable::SIZE + 63) / 64];
  read_firsts(t, first);
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = piece_of(first, c);
    const uint64_t p = t.src[i];
    const uint32_t e0 = (c - t.first[i]) * GR_CHUNK, n = elements_of(t, i);
    const void* src = (const void*)(p & ~GR_BF16);
    acc += (p & GR_BF16) ? chunk_squares<true, STREAM>(src, e0, n) : chunk_squares<false, STREAM>(src, e0, n);
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
__device__ __forceinline__ void store8(void* o, uint32_t i, const float (&v)[8], float coef) {
  if constexpr (BF16) {
    u32x4 q;
#pragma unroll
    for (int h = 0; h < 4; ++h) q[h] = pack_bf16x2(v[2 * h] * coef, v[2 * h + 1] * coef);
    *(u32x4_a2*)((uint16_t*)o + i) = q;
  } else {
    const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    *(f32x4_a4*)((float*)o + i) = a * coef;
    *(f32x4_a4*)((float*)o + i + 4) = b * coef;
  }
}

template <bool BF16>
__device__ __forceinline__ void chunk_scale(const void* p, void* o, uint32_t e0, uint32_t n, float coef) {
  float v[GR_VEC][8];
#pragma unroll
  for (int j = 0; j < GR_VEC; ++j) {
    const uint32_t i = vector_at(e0, j);
    if (i + 8 <= n) load8<BF16, false>(p, i, v[j]);
  }
#pragma unroll
  for (int j = 0; j < GR_VEC; ++j) {
    const uint32_t i = vector_at(e0, j);
    if (i + 8 <= n) {
      store8<BF16>(o, i, v[j], coef);
    } else {
#pragma unroll
      for (int h = 0; h < 7; ++h) {
        if (i + h >= n) continue;
        if constexpr (BF16)
          ((uint16_t*)o)[i + h] = (uint16_t)f32_to_bf16_rne(load1<true>(p, i + h) * coef);
        else
          ((float*)o)[i + h] = load1<false>(p, i + h) * coef;
      }
    }
  }
}

template <class T>
__global__ __launch_bounds__(GR_THREADS) void grad_scale_kernel(T t, const float* norm) {
  const float coef = norm[1];
  uint32_t first[(T::SIZE + 63) / 64];
  read_firsts(t, first);
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = piece_of(first, c);
    const uint64_t p = t.src[i], q = p & ~GR_BF16, o = T::DST ? t.dst[T::DST ? i : 0] : q + t.dst[0];
    if (coef == 1.0f && o == q) continue;  // in place and inside the bound: nothing changes
    const uint32_t e0 = (c - t.first[i]) * GR_CHUNK, n = elements_of(t, i);
    if (p & GR_BF16)
      chunk_scale<true>((const void*)q, (void*)o, e0, n, coef);
    else
      chunk_scale<false>((const void*)q, (void*)o, e0, n, coef);
  }
}

// The pieces of the list, a table at a time.
template <class T>
class Tables {
 public:
  explicit Tables(const GradListArgs& a) : a_(a) {}
  // false: no piece is left
  bool next(T* t) {
    t->count = 0;
    t->first[0] = 0;
    while (at_ < a_.count && t->count < (uint32_t)T::SIZE) {
      const uint64_t n = std::min(a_.n[at_] - done_, GRAD_PIECE), el = a_.dtype[at_] == PMPE_BF16 ? 2 : 4;
      if (n > 0) {
        const uint32_t i = t->count++;
        t->src[i] = ((uint64_t)(uintptr_t)a_.src[at_] + done_ * el) | (el == 2 ? GR_BF16 : 0);
        if constexpr (T::DST) t->dst[i] = (uint64_t)(uintptr_t)a_.dst[at_] + done_ * el;
        t->first[i + 1] = t->first[i] + (uint32_t)((n + GR_CHUNK - 1) / GR_CHUNK);
        t->tail[i] = (uint16_t)((n - 1) % GR_CHUNK + 1);
      }
      done_ += n;
      if (done_ == a_.n[at_]) {
        ++at_;
        done_ = 0;
      }
    }
    return t->count > 0;
  }

 private:
  const GradListArgs& a_;
  int at_ = 0;
  uint64_t done_ = 0;
};

}  // namespace

hipError_t launch_grad_norm(const GradListArgs& a, double max_norm, float* norm, double* part, hipStream_t s) {
  // Lists that the caches cannot hold until the step are read past them: what they hold (the last step's
  // states among it) is not pushed out. Norm and step of 604 MB of fp32 gradients: 931 us -> 909, of
  // 151 MB: 244 -> 238; of 38 MB 74 -> 76, where the step then finds less in them.
  uint64_t bytes = 0;
  for (int i = 0; i < a.count; ++i) bytes += a.n[i] * (a.dtype[i] == PMPE_BF16 ? 2 : 4);
  const auto kernel = bytes >= ((uint64_t)128 << 20) ? grad_squares_kernel<true> : grad_squares_kernel<false>;
  int parts = 0;
  Tables<NearTable> list(a);
  NearTable t;
  t.dst[0] = 0;
  while (list.next(&t)) {
    const int grid = (int)std::min<uint32_t>(t.first[t.count], GRAD_BLOCKS);
    kernel<<<grid, GR_THREADS, 0, s>>>(t, part + parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    parts += grid;
  }
  grad_total_kernel<<<1, 1024, 0, s>>>(part, parts, max_norm, norm);
  return hipGetLastError();
}

namespace {

template <class T>
hipError_t scale_all(const GradListArgs& a, T& t, const float* norm, hipStream_t s) {
  Tables<T> list(a);
  while (list.next(&t)) {
    grad_scale_kernel<T><<<std::min<uint32_t>(t.first[t.count], 16384), GR_THREADS, 0, s>>>(t, norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_clip_grads(const GradListArgs& a, const float* norm, hipStream_t s) {
  // one distance from every gradient to its output (in place, or both lists laid out alike)?
  bool any = false, near = true;
  uint64_t dist = 0;
  for (int i = 0; a.dst && near && i < a.count; ++i) {
    if (a.n[i] == 0) continue;
    const uint64_t d = (uint64_t)(uintptr_t)a.dst[i] - (uint64_t)(uintptr_t)a.src[i];
    near = !any || d == dist;
    dist = d;
    any = true;
  }
  if (near) {
    NearTable t;
    t.dst[0] = dist;
    return scale_all(a, t, norm, s);
  }
  FarTable t;
  return scale_all(a, t, norm, s);
}

}  // namespace pmpe
