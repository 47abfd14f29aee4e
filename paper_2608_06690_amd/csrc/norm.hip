// Residual add and RMS norm of a layer's input, with an output in 8 bits, and its backward.
//
//   r    = round(x + residual)                 (or x itself)
//   rstd = 1 / sqrt(mean(r^2) + eps),  y = r rstd w
//   out  = round(y);  q = e4m3(y / s_b), s_b the block scale of 32 consecutive values
//   backward, with xhat = r rstd and g = dy w:
//   dx   = rstd (g - xhat mean(g xhat)) + dres,  dw = sum over the rows of dy xhat
//
// A row is held in registers from its load to its last store: W waves take it, V vectors of 8
// consecutive values per lane. Sums are fp32. The norm is taken of the rounded r, the value that
// the residual stream carries on, so the backward needs r and rstd only.
// The 8-bit block of 32 values lies in 4 neighbouring lanes.
//
// Bound by HBM (about 10 operations per value): 16384 rows of 2048 bf16 values with residual, both
// outputs and scales (303 MB) take 57 us, 5.3 TB/s. W is as many waves as hold the row with one vector
// per lane (that batch on one wave of four vectors: 69 us, its loads in flight too few); 8 rows take
// 3.5 us on the card. The backward of 4096 such rows with dw takes 21.5 us (16.5 and 4.8 for the sum of
// its parts; 84 MB: 16.4 at the copy's rate), of 16384 rows 67 (62 and 4.8).
#include <algorithm>
#include <type_traits>

#include "mx.h"
#include "pmpe_internal.h"

namespace pmpe {
namespace {

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));  // rows of any length start at any element
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

// Values [i, i + 8) of a row of n (values past it: 0).
template <bool BF16>
__device__ __forceinline__ void load8(const void* row, int i, int n, float (&v)[8]) {
  if (i + 8 <= n) {
    if constexpr (BF16) {
      const u32x4 q = *(const u32x4_a2*)((const uint16_t*)row + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = bf16_to_f32(q[j] & 0xFFFFu);
        v[2 * j + 1] = bf16_to_f32(q[j] >> 16);
      }
    } else {
      const f32x4 a = *(const f32x4_a4*)((const float*)row + i), b = *(const f32x4_a4*)((const float*)row + i + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = 0.f;
      if (i + j < n) v[j] = BF16 ? bf16_to_f32(((const uint16_t*)row)[i + j]) : ((const float*)row)[i + j];
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* row, int i, int n, const float (&v)[8]) {
  if (i + 8 <= n) {
    if constexpr (BF16) {
      *(u32x4_a2*)((uint16_t*)row + i) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                               pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    } else {
      *(f32x4_a4*)((float*)row + i) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4_a4*)((float*)row + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) {
        if constexpr (BF16) ((uint16_t*)row)[i + j] = (uint16_t)f32_to_bf16_rne(v[j]);
        else ((float*)row)[i + j] = v[j];
      }
  }
}
__device__ __forceinline__ void load_weight8(const void* w, int bf16, int i, int n, float (&v)[8]) {
  if (bf16) load8<true>(w, i, n, v);
  else load8<false>(w, i, n, v);
}

// Sum over the W waves of a row (the same value in every lane); s: W floats per row of LDS. A
// block that has several rows has them in waves of their own (W = 1).
template <int W>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    __syncthreads();  // the row before has been read
    if (lane_id() == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += s[w];
  }
  return v;
}

template <bool BF16, int W, int V>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void rmsnorm_kernel(NormArgs a) {
  constexpr int RPB = W == 1 ? 4 : 1;  // rows of a block
  __shared__ float s_sum[W];
  const int t = blockIdx.x * RPB + (W == 1 ? (int)(threadIdx.x >> 6) : 0);
  const int l = W == 1 ? lane_id() : (int)threadIdx.x, H = a.H;
  if (t >= a.T) return;  // whole waves; W > 1: no such block
  const size_t el = BF16 ? 2 : 4, row = (size_t)t * H;
  const char* x = (const char*)a.x + row * el;
  float r[V][8], ss = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) load8<BF16>(x, (v * W * 64 + l) * 8, H, r[v]);
  if (a.residual) {
    const char* res = (const char*)a.residual + row * el;
    char* sum = (char*)a.sum_out + row * el;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float b[8];
      const int i = (v * W * 64 + l) * 8;
      load8<BF16>(res, i, H, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        r[v][j] += b[j];
        if constexpr (BF16) r[v][j] = bf16_to_f32(f32_to_bf16_rne(r[v][j]));
      }
      store8<BF16>(sum, i, H, r[v]);
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += r[v][j] * r[v][j];
  ss = row_sum<W>(ss, s_sum);
  const float rstd = 1.0f / sqrtf(ss / (float)H + a.eps);
  if (a.rstd && l == 0) a.rstd[t] = rstd;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = (v * W * 64 + l) * 8;
    float w[8];
    load_weight8(a.weight, a.w_bf16, i, H, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= r[v][j] * rstd;
    if (a.out) store8<BF16>((char*)a.out + row * el, i, H, w);
    if (a.out_q) {  // (H is a multiple of 32: the four lanes of a block are all inside or all past it)
      const float amax = mx_max_lanes<1, 2>(mx_amax8(w));
      if (i < H) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        uint32_t q0, q1;
        const int e = mx_pack8(w, amax, q0, q1);
        *(u32x2*)(a.out_q + row + i) = u32x2{q0, q1};
        if ((l & 3) == 0) a.out_scale[(row + i) >> 5] = (uint8_t)(e + 127);
      }
    }
  }
}

// Block b takes rows b, b + gridDim.x, ... (W waves to a row; W == 1: its four waves take
// every fourth of them) and adds their dw in registers, row by row; with W == 1 the waves' sums
// are added in wave order in LDS. dw_part [gridDim.x, H].
template <bool BF16, bool DY32, int W, int V>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void rmsnorm_bwd_kernel(NormBwdArgs a) {
  constexpr int RPB = W == 1 ? 4 : 1;
  __shared__ float s_sum[W];
  const int l = W == 1 ? lane_id() : (int)threadIdx.x, H = a.H, wave = threadIdx.x >> 6;
  const size_t el = BF16 ? 2 : 4, del = DY32 ? 4 : 2;
  float w[V][8], dw[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    load_weight8(a.weight, a.w_bf16, (v * W * 64 + l) * 8, H, w[v]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = 0.f;
  }
  for (int64_t t = (int64_t)blockIdx.x * RPB + (W == 1 ? wave : 0); t < a.T; t += (int64_t)gridDim.x * RPB) {
    const size_t row = (size_t)t * H;
    const float rstd = a.rstd[t];
    float g[V][8], xh[V][8], c = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      load8<BF16>((const char*)a.r + row * el, (v * W * 64 + l) * 8, H, xh[v]);
      load8<!DY32>((const char*)a.dy + row * del, (v * W * 64 + l) * 8, H, g[v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[v][j] *= rstd;
        dw[v][j] += g[v][j] * xh[v][j];
        g[v][j] *= w[v][j];
        c += g[v][j] * xh[v][j];
      }
    c = row_sum<W>(c, s_sum) / (float)H;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = (v * W * 64 + l) * 8;
      float d[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (a.dres) load8<BF16>((const char*)a.dres + row * el, i, H, d);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] += rstd * (g[v][j] - xh[v][j] * c);
      store8<BF16>((char*)a.dx + row * el, i, H, d);
    }
  }
  if (!a.dw_part) return;
  float* part = a.dw_part + (size_t)blockIdx.x * H;
  if constexpr (W == 1) {
    __shared__ float s_dw[V * 512];
    for (int q = 0; q < 4; ++q) {
      if (wave == q) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float& s = s_dw[(v * 8 + j) * 64 + l];
            s = q == 0 ? dw[v][j] : s + dw[v][j];
            if (q == 3) dw[v][j] = s;
          }
      }
      __syncthreads();
    }
    if (wave != 3) return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) store8<false>(part, (v * W * 64 + l) * 8, H, dw[v]);
}

// dw[h] = sum over the parts: 16 slices of them, eight loads in flight each, in order; then the slices in
// order. A block takes 64 columns (whole 256-byte lines of a part).
__global__ __launch_bounds__(1024) void rmsnorm_dw_kernel(const float* part, int parts, int H, float* dw) {
  __shared__ float s[16][64];
  const int c = threadIdx.x & 63, q = threadIdx.x >> 6, h = blockIdx.x * 64 + c;
  const int per = (parts + 15) / 16, p0 = min(parts, q * per), p1 = min(parts, p0 + per);
  float v = 0.f;
  if (h < H) {
    const float* src = part + h;
    int p = p0;
    for (; p + 8 <= p1; p += 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = src[(size_t)(p + i) * H];
#pragma unroll
      for (int i = 0; i < 8; ++i) v += x[i];
    }
    for (; p < p1; ++p) v += src[(size_t)p * H];
  }
  s[q][c] = v;
  __syncthreads();
  if (q == 0 && h < H) {
    for (int i = 1; i < 16; ++i) v += s[i][c];
    dw[h] = v;
  }
}

// f(W, V) for the smallest shape that holds a row of H values: W waves of V vectors of 8 per lane.
template <class F>
hipError_t by_row(int H, F&& f) {
  using std::integral_constant;
#define PMPE_ROW(w, v) return f(integral_constant<int, w>{}, integral_constant<int, v>{})
  if (H <= 512) PMPE_ROW(1, 1);
  if (H <= 1024) PMPE_ROW(2, 1);
  if (H <= 2048) PMPE_ROW(4, 1);
  if (H <= 4096) PMPE_ROW(8, 1);
  if (H <= 8192) PMPE_ROW(16, 1);
  PMPE_ROW(16, 2);
#undef PMPE_ROW
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s) {
  return by_row(a.H, [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value, RPB = W == 1 ? 4 : 1;
    const dim3 grid((a.T + RPB - 1) / RPB), block(W == 1 ? 256 : 64 * W);
    if (a.bf16)
      rmsnorm_kernel<true, W, V><<<grid, block, 0, s>>>(a);
    else
      rmsnorm_kernel<false, W, V><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
  });
}

// Blocks of the backward: four waves for each of a CU's SIMDs where rows are long enough. Fewer leave
// loads out of flight, more make parts to add: 16384 rows of 2048 67 us (512 blocks 87, 2048: 77), 4096
// rows 21.7 (21.5, 28.8).
int rmsnorm_bwd_parts(int T, int H) {
  const int waves = (H + 511) / 512;  // of a row, up to a power of two
  const int blocks = waves <= 1 ? 512 : waves <= 2 ? 1024 : waves <= 4 ? 1024 : waves <= 8 ? 512 : 256;
  return std::min((T + (waves <= 1 ? 3 : 0)) / (waves <= 1 ? 4 : 1), blocks);
}

hipError_t launch_rmsnorm_bwd(const NormBwdArgs& a, hipStream_t s) {
  const int parts = rmsnorm_bwd_parts(a.T, a.H);
  const hipError_t e = a.T == 0 ? hipSuccess : by_row(a.H, [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    const dim3 grid(parts), block(W == 1 ? 256 : 64 * W);
    if (a.bf16 && a.dy32)
      rmsnorm_bwd_kernel<true, true, W, V><<<grid, block, 0, s>>>(a);
    else if (a.bf16)
      rmsnorm_bwd_kernel<true, false, W, V><<<grid, block, 0, s>>>(a);
    else
      rmsnorm_bwd_kernel<false, true, W, V><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
  });
  if (e != hipSuccess || !a.dw) return e;
  rmsnorm_dw_kernel<<<(a.H + 63) / 64, 1024, 0, s>>>(a.dw_part, parts, a.H, a.dw);
  return hipGetLastError();
}

}  // namespace pmpe
