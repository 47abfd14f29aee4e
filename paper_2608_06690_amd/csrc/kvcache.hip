// The paged cache: rows of new tokens written into their requests' pages, as they are or in 8 bits, and
// cached rows read back.
//
//   write: position seq_len[r] - (tokens of r from this one on) of request r; q = e4m3(x 2^-e), e the block's
//   scale exponent (mx.h); read: x = q 2^e, exact in bf16
//
// A wave has one token at a time: its request is found once, then lane l takes values [8 l, 8 l + 8) of
// the token's heads, so a block of 32 values lies in 4 neighbouring lanes: its largest magnitude takes two exchanges
// and no LDS. One kernel serves both directions and k and v together, as a launch costs more than a small batch's rows.
//
// Bound by a wave's chain of loads up to its first row (request, position, page, tag), by HBM in large batches: 16417
// tokens of 4 heads of 128 written in 8 bits take 13.1 to 13.7 us for 51.0 MB (3.8 TB/s; a large copy's rate would give
// 9.8), 8289 read 9.3 to 9.9 us for 25.7 MB (2.7 TB/s; 5.0 at that rate). 8 tokens take 3.2 us, a launch; the call then
// costs 10 to 14 us of checks on the host.
#include "kvcache.h"
#include "mx.h"

namespace pmpe {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int KV_WAVES = 4;

// The request that token t belongs to, or -1.
__device__ __forceinline__ int request_of(const int32_t* offset, int R, int t) {
  if (t < R && offset[t] == t && offset[t + 1] == t + 1) return t;  // a decoding batch: a token each
  int lo = 0, hi = R;  // offset[lo] <= t, the last such in the end
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offset[mid] <= t) lo = mid;
    else hi = mid;
  }
  return offset[lo] <= t && t < offset[lo + 1] ? lo : -1;
}

// 8 values of a row to fp32 and back (bf16 or fp32 in memory, 16-byte aligned)
template <bool BF16>
__device__ __forceinline__ void load8(const void* row, int i, float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 q = *(const u32x4*)((const uint16_t*)row + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = bf16_to_f32(q[j] & 0xFFFFu);
      v[2 * j + 1] = bf16_to_f32(q[j] >> 16);
    }
  } else {
    const f32x4 a = *(const f32x4*)((const float*)row + i), b = *(const f32x4*)((const float*)row + i + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void copy8(void* to, const void* from) {
  *(u32x4*)to = *(const u32x4*)from;
  if constexpr (!BF16) *((u32x4*)to + 1) = *((const u32x4*)from + 1);
}

// WRITE: rows to cache, else cache to rows. BF16 activations or fp32; FP8: the cache is in 8 bits.
template <bool WRITE, bool BF16, bool FP8>
__global__ __launch_bounds__(64 * KV_WAVES) void kv_rows_kernel(KvRowsArgs a) {
  const CacheArgs& c = a.c;
  const int lane = lane_id(), t = __builtin_amdgcn_readfirstlane(blockIdx.x * KV_WAVES + (threadIdx.x >> 6));
  if (t >= a.T) return;
  const int r = request_of(a.offset, c.R, t);
  if (r < 0) return;
  const int64_t pos = WRITE ? (int64_t)a.at[r] - (a.offset[r + 1] - t) : (int64_t)(a.at ? a.at[r] : 0) + (t - a.offset[r]);
  const int64_t col = pos < 0 ? -1 : pos / c.page_size;
  uint32_t bad = 0;
  const int page = page_at(c, r, col, request_tag(c, r), bad);
  if (page < 0) {
    if (lane == 0) report(c, bad);
    if (WRITE) return;
  }
  const int row = page < 0 ? 0 : (int)(pos - col * c.page_size);
  const int n8 = c.kv * c.dim / 8, d8 = c.dim / 8;
  constexpr size_t EL = BF16 ? 2 : 4;
  for (int i = lane; i < n8; i += 64) {
    const int head = i / d8, d = (i - head * d8) * 8;
    const size_t hp = (size_t)(page < 0 ? 0 : page) * c.kv + head;
    const size_t at = (hp * c.page_size + row) * c.dim + d, sat = (hp * (c.dim / 32) + d / 32) * c.page_size + row;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      void* cache = kv ? c.v : c.k;
      uint8_t* scale = kv ? c.vs : c.ks;
      char* mine = (char*)(kv ? a.v : a.k) + ((size_t)t * (kv ? a.v_stride : a.k_stride) + (size_t)i * 8) * EL;
      if constexpr (!FP8) {
        char* there = (char*)cache + at * EL;
        if (WRITE) copy8<BF16>(there, mine);
        else if (page >= 0) copy8<BF16>(mine, there);
      } else if constexpr (WRITE) {
        float x[8];
        load8<BF16>(mine, 0, x);
        const float amax = mx_max_lanes<1, 2>(mx_amax8(x));
        uint32_t q0, q1;
        const int e = mx_pack8(x, amax, q0, q1);
        *(u32x2*)((uint8_t*)cache + at) = u32x2{q0, q1};
        if ((i & 3) == 0) scale[sat] = (uint8_t)(e + 127);
      } else if (page >= 0) {
        const u32x2 q = *(const u32x2*)((const uint8_t*)cache + at);
        const uint32_t e = scale[sat];
        // 2^(e - 127), also 2^-127; 255 is NaN
        const float s = __uint_as_float(e == 255 ? 0x7FC00000u : e ? e << 23 : 0x400000u);
        u32x4 o;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(q[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q[w], true);
          o[2 * w] = pack_bf16x2(lo[0] * s, lo[1] * s);
          o[2 * w + 1] = pack_bf16x2(hi[0] * s, hi[1] * s);
        }
        *(u32x4*)mine = o;
      }
      if (!WRITE && page < 0) {
        *(u32x4*)mine = u32x4{0, 0, 0, 0};
        if (!BF16) *((u32x4*)mine + 1) = u32x4{0, 0, 0, 0};
      }
    }
  }
}

template <bool WRITE>
hipError_t launch_rows(const KvRowsArgs& a, hipStream_t s) {
  const int grid = (a.T + KV_WAVES - 1) / KV_WAVES;
  if (a.c.fp8) kv_rows_kernel<WRITE, true, true><<<grid, 64 * KV_WAVES, 0, s>>>(a);
  else if (a.c.act_bf16) kv_rows_kernel<WRITE, true, false><<<grid, 64 * KV_WAVES, 0, s>>>(a);
  else kv_rows_kernel<WRITE, false, false><<<grid, 64 * KV_WAVES, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvRowsArgs& a, hipStream_t s) { return launch_rows<true>(a, s); }
hipError_t launch_kv_read(const KvRowsArgs& a, hipStream_t s) { return launch_rows<false>(a, s); }

}  // namespace pmpe
