// Attention of one new token per request over its paged cache.
//
//   s_j = scale q . k_j, out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), lse = m + ln sum_j exp(s_j - m)
//
// The query heads that share a kv head are the columns of 16 x 16 matrix products: a wave takes a tile of 32 rows of
// the cache, S^T = K Q^T (rows x heads), then O^T += V^T P^T (dims x heads), with a running maximum and sum per
// head. Operands come from memory straight into registers: lane l = (g, i) = (l / 16, l % 16) loads 16 bytes of
// row i for K (the order of dims inside a product is free, Q is laid out alike) and, for V, the dims of chunk i of
// rows 4 g .. 4 g + 3 and 16 + 4 g .. of the tile: the rows whose weights the lane holds after S^T, so weights go into
// the second product without leaving their lane, and V^T's pairs of rows are one byte permutation each.
//
// A block has a request's virtual head (a kv head and up to 16 of its query heads), its four waves every fourth tile.
// Where tables are long, a head's tiles are cut into equal parts of a length that all requests share, found from
// their lengths by every block: 32 tiles, fewer (8 at least) where CUs would be left without a part, more where there
// would be over PARTS parts and one for each head. A second kernel joins the parts in order. No atomics: equal calls
// have equal bits.
//
// Bound by HBM, and by the pattern in which it is read: 256 requests of up to 8149 rows (4047 in the mean) over 4 kv heads of
// 128 in 8 bits (1.1 GB) take 205 us, 5.4 TB/s; 64 of 8000 rows over 8 kv heads of 128 in bf16 (2.1 GB) 323 us, 6.5 TB/s. A K
// operand of 8-bit rows is 64 bytes at a time, half a line, and scales are lines of their own; plain reads of whole
// lines reach 6.6 to 7.1 TB/s, of half lines 5.7 to 6.0. Single requests over 4 kv heads are bound by latency: 700 rows 10.6
// us, 131,000 rows 43 us in 512 parts and 11 us to join them. Loads are never under a branch (a row that may not
// be used is read from page 0 and dropped): with branches each step waited for all loads of the one before it.
#include <algorithm>

#include "kvcache.h"

namespace pmpe {
namespace {

constexpr int WAVES = 4;
constexpr int TILE = 32;        // cache rows of a wave's step
constexpr int PARTS = 1536;       // parts of all tiles at most, but for one of each head: two rounds of the blocks that fit the card
constexpr int WHOLE_TILES = 32;   // tables of at most so many tiles: no head is cut (8 steps, about as long as the search and the join)
constexpr int MOST_HEADS = 8192;  // virtual heads from which none is cut
constexpr int MOST_BLOCKS = 1 << 22;  // of a launch: 2^30 threads (2^32 are more than one can have)
constexpr float LOG2E = 1.4426950408889634f;

enum { BF16 = 0, FP8 = 1, F32 = 2 };

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
// What is read once: past the caches.
template <class V>
__device__ __forceinline__ V once(const V* p) {
  return __builtin_nontemporal_load(p);
}
// max and sum over lanes l, l ^ 16, l ^ 32 and l ^ 48
__device__ __forceinline__ float rows_max(float v) {
  uint32_t u = __float_as_uint(v);
  auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
  s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
  uint32_t u = __float_as_uint(v);
  auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(__uint_as_float(s[0]) + __uint_as_float(s[1]));
  s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
// Two e4m3 values (the word's lower or upper half) times a power of two, to bf16: exact. The instruction takes the
// exponent field of its scale as the biased exponent, 255 being NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }
template <bool HI>
__device__ __forceinline__ uint32_t fp8_to_bf16x2(uint32_t q, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, s, HI));
}

struct Split {
  int groups, rows, vheads;  // parts of a kv head's query heads, heads of a part, virtual heads of a request
};
__host__ __device__ inline Split split_of(int heads, int kv) {
  const int g = heads / kv, parts = (g + 15) / 16;
  return {parts, (g + parts - 1) / parts, kv * parts};
}
// Rows of a request: [first, end), its tiles.
struct Rows {
  int first, end, t0, n;
};
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, int r) {
  const int most = a.c.max_pages * a.c.page_size, first = a.first ? max(0, a.first[r]) : 0, end = min(a.len[r], most);
  if (end <= first) return {first, end, 0, 0};
  return {first, end, first / TILE, (end + TILE - 1) / TILE - first / TILE};
}

// Waves of a SIMD that the registers of a wave leave room for.
__host__ __device__ constexpr int waves_per_simd(int type, int nb) {
  return type == F32 ? (nb <= 1 ? 4 : nb == 2 ? 3 : nb == 3 ? 2 : 1) : nb <= 2 ? 4 : nb <= 4 ? 3 : nb <= 6 ? 2 : 1;
}

// The same of a request that the whole wave has, in scalar registers.
__device__ __forceinline__ Rows uniform_rows_of(const AttnArgs& a, int r) {
  const Rows v = rows_of(a, r);
  return {__builtin_amdgcn_readfirstlane(v.first), __builtin_amdgcn_readfirstlane(v.end), __builtin_amdgcn_readfirstlane(v.t0),
          __builtin_amdgcn_readfirstlane(v.n)};
}

// Workspace: the parts of heads that are cut, in places side by side. At most SLOTS: a head of n > c tiles has
// ceil(n / c) < 2 n / c of them.
constexpr int SLOTS = 2 * PARTS;
struct Part {
  float* o;       // [SLOTS][rows][dim]
  float* ml;      // [SLOTS][rows][2]
  int32_t* what;  // [SLOTS][4]: request, virtual head and parts of the head that begins in a place (0 parts: none does)
  int32_t* used;  // places in use
};
__host__ __device__ inline Part part_of(float* ws, int rows, int dim) {
  float* ml = ws + (size_t)SLOTS * rows * dim;
  int32_t* what = (int32_t*)(ml + (size_t)SLOTS * rows * 2);
  return {ws, ml, what, what + SLOTS * 4};
}

template <int T, int NB>
struct Tile {
  static constexpr int D = 32 * NB;
  static constexpr int NK = T == BF16 ? NB : T == FP8 ? (NB + 1) / 2 : 2 * NB;  // 16-byte loads of a K row's quarter
  static constexpr int SEGS = NB / 4 + ((NB & 2) != 0) + (NB & 1);            // V: 128, 64 and 32 dims
  static constexpr int VW = T == BF16 ? D / 32 : T == FP8 ? (D + 63) / 64 : D / 16;  // words of V per row and lane
  u32x4 k[2][NK];
  uint32_t ks[2][T == FP8 ? NK : 1];
  uint32_t v[8][VW];
  uint32_t vs[2][T == FP8 ? SEGS : 1];
};
// base dim and width of segment j
template <int NB>
__device__ constexpr int seg_base(int j) {
  return j <= NB / 4 ? (j < NB / 4 ? 128 * j : 128 * (NB / 4)) : 128 * (NB / 4) + 64 * ((NB & 2) != 0);
}
template <int NB>
__device__ constexpr int seg_width(int j) {
  return j < NB / 4 ? 128 : (NB & 2) && j == NB / 4 ? 64 : 32;
}

template <int T, int NB, bool SPLIT_ROWS>
struct Wave {
  static constexpr int D = 32 * NB, EL = T == BF16 ? 2 : T == FP8 ? 1 : 4;
  typedef Tile<T, NB> TileT;
  const AttnArgs& a;
  const int lane, i, g;
  int r, h;             // request, kv head
  Rows rows;
  TileT t;
  u32x4 q[T == F32 ? 2 * NB : NB];
  f32x4 o[2 * NB];
  float m, l;
  int pages, prow;      // lane 2 n + u: page and row of half u of the wave's n-th tile from `from` on
  int from;             // index of a tile (in steps of the wave)
  uint32_t bad;

  __device__ Wave(const AttnArgs& args) : a(args), lane(lane_id()), i(lane & 15), g(lane >> 4), bad(0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int s = 0; s < TileT::NK; ++s) t.k[u][s] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < (T == FP8 ? TileT::NK : 1); ++s) t.ks[u][s] = 0;
#pragma unroll
      for (int s = 0; s < (T == FP8 ? TileT::SEGS : 1); ++s) t.vs[u][s] = 0;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < TileT::VW; ++w) t.v[j][w] = 0;
  }

  // Q of the virtual head: column i is query head h0 + (i, or i % 8: its copy for the weights' lower parts).
  __device__ void begin(int request, int kv_head, int head0, int n_heads) {
    r = request;
    h = kv_head;
    rows = uniform_rows_of(a, r);
    if (rows.end < a.len[r]) bad |= PMPE_DEV_CACHE_RANGE;
    const int col = SPLIT_ROWS ? i & 7 : i;
    const char* at = (const char*)a.q + ((size_t)r * a.q_stride + (size_t)(head0 + col) * D) * (T == F32 ? 4 : 2);
#pragma unroll
    for (int s = 0; s < (T == F32 ? 2 * NB : NB); ++s) {
      int d;
      if (T == BF16) d = s * 32 + g * 8;
      else if (T == F32) d = s * 16 + g * 4;
      else d = (NB & 1) && s == NB - 1 ? s * 32 + g * 8 : (s / 2) * 64 + g * 16 + (s & 1) * 8;
      q[s] = col < n_heads ? *(const u32x4*)(at + (size_t)d * (T == F32 ? 4 : 2)) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) o[j] = f32x4{0, 0, 0, 0};
    m = -INFINITY;
    l = 0.f;
  }

  // Pages of the wave's tiles first_tile + 4 n, n = 0 .. 31.
  __device__ void look_up(int first_tile) {
    const CacheArgs& c = a.c;
    const int p = (first_tile + WAVES * (lane >> 1)) * TILE + (lane & 1) * 16;
    pages = -1;
    prow = 0;
    if (p < rows.end && p + 16 > rows.first) {
      const int col = p / c.page_size;
      pages = page_at(c, r, col, request_tag(c, r), bad);
      prow = p - col * c.page_size;
    }
  }

  // (Rows that take no part are those of page 0: the loads are the same for every tile, so that their order is known
  // where the next ones are waited for. With branches around them every step waited for all of them.)
  __device__ const char* half(const void* cache, int n, int u, int page) const {
    const CacheArgs& c = a.c;
    return (const char*)cache + (((size_t)max(page, 0) * c.kv + h) * c.page_size + __builtin_amdgcn_readlane(prow, 2 * n + u)) * (D * EL);
  }
  __device__ const uint8_t* scales(const uint8_t* s, int n, int u, int page) const {
    const CacheArgs& c = a.c;
    return s + ((size_t)max(page, 0) * c.kv + h) * NB * c.page_size + __builtin_amdgcn_readlane(prow, 2 * n + u);
  }
  __device__ void load_k(int n) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * n + u);
      const char* at = half(a.c.k, n, u, page);
      const uint32_t off = i * (D * EL) + g * 16;
#pragma unroll
      for (int s = 0; s < TileT::NK; ++s) {
        if (T == FP8 && (NB & 1) && s == TileT::NK - 1) {
          const u32x2 x = *((const u32x2*)(at + (i * (D * EL) + g * 8 + s * 64)));
          t.k[u][s][0] = x[0];
          t.k[u][s][1] = x[1];
        } else {
          t.k[u][s] = *((const u32x4*)(at + (off + s * 64)));
        }
      }
      if constexpr (T == FP8) {
        const uint8_t* sc = scales(a.c.ks, n, u, page);
#pragma unroll
        for (int s = 0; s < TileT::NK; ++s)
          t.ks[u][s] = sc[((NB & 1) && s == TileT::NK - 1 ? 2 * s : 2 * s + (g >> 1)) * a.c.page_size + i];
      }
    }
  }
  __device__ void load_v(int n) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * n + u);
      const char* at = half(a.c.v, n, u, page);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        int w = 0;
#pragma unroll
        for (int sg = 0; sg < TileT::SEGS; ++sg) {
          const int width = seg_width<NB>(sg), per = width / 16 * EL;  // bytes of a lane
          const char* p = at + ((uint32_t)((g * 4 + j) * (D * EL) + i * per) + seg_base<NB>(sg) * EL);
          uint32_t* to = t.v[4 * u + j] + w;
          if (per == 32) {
            const u32x4 x = once((const u32x4*)p), y = once((const u32x4*)(p + 16));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              to[e] = x[e];
              to[4 + e] = y[e];
            }
          } else if (per == 16) {
            const u32x4 x = once((const u32x4*)p);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] = x[e];
          } else if (per == 8) {
            const u32x2 x = once((const u32x2*)p);
            to[0] = x[0];
            to[1] = x[1];
          } else if (per == 4) {
            to[0] = once((const uint32_t*)p);
          } else {
            to[0] = once((const uint16_t*)p);
          }
          w += (per + 3) / 4;
        }
      }
      if constexpr (T == FP8) {
        const uint8_t* sc = scales(a.c.vs, n, u, page);
#pragma unroll
        for (int sg = 0; sg < TileT::SEGS; ++sg) {
          const int width = seg_width<NB>(sg);
          const int blk = seg_base<NB>(sg) / 32 + (width == 128 ? i >> 2 : width == 64 ? i >> 3 : 0);
          t.vs[u][sg] = *(const uint32_t*)(sc + (uint32_t)(blk * a.c.page_size + g * 4));
        }
      }
    }
  }

  // S^T of half u: lane (g, i) gets rows 4 g .. 4 g + 3 of column i
  __device__ f32x4 scores(int u) const {
    f32x4 s = {0, 0, 0, 0};
    if constexpr (T == BF16) {
#pragma unroll
      for (int j = 0; j < NB; ++j) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(t.k[u][j]), as_bf16x8(q[j]), s, 0, 0, 0);
    } else if constexpr (T == FP8) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float f = scale_of(t.ks[u][j / 2]);
        const uint32_t x = t.k[u][j / 2][(j & 1) * 2], y = t.k[u][j / 2][(j & 1) * 2 + 1];
        const u32x4 k = {fp8_to_bf16x2<false>(x, f), fp8_to_bf16x2<true>(x, f), fp8_to_bf16x2<false>(y, f), fp8_to_bf16x2<true>(y, f)};
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k), as_bf16x8(q[j]), s, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[u][j][e]), __uint_as_float(q[j][e]), s, 0, 0, 0);
    }
    return s;
  }

  // O^T += V^T P^T with weights p[u][e] of row 16 u + 4 g + e
  __device__ void accumulate(const float (&p)[8]) {
    if constexpr (T == F32) {
      int w = 0, n = 0;
#pragma unroll
      for (int sg = 0; sg < TileT::SEGS; ++sg) {
        const int per = seg_width<NB>(sg) / 16;
#pragma unroll
        for (int d = 0; d < per; ++d, ++n)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[j][w + d]), p[j], o[n], 0, 0, 0);
        w += per;
      }
    } else {
      // A weight as the sum of three bf16 values, which leaves 2^-27 of it (two leave 2^-18, and four times as many
      // outputs rounded to the other side as fp32 weights do). With up to 8 heads the second parts are columns 8 .. 15 of
      // the first parts' product. The third takes 2 to 7 % of a single request of up to 1000 rows, nothing of long ones.
      u32x4 hi, lo, rest;
      float x[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = p[j] - (float)(__bf16)p[j];
        y[j] = x[j] - (float)(__bf16)x[j];
      }
      if constexpr (SPLIT_ROWS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = i < 8 ? p[j] : x[j];
          y[j] = i < 8 ? y[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) hi[j] = pk_bf16(x[2 * j], x[2 * j + 1]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          hi[j] = pk_bf16(p[2 * j], p[2 * j + 1]);
          lo[j] = pk_bf16(x[2 * j], x[2 * j + 1]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) rest[j] = pk_bf16(y[2 * j], y[2 * j + 1]);
      int w = 0, n = 0;
#pragma unroll
      for (int sg = 0; sg < TileT::SEGS; ++sg) {
        const int pairs = seg_width<NB>(sg) / 32;  // pairs of dims of a lane
        float f[8];
        if constexpr (T == FP8) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = scale_of((t.vs[j >> 2][sg] >> (8 * (j & 3))) & 0xFFu);
        }
#pragma unroll
        for (int e = 0; e < pairs; ++e) {
          uint32_t v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if constexpr (T == BF16) v[j] = t.v[j][w + e];
            else v[j] = e & 1 ? fp8_to_bf16x2<true>(t.v[j][w + e / 2], f[j]) : fp8_to_bf16x2<false>(t.v[j][w + e / 2], f[j]);
          }
#pragma unroll
          for (int odd = 0; odd < 2; ++odd, ++n) {
            u32x4 vt;
#pragma unroll
            for (int j = 0; j < 4; ++j) vt[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], odd ? 0x07060302u : 0x05040100u);
            o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt), as_bf16x8(hi), o[n], 0, 0, 0);
            if constexpr (!SPLIT_ROWS) o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt), as_bf16x8(lo), o[n], 0, 0, 0);
            o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt), as_bf16x8(rest), o[n], 0, 0, 0);
          }
        }
        w += T == BF16 ? pairs : (pairs + 1) / 2;
      }
    }
  }

  // Tile `tile` (the n-th looked up), whose K and V are loaded; with MORE, loads those of tile n + 1.
  template <bool MORE>
  __device__ void step(int tile, int n) {
    float s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 x = scores(u);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * u + e] = x[e] * (a.scale * LOG2E);
    }
    const int p0 = tile * TILE, pg0 = __builtin_amdgcn_readlane(pages, 2 * n), pg1 = __builtin_amdgcn_readlane(pages, 2 * n + 1);
    if constexpr (MORE) load_k(n + 1);
    const bool whole = pg0 >= 0 && pg1 >= 0 && p0 >= rows.first && p0 + TILE <= rows.end;
    if (!whole) {
      // rows that take no part: their weights are 0, and so is V there (0 times what memory holds may be NaN)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int p = p0 + (j >> 2) * 16 + g * 4 + (j & 3);
        const bool in = (j < 4 ? pg0 : pg1) >= 0 && p >= rows.first && p < rows.end;
        s[j] = in ? s[j] : -INFINITY;
#pragma unroll
        for (int w = 0; w < TileT::VW; ++w) t.v[j][w] = in ? t.v[j][w] : 0u;
        if constexpr (T == FP8) {
#pragma unroll
          for (int sg = 0; sg < TileT::SEGS; ++sg)
            t.vs[j >> 2][sg] = in ? t.vs[j >> 2][sg] : t.vs[j >> 2][sg] & ~(0xFFu << (8 * (j & 3)));
        }
      }
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
    top = rows_max(top);
    if (__any(top > m)) {
      const float mn = fmaxf(m, top), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(s[j] - ref);
    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    accumulate(p);
    if constexpr (MORE) load_v(n + 1);
  }

  // Tiles first, first + 4, .. below last.
  __device__ void run(int first, int last) {
    for (int tile = first; tile < last;) {
      look_up(tile);
      load_k(0);
      load_v(0);
      int n = 0;
      for (; n < 31 && tile + WAVES < last; ++n, tile += WAVES) step<true>(tile, n);
      step<false>(tile, n);
      tile += WAVES;
    }
    l = rows_sum(l);
    if constexpr (SPLIT_ROWS && T != F32) {
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] += __uint_as_float(xor_lanes(__float_as_uint(o[j][e]), 8));
    }
  }
};

template <int NB>
struct Lds {
  float ml[WAVES][16][2];
  float o[WAVES][16][32 * NB + 4];
};

// The waves' parts of a virtual head joined: the output if `whole`, else the piece's part.
template <int T, int NB, bool SPLIT_ROWS>
__device__ void finish(Wave<T, NB, SPLIT_ROWS>& w, Lds<NB>& lds, int head0, int n_heads, bool whole, const Part& part, int slot, int slot_rows) {
  constexpr int D = 32 * NB;
  const AttnArgs& a = w.a;
  const int wave = threadIdx.x >> 6;
  if (w.g == 0) {
    lds.ml[wave][w.i][0] = w.m;
    lds.ml[wave][w.i][1] = w.l;
  }
  __syncthreads();
  float M = -INFINITY;
#pragma unroll
  for (int j = 0; j < WAVES; ++j) M = fmaxf(M, lds.ml[j][w.i][0]);
  const float f = w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m - M);
  if (w.i < n_heads) {
    float* to = lds.o[wave][w.i];
    int n = 0;
#pragma unroll
    for (int sg = 0; sg < Tile<T, NB>::SEGS; ++sg) {
      const int per = seg_width<NB>(sg) / 16;
#pragma unroll
      for (int d = 0; d < per; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[seg_base<NB>(sg) + (w.g * 4 + e) * per + d] = w.o[n + d][e] * f;
      n += per;
    }
  }
  __syncthreads();
  for (int x = threadIdx.x * 4; x < n_heads * D; x += 4 * 64 * WAVES) {
    const int head = x / D, d = x % D;
    float L = 0.f, Mh = -INFINITY;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < WAVES; ++j) Mh = fmaxf(Mh, lds.ml[j][head][0]);
#pragma unroll
    for (int j = 0; j < WAVES; ++j) {
      const float mj = lds.ml[j][head][0];
      L += lds.ml[j][head][1] * (mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj - Mh));
      v += *(const f32x4*)&lds.o[j][head][d];
    }
    if (whole) {
      const size_t at = ((size_t)w.r * a.heads + head0 + head) * D + d;
      const float inv = L == 0.f ? 0.f : 1.f / L;
      v = L == 0.f ? f32x4{0, 0, 0, 0} : v * inv;
      if (T == F32) *(f32x4*)((float*)a.out + at) = v;
      else *(u32x2*)((uint16_t*)a.out + at) = u32x2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
      if (a.lse && d == 0) a.lse[(size_t)w.r * a.heads + head0 + head] = L == 0.f ? -INFINITY : (Mh + log2f(L)) * 0.6931471805599453f;
    } else {
      *(f32x4*)(part.o + ((size_t)slot * slot_rows + head) * D + d) = v;
      if (d == 0) {
        part.ml[((size_t)slot * slot_rows + head) * 2] = Mh;
        part.ml[((size_t)slot * slot_rows + head) * 2 + 1] = L;
      }
    }
  }
}

// Inclusive sums over the block's threads, and the total.
__device__ __forceinline__ int scan_block(int v, int* s, int& total) {
  const int wave = threadIdx.x >> 6;
  v = wave_incl_scan(v);
  __syncthreads();
  if (lane_id() == 63) s[wave] = v;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int j = 0; j < WAVES; ++j) {
    if (j < wave) v += s[j];
    total += s[j];
  }
  return v;
}

// DIRECT: no head is cut.
template <int T, int NB, bool SPLIT_ROWS, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, waves_per_simd(T, NB)) void attn_kernel(AttnArgs a) {
  __shared__ Lds<NB> lds;
  __shared__ int64_t s_tiles[WAVES];
  __shared__ int s_scan[WAVES], s_item[4];
  const Split sp = split_of(a.heads, a.c.kv);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  int r, vh, part = 0, parts = 1, slot = 0;
  if constexpr (DIRECT) {
    r = blockIdx.x / sp.vheads;
    vh = blockIdx.x - r * sp.vheads;
  } else {
    // The length of a part; then the heads' parts ahead of this block's and, of them, those of heads that are cut.
    // Thread x has requests [x c, (x + 1) c).
    const int c = (a.c.R + 64 * WAVES - 1) / (64 * WAVES), r0 = threadIdx.x * c, r1 = min(a.c.R, r0 + c);
    int64_t tiles = 0;
    for (int q = r0; q < r1; ++q) tiles += rows_of(a, q).n;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) tiles += __shfl_xor(tiles, off, 64);
    if (lane == 0) s_tiles[wave] = tiles;
    __syncthreads();
    tiles = 0;
#pragma unroll
    for (int j = 0; j < WAVES; ++j) tiles += s_tiles[j];
    tiles *= sp.vheads;
    // At least 32 tiles, or 8 where that leaves CUs without a part; a head of up to one and a half parts stays whole.
    const int len = (int)max((tiles + PARTS - 1) / PARTS, min((int64_t)32, max((int64_t)8, (tiles + 255) / 256)));
    const int whole = len + len / 2;
    const auto parts_of = [&](int q) {
      const int n = rows_of(a, q).n;
      return n <= whole ? 1 : (n + len - 1) / len;
    };
    int mine = 0, cut = 0, total, used;
    for (int q = r0; q < r1; ++q) {
      const int k = parts_of(q);
      mine += k;
      cut += k > 1 ? k : 0;
    }
    const int upto = scan_block(mine, s_scan, total), cut_upto = scan_block(cut, s_scan, used);
    const Part p = part_of(a.ws, sp.rows, 32 * NB);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.used = used * sp.vheads;
    if ((int)blockIdx.x >= total * sp.vheads) return;
    if ((upto - mine) * sp.vheads <= (int)blockIdx.x && (int)blockIdx.x < upto * sp.vheads) {  // one thread
      int base = upto - mine, cuts = cut_upto - cut, q = r0, k;
      for (k = parts_of(q); (base + k) * sp.vheads <= (int)blockIdx.x; k = parts_of(q)) {
        base += k;
        cuts += k > 1 ? k : 0;
        ++q;
      }
      s_item[0] = q;
      s_item[1] = blockIdx.x - base * sp.vheads;  // virtual head and part
      s_item[2] = k;
      s_item[3] = cuts * sp.vheads;
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane(s_item[0]);
    parts = __builtin_amdgcn_readfirstlane(s_item[2]);
    const int x = __builtin_amdgcn_readfirstlane(s_item[1]);
    vh = x / parts;
    part = x - vh * parts;
    slot = __builtin_amdgcn_readfirstlane(s_item[3]) + x;
    if (parts > 1 && threadIdx.x == 0) {
      p.what[4 * slot] = r;
      p.what[4 * slot + 1] = vh;
      p.what[4 * slot + 2] = part == 0 ? parts : 0;
    }
  }
  const int kv = vh / sp.groups, in_kv = (vh - kv * sp.groups) * sp.rows, group = a.heads / a.c.kv;
  const int head0 = kv * group + in_kv, n_heads = min(sp.rows, group - in_kv);
  Wave<T, NB, SPLIT_ROWS> w(a);
  w.begin(r, kv, head0, n_heads);
  const int first = (int)((int64_t)w.rows.n * part / parts), last = (int)((int64_t)w.rows.n * (part + 1) / parts);
  w.run(w.rows.t0 + first + wave, w.rows.t0 + last);
  finish<T, NB, SPLIT_ROWS>(w, lds, head0, n_heads, parts == 1, part_of(a.ws, sp.rows, 32 * NB), slot, sp.rows);
  report(a.c, w.bad);
}

// One query head of a head that was cut: its parts, in order. It has W waves of the block: one where heads are many
// and their parts few, all four where it is the other way round.
template <bool BF16_OUT, int W>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  __shared__ float s_o[W == 1 ? 1 : 256][4], s_red[8];
  const Split sp = split_of(a.heads, a.c.kv);
  const int lane = lane_id(), wave = threadIdx.x >> 6, D = a.c.dim;
  const int x = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x, s0 = x / sp.rows, row = x - s0 * sp.rows;
  const Part part = part_of(a.ws, sp.rows, D);
  if (s0 >= *part.used) return;
  const int r = part.what[4 * s0], vh = part.what[4 * s0 + 1], n = part.what[4 * s0 + 2];
  if (n == 0) return;
  const int group = a.heads / a.c.kv, kv = vh / sp.groups, in_kv = (vh - kv * sp.groups) * sp.rows + row;
  if (in_kv >= group) return;
  const auto slot = [&](int i) { return (size_t)(s0 + i) * sp.rows + row; };
  const int tid = W == 1 ? lane : threadIdx.x, per = D / 4, lanes = 64 * W / per, mine = tid / per, d = (tid - mine * per) * 4;
  // the first parts are under way while their weights are worked out
  f32x4 v0 = {0, 0, 0, 0}, v1 = {0, 0, 0, 0};
  if (mine < lanes && mine < n) v0 = *(const f32x4*)(part.o + slot(mine) * D + d);
  if (mine < lanes && mine + lanes < n) v1 = *(const f32x4*)(part.o + slot(mine + lanes) * D + d);
  float M = -INFINITY, L = 0.f;
  for (int i = tid; i < n; i += 64 * W) M = fmaxf(M, part.ml[slot(i) * 2]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __uint_as_float(xor_lanes(__float_as_uint(M), off)));
  if constexpr (W > 1) {
    if (lane == 0) s_red[wave] = M;
    __syncthreads();
    M = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  }
  const auto weight = [&](int i) {
    const float m = part.ml[slot(i) * 2];
    return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  };
  for (int i = tid; i < n; i += 64 * W) L += part.ml[slot(i) * 2 + 1] * weight(i);
  L = wave_sum(L);
  f32x4 v = {0, 0, 0, 0};
  if (mine < lanes) {
    if (mine < n) v = v0 * weight(mine);
    if (mine + lanes < n) v += v1 * weight(mine + lanes);
#pragma unroll 4
    for (int i = mine + 2 * lanes; i < n; i += lanes) v += *(const f32x4*)(part.o + slot(i) * D + d) * weight(i);
  }
  if constexpr (W > 1) {
    if (lane == 0) s_red[4 + wave] = L;
    *(f32x4*)s_o[tid] = v;
    __syncthreads();
    L = (s_red[4] + s_red[5]) + (s_red[6] + s_red[7]);
    if (mine > 0) return;
    for (int j = 1; j < lanes; ++j) v += *(const f32x4*)s_o[j * per + tid];
  } else {
    const f32x4 own = v;
    for (int j = 1; j < lanes; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += __shfl(own[e], (lane + j * per) & 63, 64);
    if (mine > 0) return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  v = L == 0.f ? f32x4{0, 0, 0, 0} : v * inv;
  const size_t at = (size_t)r * a.heads + kv * group + in_kv;
  if (BF16_OUT) *(u32x2*)((uint16_t*)a.out + at * D + d) = u32x2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
  else *(f32x4*)((float*)a.out + at * D + d) = v;
  if (tid == 0 && a.lse) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// No head is cut where tables hold no more than an uncut one, or where heads are many anyway.
bool direct(int64_t vheads, int max_pages, int page_size) {
  return (int64_t)max_pages * page_size <= WHOLE_TILES * TILE || vheads >= MOST_HEADS;
}

// Requests [r0, r0 + n) of a call whose heads are not cut.
AttnArgs part_of_call(const AttnArgs& a, int r0, int n) {
  const size_t el = a.c.act_bf16 ? 2 : 4, row = (size_t)a.heads * a.c.dim;
  AttnArgs p = a;
  p.c.R = n;
  p.c.table += (size_t)r0 * a.c.max_pages;
  if (a.c.words) p.c.words += r0;
  p.q = (const char*)a.q + (size_t)r0 * a.q_stride * el;
  if (a.first) p.first += r0;
  p.len += r0;
  p.out = (char*)a.out + r0 * row * el;
  if (a.lse) p.lse += (size_t)r0 * a.heads;
  return p;
}

template <int T, int NB>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
  const Split sp = split_of(a.heads, a.c.kv);
  const int64_t vheads = (int64_t)a.c.R * sp.vheads, rows = (int64_t)a.c.max_pages * a.c.page_size;
  if (direct(vheads, a.c.max_pages, a.c.page_size)) {
    // (more than the threads that one launch may have: so many requests at a time)
    const int most = MOST_BLOCKS / sp.vheads;
    for (int r0 = 0; r0 < a.c.R; r0 += most) {
      const AttnArgs p = part_of_call(a, r0, std::min(most, a.c.R - r0));
      if (sp.rows <= 8) attn_kernel<T, NB, true, true><<<p.c.R * sp.vheads, 64 * WAVES, 0, s>>>(p);
      else attn_kernel<T, NB, false, true><<<p.c.R * sp.vheads, 64 * WAVES, 0, s>>>(p);
    }
    return hipGetLastError();
  }
  const int grid = (int)vheads + PARTS;
  if (sp.rows <= 8) attn_kernel<T, NB, true, false><<<grid, 64 * WAVES, 0, s>>>(a);
  else attn_kernel<T, NB, false, false><<<grid, 64 * WAVES, 0, s>>>(a);
  // places that can be in use
  const int slots = (int)std::min<int64_t>(SLOTS, vheads * ((rows + 8 * TILE - 1) / (8 * TILE) + 1));
  if (vheads > 64) attn_join_kernel<T != F32, 1><<<(slots * sp.rows + 3) / 4, 256, 0, s>>>(a);
  else attn_join_kernel<T != F32, 4><<<slots * sp.rows, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int T>
hipError_t launch_type(const AttnArgs& a, hipStream_t s) {
  switch (a.c.dim / 32) {
    case 1: return launch<T, 1>(a, s);
    case 2: return launch<T, 2>(a, s);
    case 3: return launch<T, 3>(a, s);
    case 4: return launch<T, 4>(a, s);
    case 5: return launch<T, 5>(a, s);
    case 6: return launch<T, 6>(a, s);
    case 7: return launch<T, 7>(a, s);
    default: return launch<T, 8>(a, s);
  }
}

}  // namespace

size_t attn_decode_workspace(int R, int heads, const pmpe_cache_desc* c) {
  const Split sp = split_of(heads, c->n_kv_heads);
  if (R == 0 || direct((int64_t)R * sp.vheads, c->max_pages, c->page_size)) return 0;
  return ((size_t)SLOTS * (sp.rows * (c->head_dim + 2) + 4) + 4) * 4;
}

hipError_t launch_attn_decode(const AttnArgs& a, hipStream_t s) {
  if (a.c.fp8) return launch_type<FP8>(a, s);
  return a.c.act_bf16 ? launch_type<BF16>(a, s) : launch_type<F32>(a, s);
}

}  // namespace pmpe
