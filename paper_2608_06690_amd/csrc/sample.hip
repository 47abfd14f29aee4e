// One token per row of logits: temperature, top-k, top-p, min-p, and a draw by a given uniform number.
//
// The order of a row is (logit descending, id ascending); every cut leaves a leading part of it, and the
// draw is its first token whose cumulated mass exceeds u times the whole. Each of them is "the first place where
// the count, or the mass, up to it crosses a threshold".
//
// Two kernels. The first goes over the logits once, in pieces of a row that its blocks hold in registers:
// the piece's maximum, the maxima of its chunks of 512, and a histogram by x = z / temperature in bins of 1/8 (512
// of them from the maximum down: what lies lower has less than e^-64 of its mass) of counts and masses. The second
// has a block per row: it adds up the histograms, finds the bins of the thresholds, and collects the tokens down to
// the last bin that matters, from chunks that hold one. They are sorted, and everything is decided on the list.
// Where they are more than a list (ties, flat rows without a cut) it looks into one bin at a time, by
// histograms of the logits' bits in it.
//
// Masses are exact integers inside a bin (units of 2^-44 of the mass at its centre), so their sums do not depend on
// the order of the atomics; across bins they are fp64 in a fixed order.
#include <cfloat>

#include "exp64.h"
#include "pmpe_internal.h"

namespace pmpe {
namespace {

constexpr int BINS = 512;
constexpr int CHUNK = 512;      // logits that a wave loads at once, 8 a lane
constexpr int HIST_THREADS = 512;
constexpr int PIECE8 = HIST_THREADS * 8;
constexpr int THREADS = 1024;   // of the second kernel
constexpr int CAP = 2 * THREADS;  // tokens of a list
constexpr int MAX_CHUNKS = PMPE_MAX_VOCAB / CHUNK;
// rows whose top_k is at most this are counted only: their list has the masses
constexpr int COUNT_K = CAP / 2;

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float z_of(uint32_t k) { return __uint_as_float((k >> 31) ? k ^ 0x80000000u : ~k); }
// A logit as it counts: masked ones (also NaN) -inf, +inf the largest finite value, -0 as 0.
__device__ __forceinline__ float canon(float v) { return v > -INFINITY ? fminf(v, FLT_MAX) + 0.f : -INFINITY; }

// Logits [i, i + 8) of a row of n (past it: -inf).
template <bool BF16>
__device__ __forceinline__ void load8(const void* row, int i, int n, float (&v)[8]) {
  if (i + 8 <= n) {
    if constexpr (BF16) {
      const u32x4 q = *(const u32x4_a2*)((const uint16_t*)row + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = bf16_to_f32(q[j] & 0xFFFFu);
        v[2 * j + 1] = __uint_as_float(q[j] & 0xFFFF0000u);
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
      v[j] = -INFINITY;
      if (i + j < n) v[j] = BF16 ? bf16_to_f32(((const uint16_t*)row)[i + j]) : ((const float*)row)[i + j];
    }
  }
}

// Pieces of a row and the workspace: for each row its pieces' heads, the chunks' maxima, the pieces' histograms.
struct Layout {
  int pieces, g8, chunks;  // pieces of g8 * PIECE8 logits
  size_t row;              // bytes
  size_t max_at, mass_at, count_at;
};
struct Head {
  float top;        // the piece's largest logit
  uint32_t first;   // where it is first
  uint32_t live;    // tokens that are not masked
  uint32_t used;    // bins down to the last one that is not empty
};
// The largest pieces (less of the histograms' bytes) of which there are two for each CU.
__host__ __device__ inline Layout layout_of(int B, int V) {
  Layout l{};
  l.g8 = 8;
  while (l.g8 > 1 && l.g8 / 2 * PIECE8 >= V) l.g8 /= 2;
  while (l.g8 > 1 && (int64_t)B * ((V + l.g8 * PIECE8 - 1) / (l.g8 * PIECE8)) < 512) l.g8 /= 2;
  l.pieces = (V + l.g8 * PIECE8 - 1) / (l.g8 * PIECE8);
  l.chunks = (V + CHUNK - 1) / CHUNK;
  size_t at = (size_t)l.pieces * sizeof(Head);
  l.max_at = at;
  at = (at + (size_t)l.chunks * 4 + 15) / 16 * 16;
  l.mass_at = at;
  at += (size_t)l.pieces * BINS * 8;
  l.count_at = at;
  at += (size_t)l.pieces * BINS * 4;
  l.row = at;
  return l;
}

struct Row {
  bool greedy, masses;  // takes the first token; its histogram has masses
  int k;                // 0: no cut
  float p, least;       // 1 and 0: no cut
  double inv;
};
__device__ __forceinline__ Row row_of(const SampleArgs& a, int b) {
  Row r;
  const float t = a.temperature ? a.temperature[b] : 1.f;
  r.k = a.top_k ? max(a.top_k[b], 0) : 0;
  r.greedy = !(t > 0.f) || r.k == 1;
  r.p = a.top_p ? a.top_p[b] : 1.f;
  r.p = r.p < 1.f ? fmaxf(r.p, 0.f) : 1.f;
  r.least = a.min_p ? a.min_p[b] : 0.f;
  r.least = r.least > 0.f ? fminf(r.least, 1.f) : 0.f;
  r.inv = r.greedy ? 1.0 : 1.0 / (double)t;
  r.masses = !r.greedy && (r.k == 0 ? r.p < 1.f || r.least == 0.f : r.k > COUNT_K);
  return r;
}

// The bin of a logit, counted in eighths from 0 up, and its place from its centre.
__device__ __forceinline__ double bin_of(float z, double inv) { return floor((double)z * inv * 8.0); }
__device__ __forceinline__ int below(double top, double bin) {
  const double d = top - bin;
  return d < (double)BINS ? (int)d : BINS;
}
// exp of the place in units of 2^-44. |place| <= 1/16: the Taylor sum up to r^8 is off by 2^-54. (Far
// out, where eighths are below the spacing of fp64, every logit has a bin of its own and the place is 0.)
__device__ __forceinline__ uint64_t mass_in_bin(float z, double inv, double bin) {
  const double r = fabs(bin) < 0x1p52 ? __builtin_fma((double)z, inv, -(bin + 0.5) * 0.125) : 0.0;
  double p = 1.0 / 40320.0;
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 257.0);  // 256 + e: its last bit is 2^-44
  return (uint64_t)__double_as_longlong(p) - 0x4070000000000000ull;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __uint_as_float(xor_lanes(__float_as_uint(v), off)));
  return v;
}

template <bool BF16, int G8>
__global__ __launch_bounds__(HIST_THREADS) void sample_hist_kernel(SampleArgs a, Layout lay) {
  __shared__ unsigned long long s_mass[BINS];
  __shared__ uint32_t s_count[BINS];
  __shared__ float s_top[HIST_THREADS / 64];
  __shared__ uint32_t s_first, s_live, s_used;
  const int b = blockIdx.x / lay.pieces, piece = blockIdx.x - b * lay.pieces, tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const Row row = row_of(a, b);
  const char* z = (const char*)a.z + (size_t)b * a.stride * (BF16 ? 2 : 4);
  char* ws = (char*)a.ws + (size_t)b * lay.row;
  const int base = piece * (G8 * PIECE8) + tid * 8;
  float v[G8][8];
#pragma unroll
  for (int g = 0; g < G8; ++g) load8<BF16>(z, base + g * PIECE8, a.V, v[g]);
  for (int i = tid; i < BINS; i += HIST_THREADS) {
    s_mass[i] = 0;
    s_count[i] = 0;
  }
  if (tid == 0) {
    s_first = 0xFFFFFFFFu;
    s_live = 0;
    s_used = 0;
  }
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < G8; ++g) {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[g][j] = canon(v[g][j]);
      m = fmaxf(m, v[g][j]);
    }
    m = wave_max(m);
    top = fmaxf(top, m);
    const int chunk = (base + g * PIECE8) / CHUNK;
    if (lane == 0 && chunk < lay.chunks) ((float*)(ws + lay.max_at))[chunk] = m;
  }
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < HIST_THREADS / 64; ++w) top = fmaxf(top, s_top[w]);
  Head* head = (Head*)ws + piece;
  if (row.greedy || top == -INFINITY) {
    uint32_t first = 0xFFFFFFFFu;
#pragma unroll
    for (int g = G8 - 1; g >= 0; --g)
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (v[g][j] == top) first = base + g * PIECE8 + j;
    if (first != 0xFFFFFFFFu) atomicMin(&s_first, first);
    __syncthreads();
    if (tid == 0) *head = Head{top, s_first, top == -INFINITY ? 0u : 1u, 0u};
    return;
  }
  const double tb = bin_of(top, row.inv);
  uint32_t rest = 0;
#pragma unroll
  for (int g = 0; g < G8; ++g)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (v[g][j] == -INFINITY) continue;
      const double bin = bin_of(v[g][j], row.inv);
      const int i = below(tb, bin);
      if (i < BINS) {
        atomicAdd(&s_count[i], 1u);
        if (row.masses) atomicAdd(&s_mass[i], (unsigned long long)mass_in_bin(v[g][j], row.inv, bin));
      } else {
        ++rest;
      }
    }
  rest = (uint32_t)wave_sum_int((int)rest);
  if (lane == 0 && rest) atomicAdd(&s_live, rest);
  __syncthreads();
  static_assert(BINS == HIST_THREADS, "a bin for each thread");
  const uint32_t n = s_count[tid];
  const uint64_t some = __ballot(n > 0);
  const int all = wave_sum_int((int)n);
  if (lane == 0 && some) {
    atomicMax(&s_used, (uint32_t)(wave * 64 + 64 - __builtin_clzll(some)));
    atomicAdd(&s_live, (uint32_t)all);
  }
  __syncthreads();
  const uint32_t used = s_used;
  if ((uint32_t)tid < used) {
    ((uint32_t*)(ws + lay.count_at))[piece * BINS + tid] = n;
    if (row.masses) ((uint64_t*)(ws + lay.mass_at))[piece * BINS + tid] = s_mass[tid];
  }
  if (tid == 0) *head = Head{top, 0u, s_live, used};
}

// ---------------------------------------------------------------------------- a row's decision

struct Sum {
  uint32_t count;
  double mass;
};

struct Lds {
  double mass[BINS];     // up to and with a bin, relative to the centre of the first
  uint32_t count[BINS];
  unsigned long long sub_mass[BINS];
  uint32_t sub_count[BINS];
  uint64_t list[CAP];    // (descending logit, id)
  double upto[CAP];      // masses of the list up to and with a place
  uint16_t chunk[MAX_CHUNKS];
  double wave_mass[THREADS / 64];
  uint64_t wave_u[THREADS / 64];
  uint32_t wave_count[THREADS / 64];
  uint32_t chunks, n, at, id;
};

// Inclusive sums over the block's threads in order; `total` that of all.
__device__ double scan_mass(double v, Lds& s, double& total) {
  const int lane = lane_id(), wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(v, off, 64);
    if (lane >= off) v += o;
  }
  __syncthreads();
  if (lane == 63) s.wave_mass[wave] = v;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w == wave) before = total;
    total += s.wave_mass[w];
  }
  return before + v;
}
__device__ uint32_t scan_count(uint32_t v, Lds& s, uint32_t& total) {
  const int wave = threadIdx.x >> 6;
  v = (uint32_t)wave_incl_scan((int)v);
  __syncthreads();
  if (lane_id() == 63) s.wave_count[wave] = v;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w == wave) before = total;
    total += s.wave_count[w];
  }
  return before + v;
}
__device__ uint64_t scan_u64(uint64_t v, Lds& s) {
  const int lane = lane_id(), wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint64_t o = shfl_u64(v, max(lane - off, 0));
    if (lane >= off) v += o;
  }
  __syncthreads();
  if (lane == 63) s.wave_u[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += s.wave_u[w];
  return v;
}
// The lowest thread number among those whose flag is set (THREADS if none).
__device__ uint32_t first_of(bool flag, Lds& s) {
  const uint64_t m = __ballot(flag);
  __syncthreads();
  if (threadIdx.x == 0) s.at = THREADS;
  __syncthreads();
  if (m && lane_id() == 0) atomicMin(&s.at, (uint32_t)((threadIdx.x & ~63u) + __builtin_ctzll(m)));
  __syncthreads();
  return s.at;
}

template <bool BF16>
struct Decide {
  const SampleArgs& a;
  const Layout& lay;
  Lds& s;
  const int b, tid, lane, wave;
  const Row row;
  const char* z;
  const char* ws;
  float top;   // the row's largest logit
  double tb;   // its bin

  __device__ Decide(const SampleArgs& args, const Layout& l, Lds& lds)
      : a(args), lay(l), s(lds), b(blockIdx.x), tid(threadIdx.x), lane(lane_id()), wave(threadIdx.x >> 6), row(row_of(args, blockIdx.x)) {
    z = (const char*)a.z + (size_t)b * a.stride * (BF16 ? 2 : 4);
    ws = (const char*)a.ws + (size_t)b * lay.row;
  }

  // The chunks with a logit of bin `last` or above it.
  __device__ void pick_chunks(int last) {
    __syncthreads();
    if (tid == 0) s.chunks = 0;
    __syncthreads();
    for (int c0 = 0; c0 < lay.chunks; c0 += THREADS) {
      const int c = c0 + tid;
      const float m = c < lay.chunks ? ((const float*)(ws + lay.max_at))[c] : -INFINITY;
      const bool in = m > -INFINITY && below(tb, bin_of(m, row.inv)) <= last;
      const uint64_t mask = __ballot(in);
      uint32_t at = 0;
      if (lane == 0 && mask) at = atomicAdd(&s.chunks, (uint32_t)__builtin_popcountll(mask));
      at = __builtin_amdgcn_readfirstlane(at);
      if (in) s.chunk[at + __builtin_popcountll(mask & ((1ull << lane) - 1))] = (uint16_t)c;
    }
    __syncthreads();
  }
  // f(z, id, bin index) for every token of the picked chunks that is not masked; lanes without one have in = false.
  template <class F>
  __device__ void each(F f) {
    for (uint32_t n = wave; n < s.chunks; n += THREADS / 64) {
      const int i = s.chunk[n] * CHUNK + lane * 8;
      float v[8];
      load8<BF16>(z, i, a.V, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = canon(v[j]);
        const double bin = bin_of(x, row.inv);
        f(x, i + j, x > -INFINITY ? below(tb, bin) : BINS + 1, bin);
      }
    }
  }
  // The picked chunks' tokens that f takes, sorted, into the list: at most CAP. Returns their number.
  template <class F>
  __device__ int collect(F f) {
    if (tid == 0) s.n = 0;
    __syncthreads();
    each([&](float x, int id, int i, double) {
      const bool in = f(x, i);
      const uint64_t mask = __ballot(in);
      if (!mask) return;
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&s.n, (uint32_t)__builtin_popcountll(mask));
      at = __builtin_amdgcn_readfirstlane(at) + __builtin_popcountll(mask & ((1ull << lane) - 1));
      if (in && at < CAP) s.list[at] = ((uint64_t)~key_of(x) << 32) | (uint32_t)id;
    });
    __syncthreads();
    const int n = min((int)s.n, CAP);
    int n2 = 2;
    while (n2 < n) n2 <<= 1;
    for (int i = n + tid; i < n2; i += THREADS) s.list[i] = ~0ull;
    __syncthreads();
    for (int size = 2; size <= n2; size <<= 1)
      for (int step = size >> 1; step > 0; step >>= 1) {
        if (tid < n2 / 2) {
          const int i = 2 * tid - (tid & (step - 1)), j = i + step;
          const uint64_t x = s.list[i], y = s.list[j];
          if ((x > y) == ((i & size) == 0)) {
            s.list[i] = y;
            s.list[j] = x;
          }
        }
        __syncthreads();
      }
    return n;
  }
  __device__ float list_z(int i) const { return z_of(~(uint32_t)(s.list[i] >> 32)); }
  __device__ int list_id(int i) const { return (int)(uint32_t)s.list[i]; }
  // Mass relative to the largest logit's.
  __device__ double mass_of(float x) const { return exp64(((double)x - (double)top) * row.inv); }

  __device__ void answer(int token, double prob, int64_t kept) {
    if (tid != 0) return;
    a.token[b] = token;
    if (a.prob) a.prob[b] = (float)prob;
    if (a.kept) a.kept[b] = (int)kept;
  }
  __device__ double number() const {
    const float u = a.u[b];
    return u > 0.f ? (double)u : 0.0;
  }

  // ---- one bin at a time, where the tokens down to the last bin that matters are more than a list

  enum { COUNT, REACH, EXCEED };  // what crosses: the count, the mass reaching or exceeding a value
  struct Place {
    Sum sum;  // up to and with the token
    float z;
    int id;
  };
  // The first token of bin i at which the sums of the row cross `value`; the last one of the bin if none does.
  __device__ Place cross(int i, int mode, double value) {
    const uint32_t count0 = i ? s.count[i - 1] : 0;
    const double mass0 = i ? s.mass[i - 1] : 0.0, unit = exp64(-0.125 * i) * 0x1p-44;
    const double bin = tb - i;
    const auto crossed = [&](uint32_t n, uint64_t m) {
      const double mass = mass0 + unit * (double)m;
      return mode == COUNT ? (double)(count0 + n) >= value : mode == REACH ? mass >= value : mass > value;
    };
    // keys of the bin's logits lie in [lo, hi]: its edges, a little wider
    uint32_t hi = key_of(top), lo = key_of(-FLT_MAX);
    if (row.inv > 1e-60 && fabs(bin) < 0x1p52) {
      const double z0 = bin * 0.125 / row.inv, z1 = (bin + 1.0) * 0.125 / row.inv, w = (fabs(z0) + fabs(z1)) * 0x1p-20 + 1e-40;
      if (z1 + w < (double)top) hi = key_of((float)(z1 + w) + 0.f);
      if (z0 - w > -(double)FLT_MAX) lo = key_of((float)(z0 - w) + 0.f);
      if (hi < lo) hi = lo;
      hi = min(hi + 2, key_of(top));
      lo = lo > 2 ? lo - 2 : 0;
    }
    uint32_t n0 = 0, n = s.count[i] - count0;  // tokens of the bin above hi, and in [lo, hi]
    uint64_t m0 = 0;
    pick_chunks(i);
    for (;;) {
      const auto in = [=](float x, int j) { return j == i && key_of(x) >= lo && key_of(x) <= hi; };
      if (n <= (uint32_t)CAP) {
        const int len = collect(in);
        if (len == 0) return Place{{count0 + n0, mass0}, top, -1};  // (the logits have changed since the first kernel)
        // two neighbouring places a thread
        const int p = 2 * tid;
        const uint64_t e0 = p < len ? mass_in_bin(list_z(p), row.inv, bin) : 0, e1 = p + 1 < len ? mass_in_bin(list_z(p + 1), row.inv, bin) : 0;
        const uint64_t m1 = m0 + scan_u64(e0 + e1, s), mp = m1 - e1;
        const bool c0 = p < len && crossed(n0 + p + 1, mp), c1 = p + 1 < len && crossed(n0 + p + 2, m1);
        uint32_t who = first_of(c0 || c1, s);
        int at;
        if (who == THREADS) {
          at = len - 1;
          who = at / 2;
        } else {
          if ((uint32_t)tid == who) s.n = c0 ? p : p + 1;
          __syncthreads();
          at = s.n;
        }
        if ((uint32_t)tid == who) s.wave_u[0] = at == p ? mp : m1;
        __syncthreads();
        const Place r{{count0 + n0 + at + 1, mass0 + unit * (double)s.wave_u[0]}, list_z(at), list_id(at)};
        __syncthreads();
        return r;
      }
      if (lo == hi) {  // more tokens of one logit than a list: they have one mass
        const float x = z_of(lo);
        const uint64_t e = mass_in_bin(x, row.inv, bin);
        uint32_t l = 0, h = n;  // crossed at h, not at l
        while (h - l > 1) {
          const uint32_t mid = (l + h) / 2;
          if (crossed(n0 + mid, m0 + mid * e)) h = mid;
          else l = mid;
        }
        return Place{{count0 + n0 + h, mass0 + unit * (double)(m0 + h * e)}, x, nth(x, h)};
      }
      const uint32_t span = hi - lo;
      const int sh = max(0, 32 - (int)__builtin_clz(span) - 9);
      __syncthreads();
      if (tid < BINS) {
        s.sub_mass[tid] = 0;
        s.sub_count[tid] = 0;
      }
      __syncthreads();
      each([&](float x, int, int j, double) {
        if (!in(x, j)) return;
        const uint32_t q = (hi - key_of(x)) >> sh;
        atomicAdd(&s.sub_count[q], 1u);
        atomicAdd(&s.sub_mass[q], (unsigned long long)mass_in_bin(x, row.inv, bin));
      });
      __syncthreads();
      const uint32_t mine = tid < BINS ? s.sub_count[tid] : 0;
      const uint64_t mass = tid < BINS ? s.sub_mass[tid] : 0;
      uint32_t total;
      const uint32_t c = n0 + scan_count(mine, s, total);
      const uint64_t m = m0 + scan_u64(mass, s);
      uint32_t who = first_of(mine > 0 && crossed(c, m), s);
      if (who == THREADS) {  // (the last one that is not empty)
        who = THREADS - 1 - first_of_reversed(mine > 0);
        if (who >= THREADS) return Place{{count0 + n0, mass0}, top, -1};
      }
      __syncthreads();
      if ((uint32_t)tid == who) {
        s.n = c - mine;
        s.at = mine;
        s.wave_u[0] = m - mass;
      }
      __syncthreads();
      n0 = s.n;
      n = s.at;
      m0 = s.wave_u[0];
      hi -= who << sh;
      lo = max(lo, hi - min(hi, (1u << sh) - 1));
      __syncthreads();
    }
  }
  __device__ uint32_t first_of_reversed(bool flag) {
    const uint64_t m = __ballot(flag);
    __syncthreads();
    if (tid == 0) s.at = THREADS;
    __syncthreads();
    if (m && lane == 0) atomicMin(&s.at, (uint32_t)(THREADS - 1 - ((tid & ~63) + 63 - __builtin_clzll(m))));
    __syncthreads();
    return s.at;
  }
  // Id of the n-th token (from 1) whose logit is x.
  __device__ int nth(float x, uint32_t n) {
    uint32_t before = 0;
    __syncthreads();
    if (tid == 0) s.id = 0;
    for (int base = 0; base < a.V; base += THREADS * 8) {
      float v[8];
      load8<BF16>(z, base + tid * 8, a.V, v);
      uint32_t mine = 0, total;
#pragma unroll
      for (int j = 0; j < 8; ++j) mine += canon(v[j]) == x ? 1 : 0;
      const uint32_t upto = before + scan_count(mine, s, total);
      if (upto - mine < n && n <= upto) {
        uint32_t at = upto - mine;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (canon(v[j]) == x && ++at == n) s.id = base + tid * 8 + j;
      }
      before += total;
      if (before >= n) break;
    }
    __syncthreads();
    return (int)s.id;
  }
  // First bin whose sums cross; the last one that is not empty if none does.
  __device__ int bin_where(int mode, double value) {
    const bool in = tid < BINS && (tid == 0 || s.count[tid] > s.count[tid - 1]);
    const bool yes = in && (mode == COUNT ? (double)s.count[tid] >= value : mode == REACH ? s.mass[tid] >= value : s.mass[tid] > value);
    const uint32_t i = first_of(yes, s);
    return i < THREADS ? (int)i : (int)(THREADS - 1 - first_of_reversed(in));
  }
  // Count and mass (relative to the first bin's centre) of the row's tokens with (z - top) / temperature >= low.
  __device__ Sum at_least(double low) {
    Sum v{0, 0.0};
    for (int c = wave; c < lay.chunks; c += THREADS / 64) {
      if (!(((const float*)(ws + lay.max_at))[c] > -INFINITY)) continue;
      const int i = c * CHUNK + lane * 8;
      float x[8];
      load8<BF16>(z, i, a.V, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = canon(x[j]);
        const double d = ((double)y - (double)top) * row.inv;
        if (y > -INFINITY && d >= low) {
          v.count += 1;
          v.mass += exp64(d);
        }
      }
    }
    double mass;
    uint32_t count;
    scan_mass(v.mass, s, mass);
    scan_count(v.count, s, count);
    return Sum{count, mass / from_centre()};
  }
  // The mass at the centre of the first bin relative to the largest logit's.
  __device__ double from_centre() const {
    const double c = fabs(tb) < 0x1p52 ? -__builtin_fma((double)top, row.inv, -(tb + 0.5) * 0.125) : 0.0;
    return c < 0 ? exp64(c) : 1.0 / exp64(-c);
  }

  __device__ void run();
};

template <bool BF16>
__device__ void Decide<BF16>::run() {
  // the row's largest logit and its tokens
  const Head* heads = (const Head*)ws;
  float m = -INFINITY;
  uint32_t live = 0;
  for (int i = tid; i < lay.pieces; i += THREADS) {
    m = fmaxf(m, heads[i].top);
    live += heads[i].live;
  }
  m = wave_max(m);
  if (lane == 0) s.wave_mass[wave] = (double)m;
  uint32_t total;
  __syncthreads();
  top = -INFINITY;
  for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, (float)s.wave_mass[w]);
  scan_count(live, s, total);
  live = total;
  if (top == -INFINITY) {
    answer(-1, 0.0, 0);
    return;
  }
  if (row.greedy) {
    if (tid == 0) s.id = 0xFFFFFFFFu;
    __syncthreads();
    for (int i = tid; i < lay.pieces; i += THREADS)
      if (heads[i].top == top) atomicMin(&s.id, heads[i].first);
    __syncthreads();
    answer((int)s.id, 1.0, 1);
    return;
  }
  tb = bin_of(top, row.inv);
  // the pieces' histograms, each from its own maximum's bin down
  uint32_t n = 0;
  uint64_t fixed = 0;
  if (tid < BINS)
    for (int p = 0; p < lay.pieces; ++p) {
      if (heads[p].top == -INFINITY) continue;
      const int i = tid - below(tb, bin_of(heads[p].top, row.inv));
      if (i < 0 || (uint32_t)i >= heads[p].used) continue;
      n += ((const uint32_t*)(ws + lay.count_at))[p * BINS + i];
      if (row.masses) fixed += ((const uint64_t*)(ws + lay.mass_at))[p * BINS + i];
    }
  bool masses = row.masses;
  const double unit = tid < BINS ? exp64(-0.125 * tid) * 0x1p-44 : 0.0;
  double all;
  const double mass = scan_mass((double)fixed * unit, s, all);
  uint32_t binned;
  const uint32_t count = scan_count(n, s, binned);
  if (tid < BINS) {
    s.count[tid] = count;
    s.mass[tid] = mass;
  }
  __syncthreads();
  const int64_t K = row.k > 0 ? min((int64_t)row.k, (int64_t)live) : (int64_t)live;
  const bool cut_k = K < (int64_t)live && K <= (int64_t)binned;
  const double low = row.least > 0.f ? log((double)row.least) : -INFINITY;

  // the last bin that matters
  const int bk = cut_k ? bin_where(COUNT, (double)K) : BINS - 1;
  int last = bk;
  if (row.p == 1.f || (masses && !cut_k)) {  // (else top-p's sum is that of the list)
    if (row.least > 0.f) {
      const double d = tb - floor(((double)top * row.inv + low) * 8.0) + 1.0;
      if (d < (double)last) last = (int)d;
    }
    // (a little beyond the threshold, whose last bits are another sum's)
    if (masses && row.p < 1.f) last = min(last, bin_where(REACH, (double)row.p * s.mass[BINS - 1] * (1.0 + 0x1p-40)));
  }
  if (s.count[last] <= (uint32_t)CAP) {
    pick_chunks(last);
    const int len = collect([=](float, int i) { return i <= last; });
    if (len == 0) {  // (the logits have changed since the first kernel)
      answer(-1, 0.0, 0);
      return;
    }
    const int p = 2 * tid;
    const double e0 = p < len ? mass_of(list_z(p)) : 0.0, e1 = p + 1 < len ? mass_of(list_z(p + 1)) : 0.0;
    double sum;
    const double m1 = scan_mass(e0 + e1, s, sum), m0 = m1 - e1;
    s.upto[p] = p < len ? m0 : sum;
    s.upto[p + 1] = m1;
    __syncthreads();
    int cut = (int)min((int64_t)len, K);
    bool short_of = false;  // of the tokens below the bins, which have no mass
    if (row.p < 1.f) {
      double whole = s.upto[cut - 1];
      if (masses && !cut_k) whole = s.mass[BINS - 1] * from_centre();
      const double want = (double)row.p * whole;
      const uint32_t who = first_of((p < cut && m0 >= want) || (p + 1 < cut && m1 >= want), s);
      if (who < THREADS) {
        cut = min(cut, (int)(2 * who + (s.upto[2 * who] >= want ? 1 : 2)));
        short_of = true;
      }
    }
    int64_t kept = short_of ? cut : cut == len && last == BINS - 1 ? K : cut;
    if (row.least > 0.f) {
      uint32_t c;
      scan_count((p < len && ((double)list_z(p) - (double)top) * row.inv >= low ? 1u : 0u) +
                     (p + 1 < len && ((double)list_z(p + 1) - (double)top) * row.inv >= low ? 1u : 0u),
                 s, c);
      if (kept > (int64_t)len && low < -60.0) c = at_least(low).count;  // (tokens below the bins may be above low)
      kept = min(kept, (int64_t)max(c, 1u));
      cut = min(cut, (int)min(kept, (int64_t)len));
    }
    const double part = s.upto[cut - 1], want = number() * part;
    const uint32_t who = first_of((p < cut && m0 > want) || (p + 1 < cut && m1 > want), s);
    const int at = who < THREADS ? (int)(2 * who + (s.upto[2 * who] > want ? 0 : 1)) : cut - 1;
    answer(list_id(at), mass_of(list_z(at)) / part, kept);
    return;
  }

  if (!masses) {  // counted only, and too many for a list after all
    __syncthreads();
    if (tid < BINS) s.sub_mass[tid] = 0;
    pick_chunks(BINS - 1);
    each([&](float x, int, int i, double bin) {
      if (i < BINS) atomicAdd(&s.sub_mass[i], (unsigned long long)mass_in_bin(x, row.inv, bin));
    });
    __syncthreads();
    const double v = scan_mass(tid < BINS ? (double)s.sub_mass[tid] * unit : 0.0, s, all);
    if (tid < BINS) s.mass[tid] = v;
    __syncthreads();
  }
  // top-k, top-p, min-p, the draw, and (where rounding has put it behind the cut) the last token before the cut
  Sum cut{(uint32_t)K, s.mass[BINS - 1]};
  Place at{{0, 0.0}, top, -1};
  for (int step = 0; step < 5; ++step) {
    int mode = COUNT;
    double value = (double)K;
    if (step == 0) {
      if (!cut_k) continue;
    } else if (step == 1) {
      if (!(row.p < 1.f)) continue;
      mode = REACH;
      value = (double)row.p * cut.mass;
    } else if (step == 2) {
      if (row.least > 0.f) {
        const Sum c = at_least(low);
        if (c.count < cut.count) cut = c;
      }
      continue;
    } else if (step == 3) {
      mode = EXCEED;
      value = number() * cut.mass;
    } else {
      if (at.sum.count <= cut.count) continue;
      value = (double)cut.count;
    }
    const Place p = cross(bin_where(mode, value), mode, value);
    if (step >= 3) at = p;
    else if (step == 0 || p.sum.count < cut.count) cut = p.sum;
  }
  answer(at.id, mass_of(at.z) / (cut.mass * from_centre()), cut.count);
}

template <bool BF16>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a, Layout lay) {
  __shared__ Lds lds;
  Decide<BF16> d(a, lay, lds);
  d.run();
}

template <bool BF16>
hipError_t launch(const SampleArgs& a, hipStream_t s) {
  const Layout lay = layout_of(a.B, a.V);
  const int grid = a.B * lay.pieces;
  if (lay.g8 == 8) sample_hist_kernel<BF16, 8><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  else if (lay.g8 == 4) sample_hist_kernel<BF16, 4><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  else if (lay.g8 == 2) sample_hist_kernel<BF16, 2><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  else sample_hist_kernel<BF16, 1><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  sample_kernel<BF16><<<a.B, THREADS, 0, s>>>(a, lay);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace(int B, int V) { return layout_of(B, V).row * (size_t)B; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) { return a.bf16 ? launch<true>(a, s) : launch<false>(a, s); }

}  // namespace pmpe
