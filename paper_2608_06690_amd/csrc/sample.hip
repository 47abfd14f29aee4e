// One token per row of logits: temperature, top-k, top-p, min-p, and a draw by a given uniform number.
//
// The order of a row is (logit descending, id ascending); every cut leaves a leading part of it, and the
// draw is its first token whose cumulated mass exceeds u times the whole. Each of them is "the first place where
// the count, or the mass, up to it crosses a threshold".
//
// Two kernels. The first goes over the logits once, in pieces of a row that its blocks hold in registers:
// the piece's maximum, the maxima of its chunks of 512, and a histogram by x = z / temperature in bins of 1/8 (512
// of them from the maximum down: what lies lower has less than e^-63 of its mass) of counts and masses. The second
// has a block per row: it adds up the histograms, finds the bins of the thresholds, and collects the tokens of the
// bins that matter from the chunks that hold one, in LDS. A threshold's token is then found by histograms of the
// order's bits inside its bin (9 bits a round) until 64 tokens are left, which one wave ranks. Bins with more tokens
// than the list holds (ties, flat rows) have their first rounds over the logits themselves.
//
// Both are bound by issue and latency, not by memory: 256 rows of 131,072 bf16 logits (67 MB, 13 us at a large
// copy's rate) take 36 us in the first kernel, whose bins and masses are about 20 vector operations a logit, and 94 to
// 114 us in the second, whose time is its longest row's: a CU goes over a row alone, about 2 us for 8192
// logits, once more for every threshold whose bins the list did not hold. One row of 131,071: 5 + 70 us at most.
//
// Masses are integers inside a bin (units of 2^-44 of the mass at its centre, right to 2^-43), so their sums do not
// depend on the order of the atomics; across bins they are fp64 in a fixed order.
#include <cfloat>

#include "exp64.h"
#include "pmpe_internal.h"

namespace pmpe {
namespace {

constexpr int BINS = 512;
constexpr int CHUNK = 512;      // logits that a wave loads at once, 8 a lane
constexpr int HIST_THREADS = 512;
constexpr int PIECE8 = HIST_THREADS * 8;
constexpr int THREADS = 512;    // of the second kernel: a bin for each
constexpr int CAP = 16 * THREADS;  // tokens of a list
constexpr int MAX_CHUNKS = PMPE_MAX_VOCAB / CHUNK;
constexpr int MAX_PIECES = PMPE_MAX_VOCAB / PIECE8;
constexpr int ID_BITS = 19;
// rows whose top_k is at most this are counted only: their list has the masses
constexpr int COUNT_K = CAP / 4;

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float z_of(uint32_t k) { return __uint_as_float((k >> 31) ? k ^ 0x80000000u : ~k); }
// A logit as it counts: masked ones (also NaN) -inf, +inf the largest finite value, -0 as 0.
__device__ __forceinline__ float canon(float v) { return fminf(fmaxf(v, -INFINITY), FLT_MAX) + 0.f; }  // (a maximum leaves NaN out)

// Logits [i, i + 8) of a row of n as they lie in memory: the last 8 of the row where those reach past its end, so that
// every load is whole and none waits for a branch. Rows of fewer than 8 are read one by one.
template <bool BF16>
struct Eight {
  u32x4 q[BF16 ? 1 : 2];
  int at;    // index of the first of them
  int skip;  // so many of them are ahead of i
};
template <bool BF16>
__device__ __forceinline__ Eight<BF16> load8(const char* row, int i, int n) {
  Eight<BF16> e;
  e.at = min(i, n - 8);
  e.skip = i - e.at;
  if (n >= 8) {
    const char* p = row + (size_t)e.at * (BF16 ? 2 : 4);
    e.q[0] = *(const u32x4_a2*)p;
    if constexpr (!BF16) e.q[1] = *(const u32x4_a2*)(p + 16);
  } else {
#pragma unroll
    for (int j = 0; j < (BF16 ? 4 : 8); ++j) {
      const int k = e.at + (BF16 ? 2 * j : j);
      uint32_t w = 0;
      if constexpr (BF16) {
        if (k >= 0) w = ((const uint16_t*)row)[k];
        if (k >= -1) w |= (uint32_t)((const uint16_t*)row)[k + 1] << 16;
      } else {
        if (k >= 0) w = ((const uint32_t*)row)[k];
      }
      e.q[j / 4][j & 3] = w;
    }
    e.skip = max(e.skip, -e.at);
  }
  return e;
}
template <bool BF16>
__device__ __forceinline__ float value_of(const Eight<BF16>& e, int j) {
  const uint32_t w = BF16 ? e.q[0][j / 2] : e.q[BF16 ? 0 : j / 4][j & 3];
  return __uint_as_float(BF16 ? (j & 1) ? w & 0xFFFF0000u : w << 16 : w);
}
// Their values as they count; -inf for those ahead of i.
template <bool BF16>
__device__ __forceinline__ void values8(const Eight<BF16>& e, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = j >= e.skip ? canon(value_of<BF16>(e, j)) : -INFINITY;
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
// The largest pieces (less of the histograms' bytes) of which there are two for each CU; still larger ones load and
// count by turns (256 rows of 131072 bf16 logits: 44 us with pieces of 32768, 37 with 16384, 35 with 8192).
__host__ __device__ inline Layout layout_of(int B, int V) {
  Layout l{};
  l.g8 = 4;
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
  double t, inv;        // the temperature and its reciprocal
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
  r.t = r.greedy ? 1.0 : (double)t;
  r.inv = 1.0 / r.t;
  r.masses = !r.greedy && (r.k == 0 ? r.p < 1.f || r.least == 0.f : r.k > COUNT_K);
  return r;
}

// The bins of a row: floor(fl(z 8 / T)) in fp32, counted down from that of the row's (or a piece's) largest logit. What
// counts is that this never falls with z; a logit may lie beyond its bin's edges by 2^-23 of 8 z / T, and its mass is that
// of its exact place. Where 8 z / T is FAR or more at the row's top (temperatures next to 0, say), fp64 makes the bins. A
// piece whose top is among the row's bins may lie BINS below it: its own limit is so much larger that it has its histogram
// in every row that needs it.
constexpr float FAR = 0x1p20f, FAR_PIECE = FAR + 2 * BINS;
struct Bins {
  double inv;   // 1 / T
  float inv8;   // 8 / T
  bool far;
  double top;   // the first bin (a whole number)
};
__device__ __forceinline__ Bins bins_of(const Row& r, float top, float limit) {
  Bins b;
  b.inv = r.inv;
  b.inv8 = (float)(8.0 * r.inv);
  b.far = !(fabsf(top * b.inv8) < limit);
  b.top = b.far ? floor((double)top * r.inv * 8.0) : (double)floorf(top * b.inv8);
  return b;
}
// BINS where a logit lies below them.
__device__ __forceinline__ int bin_of(const Bins& b, float z) {
  if (b.far) {
    const double d = b.top - floor((double)z * b.inv * 8.0);
    return d < (double)BINS ? (int)d : BINS;
  }
  const float d = (float)b.top - floorf(z * b.inv8);
  return d < (float)BINS ? (int)d : BINS;
}
// The logit's place from the centre of bin i over the temperature, at most 0.08. (Far out, where eighths are below the
// spacing of fp64, every logit has a bin of its own and the place is 0.)
__device__ __forceinline__ double place_in_bin(const Bins& b, float z, int i) {
  if (b.far && !(fabs(b.top) < 0x1p51)) return 0.0;
  return __builtin_fma((double)z, b.inv, -((b.top - i) + 0.5) * 0.125);
}
// exp of that in units of 2^-44. The terms from r^4 on are below 2^-19 and come from fp32, off by 2^-43; with r^9
// and later left out, by 2^-51.
__device__ __forceinline__ uint64_t units_in_bin(const Bins& b, float z, int i) {
  const double r = place_in_bin(b, z, i);
  const float f = (float)r;
  float q = 1.f / 40320.f;
  q = __builtin_fmaf(q, f, 1.f / 5040.f);
  q = __builtin_fmaf(q, f, 1.f / 720.f);
  q = __builtin_fmaf(q, f, 1.f / 120.f);
  q = __builtin_fmaf(q, f, 1.f / 24.f);
  double p = (double)q;
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
  Eight<BF16> raw[G8];
#pragma unroll
  for (int g = 0; g < G8; ++g) raw[g] = load8<BF16>(z, base + g * PIECE8, a.V);
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
    values8<BF16>(raw[g], v[g]);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, v[g][j]);
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
        if (v[g][j] == top) first = raw[g].at + j;
    if (first != 0xFFFFFFFFu) atomicMin(&s_first, first);
    __syncthreads();
    if (tid == 0) *head = Head{top, s_first, top == -INFINITY ? 0u : 1u, 0u};
    return;
  }
  const Bins bins = bins_of(row, top, FAR_PIECE);
  uint32_t rest = 0;
  if (bins.far) {  // too far from its row's top for the histogram, or all of the row is
#pragma unroll
    for (int g = 0; g < G8; ++g)
#pragma unroll
      for (int j = 0; j < 8; ++j) rest += v[g][j] > -INFINITY ? 1 : 0;
  } else {
#pragma unroll
    for (int g = 0; g < G8; ++g)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = v[g][j], d = (float)bins.top - floorf(z * bins.inv8);
        if (d < (float)BINS) {
          const int i = (int)d;
          atomicAdd(&s_count[i], 1u);
          if (row.masses) atomicAdd(&s_mass[i], (unsigned long long)units_in_bin(bins, z, i));
        } else {
          rest += z > -INFINITY ? 1 : 0;
        }
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
  uint64_t list[CAP];    // places in the order
  uint64_t few[64];
  uint16_t chunk[MAX_CHUNKS];
  int shift[MAX_PIECES], used[MAX_PIECES];
  double wave_mass[THREADS / 64];
  uint64_t wave_u[THREADS / 64];
  uint32_t wave_count[THREADS / 64];
  uint32_t chunks, n, at, pos, rest;
  uint64_t place, mass_at;
};

// What all threads have alike, in scalar registers.
__device__ __forceinline__ uint32_t uni(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uni(float v) { return __uint_as_float(uni(__float_as_uint(v))); }
__device__ __forceinline__ uint64_t uni(uint64_t v) { return ((uint64_t)uni((uint32_t)(v >> 32)) << 32) | uni((uint32_t)v); }
__device__ __forceinline__ double uni(double v) { return __longlong_as_double((long long)uni((uint64_t)__double_as_longlong(v))); }

__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {
  const int lane = lane_id();
#pragma unroll 1
  for (int off = 1; off < 64; off <<= 1) {
    const uint64_t o = shfl_u64(v, max(lane - off, 0));
    if (lane >= off) v += o;
  }
  return v;
}
// Inclusive sums over the block's threads.
__device__ __forceinline__ void scan_both(Lds& s, uint32_t& count, uint64_t& mass) {
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  count = (uint32_t)wave_incl_scan((int)count);
  mass = wave_scan_u64(mass);
  __syncthreads();
  if (lane == 63) {
    s.wave_count[wave] = count;
    s.wave_u[wave] = mass;
  }
  __syncthreads();
#pragma unroll 1
  for (int w = 0; w < wave; ++w) {
    count += s.wave_count[w];
    mass += s.wave_u[w];
  }
}
// The bins' sums from the top down into s.count and s.mass.
__device__ __forceinline__ void scan_bins(Lds& s, uint32_t count, double mass) {
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  count = (uint32_t)wave_incl_scan((int)count);
#pragma unroll 1
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(mass, off, 64);
    if (lane >= off) mass += o;
  }
  __syncthreads();
  if (lane == 63) {
    s.wave_count[wave] = count;
    s.wave_mass[wave] = mass;
  }
  __syncthreads();
  uint32_t c = 0;
  double m = 0.0;
#pragma unroll 1
  for (int w = 0; w < wave; ++w) {
    c += s.wave_count[w];
    m += s.wave_mass[w];
  }
  s.count[threadIdx.x] = c + count;
  s.mass[threadIdx.x] = m + mass;
  __syncthreads();
}
// The lowest thread number among those whose flag is set, else the highest among those whose second flag is set
// (THREADS or more: none).
__device__ __forceinline__ int first_of(Lds& s, bool flag, bool other) {
  const uint64_t m = __ballot(flag), o = __ballot(other);
  const uint32_t base = threadIdx.x & ~63u;
  __syncthreads();
  if (threadIdx.x == 0) {
    s.at = THREADS;
    s.pos = THREADS;
  }
  __syncthreads();
  if (lane_id() == 0) {
    if (m) atomicMin(&s.at, base + (uint32_t)__builtin_ctzll(m));
    if (o) atomicMin(&s.pos, (uint32_t)(THREADS - 1 - (base + 63 - __builtin_clzll(o))));
  }
  __syncthreads();
  const uint32_t at = uni(s.at), pos = uni(s.pos);
  return (int)(at < THREADS ? at : THREADS - 1 - pos);
}

// A token's place in the order: descending logit, then id.
__device__ __forceinline__ uint64_t place_of(float z, int id) { return ((uint64_t)~key_of(z) << ID_BITS) | (uint32_t)id; }
__device__ __forceinline__ float place_z(uint64_t p) { return z_of(~(uint32_t)(p >> ID_BITS)); }
__device__ __forceinline__ int place_id(uint64_t p) { return (int)(p & ((1u << ID_BITS) - 1)); }

// One way over tokens: those of the list, or of the row's chunks that hold a logit of z0 .. z1 or z2 .. z3. Of these,
// tokens count whose place is in lo .. hi. They are appended to the list, or counted, with their masses, in place
// (place - lo) >> sh, or (by_bin) in their bin's, of the sub-histogram (`rest`: below the bins).
struct Pass {
  bool listed, append, by_bin;
  int sh;
  float z0, z1, z2, z3;
  uint64_t lo, hi;
  // the row
  float top;
  Bins bins;
  const char* z;
  const float* chunk_top;
  int V, chunks;
};
template <bool BF16>
__device__ __forceinline__ void go_over(Lds& s, const Pass& p) {
  const int tid = threadIdx.x, lane = lane_id(), wave = uni(tid >> 6);
  constexpr int WAVES = THREADS / 64, U = 2;  // chunks that a wave takes at once, as many more under way
  __syncthreads();
  if (p.append) {
    if (tid == 0) s.n = 0;
  } else {
    s.sub_mass[tid] = 0;
    s.sub_count[tid] = 0;
  }
  if (tid == 0) {
    s.chunks = 0;
    s.rest = 0;
  }
  __syncthreads();
  // the chunks that hold one
  if (!p.listed) {
    const float least = fminf(p.z0, p.z2);
#pragma unroll 1
    for (int c0 = 0; c0 < p.chunks; c0 += THREADS) {
      const int c = c0 + tid;
      const bool in = c < p.chunks && p.chunk_top[c] >= least;
      const uint64_t mask = __ballot(in);
      uint32_t at = 0;
      if (lane == 0 && mask) at = atomicAdd(&s.chunks, (uint32_t)__builtin_popcountll(mask));
      at = uni(at);
      if (in) s.chunk[at + __builtin_popcountll(mask & ((1ull << lane) - 1))] = (uint16_t)c;
    }
    __syncthreads();
  }
  // (the list goes through the same steps, one of its places a lane)
  const uint32_t n = uni(p.listed ? s.n : s.chunks);
  Eight<BF16> next[U];
  const auto load = [&](uint32_t c) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = load8<BF16>(p.z, c + u < n ? s.chunk[c + u] * CHUNK + lane * 8 : p.V, p.V);
  };
  if (!p.listed) load(wave * U);
  const uint32_t step = p.listed ? THREADS : WAVES * U;
#pragma unroll 1
  for (uint32_t c = p.listed ? wave * 64 : wave * U; c < n; c += step) {
    float v[U * 8];
    int at[U];
    uint64_t place = 0;
    uint32_t left = 0;
    if (p.listed) {
      if (c + lane < n) {
        place = s.list[c + lane];
        left = place >= p.lo && place <= p.hi && place_z(place) >= p.z0 && place_z(place) <= p.z1 ? 1u : 0u;
      }
    } else {
      // (a bit for each of the lane's logits that counts; NaN does in no comparison, and without an upper end +inf does)
      Eight<BF16> now[U];
#pragma unroll
      for (int u = 0; u < U; ++u) now[u] = next[u];
      load(c + step);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        at[u] = now[u].at;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u * 8 + j] = value_of<BF16>(now[u], j);
      }
#pragma unroll
      for (int j = 0; j < 8 * U; ++j) left |= v[j] >= p.z0 ? 1u << j : 0u;
      if (p.z1 < p.top) {
        uint32_t above = 0;
#pragma unroll
        for (int j = 0; j < 8 * U; ++j) above |= v[j] > p.z1 ? 1u << j : 0u;
        left &= ~above;
      }
      if (p.z2 <= p.z3) {
#pragma unroll
        for (int j = 0; j < 8 * U; ++j) left |= v[j] >= p.z2 && v[j] <= p.z3 ? 1u << j : 0u;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (now[u].skip > 0) left &= ~(((1u << min(now[u].skip, 8)) - 1) << (8 * u));
    }
    while (__any(left != 0)) {
      const int j = left ? __builtin_ctz(left) : 0;
      float x = place_z(place);
      if (!p.listed) {
        x = v[0];
#pragma unroll
        for (int q = 1; q < 8 * U; ++q) x = j == q ? v[q] : x;
        int id = at[0];
#pragma unroll
        for (int u = 1; u < U; ++u) id = j >= 8 * u ? at[u] : id;
        x = canon(x);
        place = place_of(x, id + (j & 7));
      }
      const bool in = left != 0 && place >= p.lo && place <= p.hi;
      if (p.append) {
        const uint64_t mask = __ballot(in);
        uint32_t to = 0;
        if (lane == 0) to = atomicAdd(&s.n, (uint32_t)__builtin_popcountll(mask));
        to = uni(to) + __builtin_popcountll(mask & ((1ull << lane) - 1));
        if (in && to < CAP) s.list[to] = place;
      } else if (in) {
        const int i = bin_of(p.bins, x);
        const uint32_t q = p.by_bin ? (uint32_t)i : (uint32_t)((place - p.lo) >> p.sh);
        atomicAdd(q < BINS ? &s.sub_count[q] : &s.rest, 1u);
        if (q < BINS && i < BINS) atomicAdd(&s.sub_mass[q], (unsigned long long)units_in_bin(p.bins, x, i));
      }
      left &= left - 1;
    }
  }
  __syncthreads();
  if (p.append && tid == 0) s.n = min(s.n, (uint32_t)CAP);
  __syncthreads();
}

// The smallest logit of [-FLT_MAX, top] that `ok` holds for, where it holds for all larger ones and for top: a wave tries
// 64 logits at a time, first those around `near`.
template <class F>
__device__ __forceinline__ float smallest(float near, float top, F ok) {
  uint32_t a = key_of(-FLT_MAX), b = key_of(top);
  const uint32_t from = min(max(key_of(near), a + 32) - 32, b);
  uint32_t k = min(from + lane_id(), b);
  uint64_t yes = __ballot(ok(z_of(k)));
  if (yes == 0) {
    a = min(uni(from) + 64, b);
  } else if (yes & 1) {
    b = uni(from);
  } else {
    return z_of(uni(from) + (uint32_t)__builtin_ctzll(yes));
  }
#pragma unroll 1
  while (a < b) {
    const uint32_t step = ((b - a) >> 6) + 1;
    k = b - a < step * lane_id() ? b : a + step * lane_id();
    yes = __ballot(ok(z_of(k)) || k == b);
    if (yes == 0) {  // (64 steps of the rounded width may end ahead of b)
      a = (uint32_t)__builtin_amdgcn_readlane((int)k, 63) + 1;
      continue;
    }
    const int f = __builtin_ctzll(yes);
    const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)k, f);
    if (f == 0) {
      b = a;
    } else {
      a = min(at, (uint32_t)__builtin_amdgcn_readlane((int)k, f - 1) + 1);
      b = at;
    }
  }
  return z_of(a);
}

enum { COUNT, REACH, EXCEED };  // what crosses a value: the count, the mass reaching or exceeding it
__device__ __forceinline__ bool crossed(int mode, double value, uint32_t count, double mass) {
  return mode == COUNT ? (double)count >= value : mode == REACH ? mass >= value : mass > value;
}

template <bool BF16>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a, Layout lay) {
  __shared__ Lds s;
  const int b = blockIdx.x, tid = threadIdx.x, lane = lane_id(), wave = uni(tid >> 6);
  const Row row = row_of(a, b);
  const char* ws = (const char*)a.ws + (size_t)b * lay.row;
  const auto answer = [&](int token, double prob, int64_t kept) {
    if (tid != 0) return;
    a.token[b] = token;
    if (a.prob) a.prob[b] = (float)prob;
    if (a.kept) a.kept[b] = (int)kept;
  };

  // the row's largest logit and its tokens
  static_assert(MAX_PIECES <= THREADS && BINS == THREADS, "a piece and a bin for each thread");
  Head head{-INFINITY, 0xFFFFFFFFu, 0u, 0u};
  if (tid < lay.pieces) head = ((const Head*)ws)[tid];
  {
    const float m = wave_max(head.top);
    const int n = wave_sum_int((int)head.live);
    if (lane == 0) {
      s.wave_mass[wave] = (double)m;
      s.wave_count[wave] = (uint32_t)n;
    }
    if (tid == 0) s.pos = 0xFFFFFFFFu;
  }
  uint32_t live = 0;
  float top = -INFINITY;
  __syncthreads();
#pragma unroll 1
  for (int w = 0; w < (lay.pieces + 63) / 64; ++w) {
    top = fmaxf(top, (float)s.wave_mass[w]);
    live += s.wave_count[w];
  }
  top = uni(top);
  live = uni(live);
  if (top == -INFINITY) {
    answer(-1, 0.0, 0);
    return;
  }
  if (row.greedy) {
    if (head.top == top) atomicMin(&s.pos, head.first);
    __syncthreads();
    answer((int)s.pos, 1.0, 1);
    return;
  }
  const double inv = row.inv;
  Bins bins = bins_of(row, top, FAR);
  bins.inv8 = uni(bins.inv8);
  bins.top = uni(bins.top);
  bins.far = uni((int)bins.far) != 0;
  const auto index_of = [&](float x) { return bin_of(bins, x); };
  // The smallest logit of bin i or a nearer one, and the largest of bin i or a farther one.
  const auto low_edge = [&](int i) {
    if (i >= BINS) return -FLT_MAX;
    return smallest((float)fmin(fmax((bins.top - i) * 0.125 * row.t, -(double)FLT_MAX), (double)top), top, [&](float x) { return index_of(x) <= i; });
  };
  const auto high_edge = [&](int i) { return i == 0 ? top : z_of(key_of(low_edge(i - 1)) - 1); };

  // the pieces' histograms, each from its own maximum's bin down
  if (tid < lay.pieces) {
    const bool some = head.top > -INFINITY && !bins.far;
    s.shift[tid] = some ? index_of(head.top) : BINS;
    s.used[tid] = some ? (int)head.used : 0;
  }
  __syncthreads();
  const double unit = exp64(-0.125 * tid) * 0x1p-44;
  {
    uint32_t n = 0;
    uint64_t fixed = 0;
#pragma unroll 4
    for (int p = 0; p < lay.pieces; ++p) {
      const int i = tid - s.shift[p];
      const bool in = i >= 0 && i < s.used[p];
      const int at = p * BINS + (in ? i : 0);
      const uint32_t c = ((const uint32_t*)(ws + lay.count_at))[at];
      const uint64_t m = row.masses ? ((const uint64_t*)(ws + lay.mass_at))[at] : 0;
      n += in ? c : 0;
      fixed += in ? m : 0;
    }
    scan_bins(s, n, (double)fixed * unit);
  }
  // First bin at which the sums cross; the last one that is not empty if none does.
  const auto bin_where = [&](int mode, double value) {
    const bool in = tid == 0 || s.count[tid] > s.count[tid - 1];
    return first_of(s, in && crossed(mode, value, s.count[tid], s.mass[tid]), in);
  };
  const uint32_t K = row.k > 0 ? min((uint32_t)row.k, live) : live;
  const bool masses = row.masses || bins.far;  // (whether the histogram has them)
  const float uf = a.u[b];
  const double u = uf > 0.f ? (double)uf : 0.0;

  // Top-k, top-p, min-p, the draw, and (where rounding has put it behind the cut) the last token before the cut, as
  // one sequence of passes over tokens.
  enum { FILL, PLAN, LIST, MASSES, NEXT, FIND, LEAST };
  Pass p{};
  p.top = top;
  p.bins = bins;
  p.z = (const char*)a.z + (size_t)b * a.stride * (BF16 ? 2 : 4);
  p.chunk_top = (const float*)(ws + lay.max_at);
  p.V = a.V;
  p.chunks = lay.chunks;
  int state = bins.far ? FILL : PLAN, step = -1;
  uint32_t binned = 0;
  bool cut_k = false, whole = false;
  float least = -INFINITY;          // the smallest logit that min-p leaves, and its bin
  int bm = BINS;
  int bk = BINS - 1, last = 0;      // bins of top-k's cut, and the last one that matters
  int f0 = 0, f1 = 0, f2 = 1, f3 = 0;
  bool in_list = false;             // bins f0 .. f1 and f2 .. f3 are in the list
  Sum cut{K, 0.0};
  uint32_t at_count = 0;            // of the draw's token: the count up to it, its logit, its id
  float at_z = top;
  int at_id = -1;
  // the search of FIND: bin i (BINS: what lies below them), tokens and units of it ahead of places lo .. hi, tokens in them
  int i = 0, mode = COUNT;
  double value = 0.0, mass0 = 0.0, scale = 0.0;
  uint32_t count0 = 0, n0 = 0, n = 0;
  uint64_t m0 = 0, lo = 0, hi = 0;
  bool listed = false, fresh = false;
#pragma unroll 1
  for (;;) {
    if (state == PLAN) {
      binned = uni(s.count[BINS - 1]);
      cut_k = K < live && K <= binned;
      if (row.least > 0.f) {
        const double low = uni(log((double)row.least));
        least = smallest((float)fmax((double)top + low * row.t, -(double)FLT_MAX), top, [&](float x) { return ((double)x - (double)top) * inv >= low; });
        bm = uni(index_of(least));
      }
      // the last bin that matters
      if (cut_k) bk = bin_where(COUNT, (double)K);
      last = bk;
      int bp = -1;
      if (row.p == 1.f || (masses && !cut_k)) {  // (else top-p's sum is that of the list)
        last = min(last, bm);
        // (a little beyond the threshold, whose last bits are another sum's)
        if (masses && row.p < 1.f) {
          bp = bin_where(REACH, (double)row.p * uni(s.mass[BINS - 1]) * (1.0 + 0x1p-40));
          last = min(last, bp);
        }
      }
      whole = uni(s.count[last]) <= (uint32_t)CAP;
      f0 = 0;
      f1 = last;
      in_list = whole;
      if (!whole && masses && !cut_k && row.least == 0.f) {
        // top-p's bin and those that the draw may fall into, if they fit
        const double most = uni(s.mass[BINS - 1]), part = row.p < 1.f ? (double)row.p * most * (1.0 - 0x1p-40) : most;
        f0 = bin_where(EXCEED, u * part);
        f1 = row.p < 1.f ? bin_where(EXCEED, u * uni(s.mass[bp])) : f0;
        if (bp > f1) f2 = f3 = bp;
        const uint32_t total = s.count[f1] - (f0 ? s.count[f0 - 1] : 0) + (bp > f1 ? s.count[bp] - s.count[bp - 1] : 0);
        in_list = uni(total) <= (uint32_t)CAP;
      }
      state = in_list ? LIST : masses ? NEXT : MASSES;
      if (state == NEXT) continue;
    }
    if (state == NEXT) {
      if (++step == 0) cut.mass = uni(s.mass[BINS - 1]);
      if (step == 5) break;
      // (u of 1 or more: the last token before the cut, which may lie below the bins)
      mode = step == 1 ? REACH : step == 3 && u < 1.0 ? EXCEED : COUNT;
      value = step == 0 ? (double)K : step == 1 ? (double)row.p * cut.mass : mode == EXCEED ? u * cut.mass : (double)cut.count;
      if (step == 0 && !cut_k) continue;
      if (step == 0 && uni(s.count[bk]) == K) {
        cut.mass = uni(s.mass[bk]);
        continue;
      }
      if (step == 1 && row.p == 1.f) continue;
      if (step == 2) {
        if (row.least > 0.f) state = LEAST;
        else continue;
      } else {
        if (step == 4 && at_count <= cut.count) break;
        i = mode == COUNT && value > (double)binned ? BINS : bin_where(mode, value);
        count0 = uni(i ? s.count[i - 1] : 0u);
        mass0 = uni(i ? s.mass[i - 1] : 0.0);
        scale = uni(exp64(-0.125 * i) * 0x1p-44);
        n = (i < BINS ? uni(s.count[i]) : live) - count0;
        n0 = 0;
        m0 = 0;
        listed = in_list && ((i >= f0 && i <= f1) || (i >= f2 && i <= f3));
        fresh = true;
        state = FIND;
      }
    }
    // the pass
    int b0 = i, b1 = i;
    if (state == LIST) {
      b0 = f0;
      b1 = f1;
    } else if (state == MASSES) {
      b0 = 0;
      b1 = last;
    } else if (state == LEAST) {
      b0 = b1 = bm;  // (BINS: tokens without a mass)
    } else if (state == FILL) {
      b0 = 0;
      b1 = BINS;
    }
    p.append = state == LIST;
    p.by_bin = state == MASSES || state == LEAST || state == FILL;
    p.listed = state == MASSES ? whole : state == LEAST ? in_list && f0 == 0 && bm <= f1 : false;
    p.lo = 0;
    p.hi = ~0ull;
    if (state != FIND || fresh) {
      p.z0 = low_edge(b1);
      p.z1 = high_edge(b0);
      p.z2 = INFINITY;
      p.z3 = -INFINITY;
      if (state == LIST && f3 >= f2) {
        p.z2 = low_edge(f3);
        p.z3 = high_edge(f2);
      }
      if (state == LEAST) p.z0 = least;
    }
    if (state == FIND) {
      if (fresh) {
        lo = place_of(p.z1, 0);
        hi = place_of(p.z0, (1 << ID_BITS) - 1);
        fresh = false;
      }
      p.append = !listed && n <= (uint32_t)CAP;
      p.listed = listed;
      p.lo = lo;
      p.hi = hi;
      p.sh = max(0, 64 - (int)__builtin_clzll((hi - lo) | 1) - 9);
    }
    if (state != FIND || !listed || n > 64) go_over<BF16>(s, p);

    if (state == FILL) {
      scan_bins(s, s.sub_count[tid], (double)s.sub_mass[tid] * unit);
      state = PLAN;
    } else if (state == LIST) {
      state = masses ? NEXT : MASSES;
    } else if (state == MASSES) {  // counted only until now
      const uint32_t c = s.count[tid] - (tid ? s.count[tid - 1] : 0);
      scan_bins(s, c, (double)s.sub_mass[tid] * unit);
      state = NEXT;
    } else if (state == LEAST) {
      // (tokens below the bins are counted in none of them)
      const uint32_t c = bm == BINS ? binned + s.rest : (bm ? s.count[bm - 1] : 0) + s.sub_count[bm];
      const double m = bm == BINS ? s.mass[BINS - 1] : (bm ? s.mass[bm - 1] : 0.0) + (double)s.sub_mass[bm] * (exp64(-0.125 * bm) * 0x1p-44);
      __syncthreads();
      if (uni(c) < cut.count) cut = Sum{uni(c), uni(m)};
      state = NEXT;
    } else if (p.append) {
      in_list = false;  // (this bin's tokens only)
      listed = true;
    } else if (!listed || n > 64) {
      const uint32_t mine = s.sub_count[tid];
      const uint64_t mass = s.sub_mass[tid];
      uint32_t c = mine;
      uint64_t m = mass;
      scan_both(s, c, m);
      const int who = first_of(s, mine > 0 && crossed(mode, value, count0 + n0 + c, mass0 + scale * (double)(m0 + m)), mine > 0);
      if (who >= THREADS) {  // (the logits have changed since the first kernel)
        state = NEXT;
        continue;
      }
      __syncthreads();
      if (tid == who) {
        s.at = mine;
        s.pos = c - mine;
        s.mass_at = m - mass;
      }
      __syncthreads();
      n = uni(s.at);
      n0 += uni(s.pos);
      m0 += uni(s.mass_at);
      lo += (uint64_t)who << p.sh;
      hi = min(hi, lo + ((1ull << p.sh) - 1));
    } else {
      // the last few, in one wave
      __syncthreads();
      if (tid == 0) s.pos = 0;
      __syncthreads();
#pragma unroll 1
      for (uint32_t t = tid; t < s.n; t += THREADS) {
        const uint64_t q = s.list[t];
        if (q >= lo && q <= hi) {
          const uint32_t to = atomicAdd(&s.pos, 1u);
          if (to < 64) s.few[to] = q;
        }
      }
      __syncthreads();
      const int len = (int)min(uni(s.pos), 64u);
      state = NEXT;
      if (len == 0) continue;
      __syncthreads();
      if (wave == 0) {
        // a token's rank is the number of those ahead of it, and so are its sums
        const uint64_t q = lane < len ? s.few[lane] : ~0ull;
        const uint64_t e = lane < len ? units_in_bin(bins, place_z(q), i) : 0;
        uint32_t rank = 0;
        uint64_t m = m0 + e;
#pragma unroll 1
        for (int x = 0; x < len; ++x) {
          const uint64_t other = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(q >> 32), x) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)q, x);
          const uint64_t units = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(e >> 32), x) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)e, x);
          rank += other < q ? 1 : 0;
          m += other < q ? units : 0;
        }
        const uint64_t yes = __ballot(lane < len && crossed(mode, value, count0 + n0 + rank + 1, mass0 + scale * (double)m));
        // (once crossed, all later ones are: the first of them is as many from the end as there are)
        const uint32_t at = len - (yes ? __builtin_popcountll(yes) : 1);
        if (lane < len && rank == at) {
          s.place = q;
          s.mass_at = m;
          s.pos = n0 + rank + 1;
        }
      }
      __syncthreads();
      const Sum sum{count0 + uni(s.pos), mass0 + scale * (double)uni(s.mass_at)};
      const uint64_t found = uni(s.place);
      if (step >= 3) {
        at_count = sum.count;
        at_z = place_z(found);
        at_id = place_id(found);
      } else if (step == 0 || sum.count < cut.count) {
        cut = sum;
      }
    }
  }
  // the mass at the centre of the first bin relative to the largest logit's
  const double c = -place_in_bin(bins, top, 0);
  const double e = exp64(-fabs(c)), mine = exp64(((double)at_z - (double)top) * inv);
  answer(at_id, c < 0 ? mine / (cut.mass * e) : mine * e / cut.mass, cut.count);
}

template <bool BF16>
hipError_t launch(const SampleArgs& a, hipStream_t s) {
  const Layout lay = layout_of(a.B, a.V);
  const int grid = a.B * lay.pieces;
  if (lay.g8 == 4) sample_hist_kernel<BF16, 4><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  else if (lay.g8 == 2) sample_hist_kernel<BF16, 2><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  else sample_hist_kernel<BF16, 1><<<grid, HIST_THREADS, 0, s>>>(a, lay);
  sample_kernel<BF16><<<a.B, THREADS, 0, s>>>(a, lay);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace(int B, int V) { return layout_of(B, V).row * (size_t)B; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) { return a.bf16 ? launch<true>(a, s) : launch<false>(a, s); }

}  // namespace pmpe
