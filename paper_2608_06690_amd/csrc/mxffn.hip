// Expert FFN on 8-bit operands: activations in e4m3 with a power-of-two scale for every 32 values of
// a row (mx.h), weights in e4m3 with a power-of-two scale per weight row.
//
//   GEMM1  [rows, H] x [H, 2I]: a tile holds BN/2 gate and the matching up columns; h = silu(g) u is
//          formed in registers and leaves in the activations' format: a wave holds 32 consecutive
//          h columns of a row in the four lanes that share it, so the block scale costs two
//          lane exchanges
//   GEMM2  [rows, I] x [I, H] -> y_perm (bf16), and the execution audit
//
// v_mfma_scale_f32_16x16x128_f8f6f4: one instruction multiplies 128 values of K, twice the rate of the
// bf16 instruction, and applies the block scales of the activations itself (lane l carries the scale
// of row l % 16 and of the 32 values 32 (l / 16) .. + 31 of the step; its data are the 16-byte chunks
// l / 16 and 4 + l / 16). The weights' row scales are powers of two and multiply the accumulators.
// The weight fragment is the first operand, and the weight rows of a 32-row block are permuted in
// LDS, so that a lane's results are 8 consecutive output columns of one row.
//
// Precision: the accumulators are fp32. Inside the instruction the products of 8 consecutive k are
// aligned to the largest of them and what lies below 2^-13 of its power of two is dropped (measured);
// on random rows that leaves a sum within 1.2e-5 of the sum of magnitudes, far below the rounding of h
// to e4m3 and of y to bf16. Widening both operands to bf16 would keep every bit at half the rate.
//
// A K step is 128 values (whole 128-byte lines of every row); its operands and the rows' four scale
// bytes go through a ring of global->LDS copies that runs on across tile boundaries. Tile list,
// XCD mapping and row gather as in the bf16 kernels.
#include <type_traits>

#include "lds_dma.h"
#include "mx.h"
#include "pmpe_internal.h"

namespace pmpe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
constexpr int MAXE = 2 * PMPE_MAX_POOL;

template <int BM_, int BN_, int WM_, int WN_, int STAGES_, bool NT_, int SPC_>
struct MxCfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr bool NT = NT_;  // weights are read once: keep them from evicting the activations
  // Steps whose scale bytes one copy brings: 64 / SPC rows of a wave. A row's are neighbours in memory, so
  // four steps cost a request per row where four copies cost four.
  static constexpr int SPC = SPC_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, SC_BYTES = BM * 4 * SPC;
  static constexpr int STAGE = A_BYTES + B_BYTES;
  static constexpr int A_DMA = BM / 8 / WAVES, B_DMA = BN / 8 / WAVES, NDMA = A_DMA + B_DMA;
  static constexpr int SC_WAVES = BM * SPC / 64;  // waves that copy scales
  static constexpr int MB = BM / WM / 16;  // 16-row blocks of a wave: blocks j * WM + wm
  // gather slices: a tile's is copied two tiles before its first step is issued (a tile may have one
  // step), and the audit reads it when the tile ends; scale slices: one tile before their use
  static constexpr int NRT = STAGES + 2, NWS = STAGES;
  // a copy's steps are one at least and the producer is STAGES - 1 steps ahead: STAGES buffers
  static constexpr int LDS = STAGES * (STAGE + SC_BYTES) + NRT * BM * 4 + NWS * BN * 4 + (MAXE + 1) * 8;
  static_assert(A_DMA * 8 * WAVES == BM && B_DMA * 8 * WAVES == BN, "copy split");
  static_assert(SC_WAVES <= WAVES && SC_WAVES * 64 == BM * SPC, "scale copies");
  static_assert(BM <= 64 * WAVES && BN <= 64 * WAVES, "one slice copy per wave");
};

struct MxTile {
  int g, m0, n0, rows, base;
};

template <class C, bool GATED>
__global__ __launch_bounds__(C::THREADS) void mx_gemm_kernel(MxFfnArgs a) {
  constexpr int BM = C::BM, BN = C::BN, S = C::STAGES, MB = C::MB, NRT = C::NRT, NWS = C::NWS;
  constexpr int NCOLS = GATED ? BN / 2 : BN;  // output columns of a tile
  constexpr int WC = NCOLS / C::WN;           // of a wave
  constexpr int NQ = WC / 32;                 // its 32-column groups
  constexpr int NB = (GATED ? 2 : 1) * WC / 16;
  static_assert(WC % 32 == 0, "a wave holds whole 32-column groups");
  __shared__ __attribute__((aligned(16))) unsigned char smem[S * C::STAGE];
  __shared__ __attribute__((aligned(16))) uint8_t s_sc[S][C::SC_BYTES];  // [buffer][row][step]: four bytes
  __shared__ __attribute__((aligned(16))) int s_rt[NRT][BM];
  __shared__ __attribute__((aligned(16))) float s_ws[NWS][BN];
  __shared__ int s_cum[MAXE + 1];
  __shared__ int s_off[MAXE + 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  const int E = a.n_pub + a.n_priv, H = a.H, I = a.I;
  const int TK = a.T * a.k;
  const int K = GATED ? H : I, width = GATED ? I : H;
  const int ntn = (width + NCOLS - 1) / NCOLS;

  // tiles of the experts before expert g, and the experts' first rows
  for (int i = tid; i <= E; i += C::THREADS) s_off[i] = a.offset[i];
  __syncthreads();
  if (tid < 64) {
    int running = 0;
    for (int g0 = 0; g0 < E; g0 += 64) {
      const int g = g0 + tid;
      const int nt = g < E ? (s_off[g + 1] - s_off[g] + BM - 1) / BM * ntn : 0;
      const int incl = wave_incl_scan(nt);
      if (g < E) s_cum[g + 1] = running + incl;
      running += __shfl(incl, 63, 64);
    }
    if (tid == 0) s_cum[0] = 0;
  }
  __syncthreads();
  const int total = s_cum[E];
  const int b = blockIdx.x, x = b & 7, q = b >> 3;
  const int nbx = ((int)gridDim.x - x + 7) >> 3;
  const int cnt_x = (total >> 3) + (x < (total & 7) ? 1 : 0);
  const int start_x = x * (total >> 3) + min(x, total & 7);
  const int ntl = (cnt_x > q && q < nbx) ? (cnt_x - q + nbx - 1) / nbx : 0;
  if (ntl == 0) return;

  auto tile_of = [&](int i) {
    const int L = start_x + q + i * nbx;
    int lo = 0, hi = E - 1;  // last expert with s_cum[g] <= L (one with tiles)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_cum[mid] <= L) lo = mid; else hi = mid - 1;
    }
    MxTile t;
    t.g = __builtin_amdgcn_readfirstlane(lo);
    const int off = __builtin_amdgcn_readfirstlane(s_off[t.g]);
    const int cnt = __builtin_amdgcn_readfirstlane(s_off[t.g + 1]) - off;
    const int mt = (cnt + BM - 1) / BM, local = L - __builtin_amdgcn_readfirstlane(s_cum[t.g]);
    const int n = local / mt, m = local - n * mt;
    t.m0 = m * BM;
    t.n0 = n * NCOLS;
    t.rows = min(BM, cnt - t.m0);
    t.base = off + t.m0;
    return t;
  };
  auto is_private = [&](const MxTile& t) { return t.g >= a.n_pub; };
  auto has_weights = [&](const MxTile& t) { return !(is_private(t) && (a.w13_priv == nullptr || a.w2_priv == nullptr)); };

  const uint32_t lds0 = lds_addr(smem), sc0 = lds_addr(&s_sc[0][0]);
  const uint32_t rt0 = lds_addr(&s_rt[0][0]), ws0 = lds_addr(&s_ws[0][0]);
  // row_token of tile i's rows (GEMM1 gathers by it, GEMM2's audit reads it), clamped into the array
  auto issue_rt = [&](int i) {
    if (i >= ntl) return;
    const MxTile t = tile_of(i);
    if (wave < BM / 64 && (GATED || is_private(t)))
      dma4(a.row_token + min(t.base + wave * 64 + lane, TK - 1), rt0 + ((i % NRT) * BM + wave * 64) * 4);
  };
  // weight row of tile B row r (clamped past the width)
  auto weight_row = [&](const MxTile& t, int r) {
    if (GATED) return r < BN / 2 ? min(t.n0 + r, I - 1) : I + min(t.n0 + r - BN / 2, I - 1);
    return min(t.n0 + r, H - 1);
  };
  auto issue_ws = [&](const MxTile& t, int i) {
    const bool pub = !is_private(t) || !has_weights(t);
    const float* s = pub ? (GATED ? a.w13s_pub : a.w2s_pub) : (GATED ? a.w13s_priv : a.w2s_priv);
    const int g = is_private(t) ? (pub ? 0 : t.g - a.n_pub) : t.g;
    if (wave < BN / 64)
      dma4(s + (size_t)g * (GATED ? 2 * I : H) + weight_row(t, wave * 64 + lane), ws0 + ((i % NWS) * BN + wave * 64) * 4);
  };

  // Copies of this lane: copy i of a wave fills 8 rows; 16-byte chunk c of LDS row r holds logical
  // chunk c ^ (r & 7), so that fragment reads of 8 consecutive rows at one chunk cover the banks once.
  const int crow = lane >> 3;
  const uint32_t cchunk = (uint32_t)(((lane & 7) ^ crow) * 16);
  // weight row (within 32) held by an LDS row: row 16 nb + j holds 8 (j / 4) + 4 nb + j % 4
  auto bperm = [](int r) { return (r & ~31) + 8 * ((r >> 2) & 3) + 4 * ((r >> 4) & 1) + (r & 3); };
  uint32_t offA[C::A_DMA], offB[C::B_DMA];
  const unsigned char* baseB = nullptr;
  uint32_t offS = 0;  // this lane's scales: row wave * 64 / SPC + lane / SPC
  auto setup = [&](const MxTile& t, int i) {
    const size_t per = (size_t)(GATED ? 2 : 1) * I * H;
    const unsigned char* w = (const unsigned char*)(GATED ? a.w13_pub : a.w2_pub);
    if (!is_private(t))
      w += (size_t)t.g * per;
    else if (has_weights(t))
      w = (const unsigned char*)(GATED ? a.w13_priv : a.w2_priv) + (size_t)(t.g - a.n_pub) * per;
    // (private rows without private weights: the copies read public rows, nothing is computed)
    baseB = w;
    auto row_of = [&](int r) {
      const int rr = min(r, t.rows - 1);  // rows past the valid count reload a valid row
      return GATED ? (uint32_t)s_rt[i % NRT][rr] : (uint32_t)(t.base + rr);
    };
#pragma unroll
    for (int j = 0; j < C::A_DMA; ++j) offA[j] = row_of((wave * C::A_DMA + j) * 8 + crow) * (uint32_t)K + cchunk;
#pragma unroll
    for (int j = 0; j < C::B_DMA; ++j)
      offB[j] = (uint32_t)weight_row(t, bperm((wave * C::B_DMA + j) * 8 + crow)) * (uint32_t)K + cchunk;
    offS = row_of(min((wave * 64 + lane) / C::SPC, BM - 1)) * (uint32_t)(K / 32);
    return K / 128;
  };
  const unsigned char* baseA = (const unsigned char*)(GATED ? a.xq : a.hq);
  auto issue = [&](int slot, int step) {
    const uint32_t st = __builtin_amdgcn_readfirstlane(lds0 + slot * C::STAGE);
    const uint32_t wa = st + wave * C::A_DMA * 1024, wb = st + C::A_BYTES + wave * C::B_DMA * 1024;
    const unsigned char *ba = baseA + step * 128, *bb = baseB + step * 128;
    Unroll<0, C::A_DMA>::run([&](auto j) { dma16s<j.value * 1024, false>(offA[j.value], ba, wa); });
    Unroll<0, C::B_DMA>::run([&](auto j) { dma16s<j.value * 1024, C::NT>(offB[j.value], bb, wb); });
  };

  int pi = 0, pk = 0, pnk = 0, issued = 0, pq = 0;
  // The next SPC steps' scales, ahead of the first of them (the waits count the operands' copies only:
  // one more in flight makes them wait for one more).
  auto issue_scales = [&]() {
    if (wave < C::SC_WAVES)
      dma4s(offS + 4 * (uint32_t)min(pk + lane % C::SPC, pnk - 1), GATED ? a.xs : a.hs, sc0 + pq * C::SC_BYTES + wave * 256);
    pq = pq == S - 1 ? 0 : pq + 1;
  };
  issue_rt(0);
  issue_rt(1);
  wait_vmcnt<0>();
  __syncthreads();
  {
    const MxTile t = tile_of(0);
    issue_rt(2);
    issue_ws(t, 0);
    pnk = setup(t, 0);
  }
  auto produce = [&](int slot) {
    if (pi >= ntl) return;
    if (pk == pnk) {
      ++pi;
      pk = 0;
      if (pi >= ntl) return;
      const MxTile t = tile_of(pi);
      issue_rt(pi + 2);
      issue_ws(t, pi);
      pnk = setup(t, pi);
    }
    if (pk % C::SPC == 0) issue_scales();
    issue(slot, pk);
    ++pk;
    ++issued;
  };
#pragma unroll
  for (int s = 0; s < S - 1; ++s) produce(s);

  const int g4 = lane >> 4, r16 = lane & 15;
  const uint32_t lane_off = (uint32_t)(r16 * 128 + ((g4 ^ (lane & 7)) << 4));
  auto frag = [&](uint32_t p) {
    const u32x4 lo = *(const u32x4*)(smem + p), hi = *(const u32x4*)(smem + (p ^ 64));
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  int gs = 0, cq = 0;
  auto tile_body = [&](auto mbl, const MxTile& ct, int ci, int live) {
    constexpr int MBL = decltype(mbl)::value;
    f32x4 acc[MBL][NB];
#pragma unroll
    for (int mb = 0; mb < MBL; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = f32x4{0, 0, 0, 0};
    const int nk = K / 128;
    for (int kc = 0; kc < nk; ++kc, ++gs) {
      // this wave's copies of step gs are done (younger steps may be in flight) ...
      if (issued - 1 - gs >= S - 2)
        wait_vmcnt<(S - 2) * C::NDMA>();
      else
        wait_vmcnt<0>();
      // ... and every other wave's; every read of step gs - 1 is finished
      barrier_raw();
      produce((gs + S - 1) % S);
      if (live > 0) {
        const uint32_t st = (uint32_t)(gs % S) * C::STAGE;
        i32x8 fa[MBL], fb[NB];
        int sc[MBL];
#pragma unroll
        for (int mb = 0; mb < MBL; ++mb) {
          const uint32_t row0 = (uint32_t)(mb * C::WM + wm) * 16;
          fa[mb] = frag(st + row0 * 128 + lane_off);
          sc[mb] = s_sc[cq][(row0 + r16) * 4 * C::SPC + kc % C::SPC * 4 + g4];
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int col = GATED ? (nb < NB / 2 ? nb * 16 : BN / 2 + (nb - NB / 2) * 16) : nb * 16;
          fb[nb] = frag(st + C::A_BYTES + (wn * WC + col) * 128 + lane_off);
        }
#pragma unroll
        for (int mb = 0; mb < MBL; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            acc[mb][nb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[nb], fa[mb], acc[mb][nb], 0, 0, 0, 0x7F7F7F7F,
                                                                           0, sc[mb]);
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's reads of the slot are done
      }
      if (kc % C::SPC == C::SPC - 1 || kc == nk - 1) cq = cq == S - 1 ? 0 : cq + 1;
    }
    if (!has_weights(ct)) return;
    // Output: lane l holds columns 8 (l / 16) .. + 7 of each 32-column group, row l % 16 of a block.
    const float* ws = s_ws[ci % NWS];
#pragma unroll
    for (int mb = 0; mb < MBL; ++mb) {
      const int r = (mb * C::WM + wm) * 16 + r16;
      if (mb >= live) continue;  // (wave-uniform)
#pragma unroll
      for (int p = 0; p < NQ; ++p) {
        const int c = wn * WC + p * 32 + g4 * 8;
        const f32x4 s0 = *(const f32x4*)(ws + c), s1 = *(const f32x4*)(ws + c + 4);
        const f32x4 v0 = acc[mb][2 * p] * s0, v1 = acc[mb][2 * p + 1] * s1;
        const size_t row = (size_t)(ct.base + r);
        const int col = ct.n0 + c;
        if constexpr (GATED) {
          const f32x4 t0 = *(const f32x4*)(ws + BN / 2 + c), t1 = *(const f32x4*)(ws + BN / 2 + c + 4);
          const f32x4 u0 = acc[mb][NB / 2 + 2 * p] * t0, u1 = acc[mb][NB / 2 + 2 * p + 1] * t1;
          float h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = mx_silu(v0[e]) * u0[e];
            h[4 + e] = mx_silu(v1[e]) * u1[e];
          }
          const float amax = mx_max_rows(mx_amax8(h));
          if (r < ct.rows && col < width) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            uint32_t q0, q1;
            const int e = mx_pack8(h, amax, q0, q1);
            *(u32x2*)(a.hq + row * I + col) = u32x2{q0, q1};
            if (g4 == 0) a.hs[row * (I / 32) + (col >> 5)] = (uint8_t)(e + 127);
          }
        } else if (r < ct.rows && col < width) {
          *(u32x4*)((uint16_t*)a.y_perm + row * H + col) =
              u32x4{pack_bf16x2(v0[0], v0[1]), pack_bf16x2(v0[2], v0[3]), pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3])};
        }
      }
    }
  };

  for (int ci = 0; ci < ntl; ++ci) {
    const MxTile ct = tile_of(ci);
    const bool valid = has_weights(ct);
    const int nblk = (ct.rows + 15) / 16;
    const int live = valid ? max(0, min(MB, (nblk - wm + C::WM - 1) / C::WM)) : 0;
    if (MB >= 2 && live <= MB / 2)
      tile_body(std::integral_constant<int, (MB >= 2 ? MB / 2 : MB)>{}, ct, ci, live);
    else
      tile_body(std::integral_constant<int, MB>{}, ct, ci, live);
    if constexpr (!GATED) {
      if (!valid) {
        // private rows without private weights: not executed, not audited, y zeroed
        if (tid == 0 && a.dev_status) atomicOr(a.dev_status, PMPE_DEV_PRIV_WEIGHTS_MISSING);
        for (int i = tid; i < ct.rows * (NCOLS / 8); i += C::THREADS) {
          const int r = i / (NCOLS / 8), c = ct.n0 + (i - r * (NCOLS / 8)) * 8;
          if (c < width) *(u32x4*)((uint16_t*)a.y_perm + (size_t)(ct.base + r) * H + c) = u32x4{0, 0, 0, 0};
        }
      } else if (is_private(ct) && ct.n0 == 0) {
        // execution audit: the first N tile of every private M tile counts its rows
        for (int r = tid; r < ct.rows; r += C::THREADS) atomicAdd(&a.audit_rows[s_rt[ci % NRT][r]], 1u);
        if (ct.m0 == 0 && tid == 0 && a.audit_calls) atomicAdd(&a.audit_calls[ct.g - a.n_pub], 1u);
      }
    }
  }
  wait_vmcnt<0>();  // no copy may still be writing LDS when the block exits
}

int cu_count() {
  int dev = 0, v = 0;
  if (hipGetDevice(&dev) == hipSuccess &&
      hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0)
    return v;
  return 256;
}

using MxSmall = MxCfg<64, 128, 2, 2, 3, true, 1>;  // two blocks per CU
using MxMid = MxCfg<128, 256, 2, 4, 3, false, 4>;

template <class C, bool GATED>
hipError_t launch(const MxFfnArgs& a, hipStream_t s) {
  constexpr int NCOLS = GATED ? C::BN / 2 : C::BN, PER_CU = (160 * 1024) / ((C::LDS + 1279) / 1280 * 1280);
  static_assert(PER_CU >= 1, "LDS");
  const int64_t w = GATED ? a.I : a.H;
  // at most one partly filled M tile per expert
  const int64_t tiles = ((int64_t)a.T * a.k / C::BM + a.n_pub + a.n_priv) * ((w + NCOLS - 1) / NCOLS);
  int64_t grid = (int64_t)cu_count() * PER_CU;
  if (tiles < grid) grid = (tiles + 7) / 8 * 8;
  hipLaunchKernelGGL((mx_gemm_kernel<C, GATED>), dim3((unsigned)grid), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_ffn_mx(const MxFfnArgs& a, hipStream_t s) {
  // Rows per expert, on average, choose the tile; us of both products (160 experts of 2048 x 768 / 52 of
  // 1664 x 640 / 80 of 2048 x 1408), all experts alike:
  //   rows                 48            56            64            96            128           192           384
  //   64 x 128     163  53 148   186  55 161   237  67 206   315  81 281   356  90 315   510 120 452   870 188 740
  //   128 x 256    171  63 153   174  65 156   178  62 160   196  69 177   251  78 224   317  92 271   540 136 446
  //   256 x 256    196  80 180   202  82 183   202  79 187   220  83 198   227  91 211   266 101 243   449 137 372
  // (32 rows: 149, 51, 130 and 165, 61, 148 with the two smaller.) 52 rows is the line of the two layers that
  // fill the chip; the 52 experts, with about one large tile per CU, would have theirs at about 60 and lose 10 us at
  // 56 rows. The large kernel needs a few tiles per
  // CU (the 52 experts give it one or two), and two K steps.
  const int64_t E = a.n_pub + a.n_priv, rows = (int64_t)a.T * a.k / E;
  hipError_t e;
  if (rows < 52) {
    e = launch<MxSmall, true>(a, s);
    return e != hipSuccess ? e : launch<MxSmall, false>(a, s);
  }
  const int64_t large_tiles = E * ((rows + 255) / 256) * (a.I / 128);
  if (rows >= 120 && large_tiles >= 3 * cu_count() && a.H >= 256 && a.I >= 256) {
    FfnArgs f{};
    f.T = a.T; f.H = a.H; f.I = a.I; f.n_pub = a.n_pub; f.n_priv = a.n_priv; f.k = a.k;
    f.x = a.xq; f.x_scale = a.xs; f.count = a.count; f.offset = a.offset; f.row_token = a.row_token;
    f.w13_pub = a.w13_pub; f.w2_pub = a.w2_pub; f.w13_priv = a.w13_priv; f.w2_priv = a.w2_priv;
    f.w13_scale_pub = a.w13s_pub; f.w2_scale_pub = a.w2s_pub; f.w13_scale_priv = a.w13s_priv; f.w2_scale_priv = a.w2s_priv;
    f.y_perm = a.y_perm; f.audit_rows = a.audit_rows; f.audit_calls = a.audit_calls; f.dev_status = a.dev_status;
    f.h = a.hq; f.h_scale = a.hs;
    return launch_gemm256_mx(f, s);
  }
  e = launch<MxMid, true>(a, s);
  return e != hipSuccess ? e : launch<MxMid, false>(a, s);
}

}  // namespace pmpe
