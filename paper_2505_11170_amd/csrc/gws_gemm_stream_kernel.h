// The kernel for few rows of X (gws_gemm_stream.hip says what it is and what bounds it), also for those that do something else with its sums (internal
// to csrc/).
#pragma once

#include "gws_gemm_stream_core.h"

namespace gws {

// What the kernel keeps from the start for its way out: nothing.
struct NothingHeldStream {};
template <int MT, int NT, int P, int BM, int BN>
__device__ __forceinline__ NothingHeldStream before_stream(const GemmArgs&, uint32_t, uint32_t) { return {}; }

template <int MT, int NT, int P, int BM, int BN>
void finish_stream();   // the way outs' (gws_dense_out.h)

// A wavefront's share of a tile's columns of the weight, fetched into the XCD's L2 and dropped: one load instruction touches 64 pieces
// of lines, every part-th unit of 64 k.  A compute unit gets about 60 B/ns from beyond its L2, a line every 2 ns whether 64 bytes of it are
// wanted or 128, so few tiles on few compute units wait for the weight while the others idle; what an idle one has fetched comes at 150.
// A wavefront has one load on its way: the empty statement uses its register, so the next one waits for it.  How many workgroups a tile
// fetch (stream_plan) is fitted to that.
template <int BN, bool W_NK>
__device__ __forceinline__ void warm_l2(const GemmArgs& g, uint32_t n0, uint32_t u0, uint32_t u1, uint32_t part, uint32_t parts) {
  const uint32_t lane = threadIdx.x & 63;
  constexpr uint32_t UNITS = W_NK ? 64 / BN : 1;   // of an instruction
  for (uint32_t u = u0 + part * UNITS; u < u1; u += parts * UNITS) {
    const uint32_t k = stream::umin(64 * (u + (W_NK ? lane / BN : 0)), g.K - 64);
    const uint32_t v = *(const uint32_t*)(W_NK ? g.w + (size_t)stream::umin(n0 + lane % BN, g.N - 1) * g.ldw + k : g.w + (size_t)(k + lane) * g.ldw + n0);
    asm volatile("" ::"v"(v));
  }
}

// A wavefront keeps D units of 64 k on their way into its own ring of LDS stages (global_load_lds_dwordx4, 8 rows x 128
// contiguous bytes per instruction).  Loaded straight into the MFMA's register layout instead (16 rows x 64 bytes: a
// quarter-wavefront touches 16 cache lines for 16 bytes each) a compute unit takes 39 B/ns whatever is in flight; in this
// form 130-180 B/ns (L2-resident operands, one workgroup per compute unit).  Layouts as in gws_gemm256_core.h: rows of 128
// bytes with chunk c of row r in slot c ^ ((r / 2) % 8); a [K x N] weight as 64 k-rows of 32 NT bytes, read with the
// transposing LDS load, chunk c of row k in slot c ^ swizzle(k).
// WARM: the grid has more workgroups a tile (blockIdx.y > 0) that only warm_l2; they share nothing with the others.
// BM x BN is the workgroup's tile: 16 MT x 16 NT, or eight rows, eight columns where one MFMA tile has that many of use (the others
// are computed on repeated ones and not stored).  Without `way_out` the kernel stores Y; with one (its functions: before_stream, finish_stream) that takes the
// partial sums instead.
template <int MT, int NT, int P, int D, bool W_NK, int BM = 16 * MT, int BN = 16 * NT, bool WARM = false, class... WayOut>
__global__ __launch_bounds__(64 * P) void gemm_stream_kernel(GWS_GEMM_PARAMS, const WayOut... way_out) {
  using namespace stream;
  const GemmArgs g = GWS_GEMM_GATHER({});
  static_assert((BM == 16 * MT || (BM == 8 && MT == 1)) && (BN == 16 * NT || (BN == 8 && NT == 1 && W_NK)), "whole MFMA tiles or half a one");
  constexpr int XS = BM * 64, WS = BN * 64, STG = XS + WS;          // elements of a stage
  constexpr int QX = BM / 8, QW = BN / 8, LOADS = QX + QW;          // load instructions of a unit
  static_assert(LOADS * (D - 1) <= 63, "the wait for a unit counts the loads behind it");
  static_assert(W_NK || NT == 2 || NT == 4 || NT == 8, "swizzle of the [K x N] stage");
  constexpr int MC = MT > 4 ? 4 : MT;                               // row tiles of a pass of the reduction
  constexpr int kRing = P * D * STG * 2, kRed = red_bytes(MC, NT, P);
  __shared__ __attribute__((aligned(1024))) char lds[kRing > kRed ? kRing : kRed];
  const uint32_t lane = threadIdx.x & 63, li = lane & 15, grp = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* ring = (uint16_t*)lds + wave * (D * STG);
  const TileGrid t = {(g.M + BM - 1) / BM, (g.N + BN - 1) / BN, g.inv_band, g.inv_last};
  uint32_t m0, n0;
  if (t.joined()) tile_of_joined(t, blockIdx.x, m0, n0);   // StreamPlan::parts
  else tile_of_groups(t, !W_NK && NT == 2, blockIdx.x, m0, n0);
  m0 *= BM;
  n0 *= BN;
  uint32_t u0, u1;
  unit_range(g.K, wave, P, u0, u1);
  if (WARM && (blockIdx.y > 0 || blockIdx.x >= t.mt * t.nt)) {   // uniform; a row of the grid is whole rounds of the XCDs
    if (blockIdx.x < t.mt * t.nt) warm_l2<BN, W_NK>(g, n0, u0, u1, blockIdx.y - 1, gridDim.y - 1);
    return;
  }

  [[maybe_unused]] auto held = before_stream<MT, NT, P, BM, BN>(g, m0, n0, way_out...);

  // lane offsets in bytes; rows and columns past the edge are read from the last ones and not stored
  uint32_t xo[QX], wo[W_NK ? QW : 1];
#pragma unroll
  for (int q = 0; q < QX; ++q)
    xo[q] = (umin(8u * q + (lane >> 3), g.M - 1 - m0) * g.ldx + ((lane & 7) ^ (4 * (q & 1) + (lane >> 4))) * 8) * 2;
  if (W_NK) {
#pragma unroll
    for (int q = 0; q < QW; ++q)
      wo[q] = (umin(8u * q + (lane >> 3), g.N - 1 - n0) * g.ldw + ((lane & 7) ^ (4 * (q & 1) + (lane >> 4))) * 8) * 2;
  }
  // [K x N]: an instruction covers RPI k-rows of 2 NT chunks
  constexpr uint32_t CPR = 2 * NT, RPI = 64 / CPR;
  const uint32_t wk = lane / CPR, ws = lane % CPR;
  const GWS_GLOBAL char* xb = (const GWS_GLOBAL char*)(g.x + (size_t)m0 * g.ldx);
  const GWS_GLOBAL char* wb = (const GWS_GLOBAL char*)(W_NK ? g.w + (size_t)n0 * g.ldw : g.w + n0);
  const uint32_t last_chunk = (g.N - n0) / 8 - 1;
  constexpr int NV = W_NK ? 1 : 16 / RPI;   // the swizzle depends on k % 16
  uint32_t wv[NV];
  if (!W_NK) {
#pragma unroll
    for (int v = 0; v < NV; ++v) wv[v] = (wk * g.ldw + umin(ws ^ oc_swizzle<W_NK ? 2 : NT>(wk + RPI * v), last_chunk) * 8) * 2;
  }
  auto load = [&](uint32_t u, uint32_t slot) {
    uint16_t* st = ring + slot * STG;
    const uint32_t k0 = umin(64 * u, g.K - 64);   // the half unit at the end of K is fetched as the second half of a whole one
#pragma unroll
    for (int q = 0; q < QW; ++q) {
      if (W_NK) direct(wb + (size_t)k0 * 2, wo[q], st + XS + q * 512);
      else direct(wb + (size_t)(k0 + RPI * q) * g.ldw * 2, wv[q % NV], st + XS + q * 512);
    }
#pragma unroll
    for (int q = 0; q < QX; ++q) direct(xb + (size_t)k0 * 2, xo[q], st + q * 512);
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t n = u1 - u0;
#pragma unroll
  for (int d = 0; d < D; ++d)
    if ((uint32_t)d < n) load(u0 + d, d);
  uint32_t slot = 0;
  const uint32_t lx = BM == 8 ? li & 7 : li, lw = BN == 8 ? li & 7 : li;
  for (uint32_t i = 0; i < n; ++i) {
    if (i + D <= n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS * (D - 1)) : "memory");   // the unit has landed
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const uint16_t* xs = ring + slot * STG;
    const uint16_t* wsg = xs + XS;
    Frag8 fx[2][MT], fw[2][NT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int r = 0; r < MT; ++r) fx[h][r].u = *(const u32x4*)(xs + (16 * r + lx) * 64 + (((4 * h + grp) ^ ((lx >> 1) & 7)) * 8));
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (W_NK) {
          fw[h][j].u = *(const u32x4*)(wsg + (16 * j + lw) * 64 + (((4 * h + grp) ^ ((lw >> 1) & 7)) * 8));
        } else {
          fw[h][j] = read_oc<W_NK ? 2 : NT>(wsg, h, j, li, grp);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read: the stage can be filled again
    __builtin_amdgcn_sched_barrier(0);
    if (i + D < n) load(u0 + i + D, slot);
    slot = slot + 1 == D ? 0 : slot + 1;
    const bool half = 64 * (u0 + i) + 64 > g.K;   // only the second half of the stage belongs to this unit
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 0 && half) continue;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < MT; ++r) acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[h][j].v, fx[h][r].v, acc[r][j], 0, 0, 0);
    }
  }
  if constexpr (sizeof...(WayOut) > 0) finish_stream<MT, NT, P, BM, BN>(g, acc, held, lds, m0, n0, way_out...);
  else reduce_store<MT, NT, P, MC, BM, BN>(acc, lds, g, m0, n0);
}

// WARM_KN, WARM_NK: the forms that stream_plan lets warm the L2
template <int MT, int NT, int P, int D, int BM = 16 * MT, int BN = 16 * NT, bool WARM_KN = false, bool WARM_NK = false, class... WayOut>
inline void launch_plain(GemmArgs g, int w_is_nk, const StreamPlan& p, hipStream_t s, const WayOut&... way_out) {
  const int warm = WARM_KN || WARM_NK ? p.warm : 0;
  const dim3 tiles(stream::tile_grid(g, BM, BN, p.parts != 0)), grid(warm ? (tiles.x + 7) / 8 * 8 : tiles.x, 1 + warm), block(64 * P);
  if constexpr (WARM_NK) {
    if (w_is_nk && warm) {
      hipLaunchKernelGGL((gemm_stream_kernel<MT, NT, P, D, true, BM, BN, true, WayOut...>), grid, block, 0, s, GWS_GEMM_PASS(g), way_out...);
      return;
    }
  }
  if constexpr (WARM_KN) {
    if (!w_is_nk && warm) {
      hipLaunchKernelGGL((gemm_stream_kernel<MT, NT, P, D, false, BM, BN, true, WayOut...>), grid, block, 0, s, GWS_GEMM_PASS(g), way_out...);
      return;
    }
  }
  if (w_is_nk) {
    hipLaunchKernelGGL((gemm_stream_kernel<MT, NT, P, D, true, BM, BN, false, WayOut...>), tiles, block, 0, s, GWS_GEMM_PASS(g), way_out...);
  } else if constexpr (NT >= 2) {
    hipLaunchKernelGGL((gemm_stream_kernel<MT, NT, P, D, false, BM, BN, false, WayOut...>), tiles, block, 0, s, GWS_GEMM_PASS(g), way_out...);
  }
}

template <class... WayOut>
inline int launch_stream_tiles(const GemmArgs& g, int w_is_nk, const StreamPlan& p, hipStream_t s, const WayOut&... way_out) {
  // Up to 16 rows of X on [N x K] weights: two units on their way a wavefront; more are in the way where the weight is in a cache.  us with two,
  // three and four, 4 x 5632 -> 2048 (8 x 8) in the last-level cache 5.7, 5.8, 5.9, from HBM 6.8, 6.2, 6.2; 16 x 5632 -> 2048 (16 x 8) 5.9, 6.1, 6.2 and
  // 7.8, 7.9, 8.0; 16 x 768 -> 768 (16 x 16) 2.6, 2.6, 2.6 and 3.0, 3.1, 3.1.
  if (p.bn == 8) p.bm == 8 ? launch_plain<1, 1, 8, 2, 8, 8>(g, w_is_nk, p, s, way_out...) : launch_plain<1, 1, 8, 2, 16, 8>(g, w_is_nk, p, s, way_out...);
  else if (p.bn == 16) p.bm == 8 ? launch_plain<1, 1, 8, 2, 8, 16>(g, w_is_nk, p, s, way_out...) : launch_plain<1, 1, 8, 2>(g, w_is_nk, p, s, way_out...);
  else if (p.bm == 8) launch_plain<1, 2, 8, 2, 8, 32, true>(g, w_is_nk, p, s, way_out...);
  else if (p.mt == 1) launch_plain<1, 2, 8, 2, 16, 32, true>(g, w_is_nk, p, s, way_out...);
  else if (p.mt == 2 && p.nt == 2) launch_plain<2, 2, 8, 2, 32, 32, true, true>(g, w_is_nk, p, s, way_out...);
  else if (p.mt == 2) launch_plain<2, 4, 4, 3>(g, w_is_nk, p, s, way_out...);
  else if (p.mt == 4) launch_plain<4, 4, 4, 2>(g, w_is_nk, p, s, way_out...);
  else launch_plain<8, 4, 4, 1>(g, w_is_nk, p, s, way_out...);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

}  // namespace gws
