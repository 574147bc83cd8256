// The products of the gated block for few tokens, or for so few tiles that compute units would idle (gfx950): as
// gws_gemm_stream.hip, a workgroup owns a small piece of the result, its wavefronts split the contraction, each with its own ring of
// LDS stages, and meet only for the partial sums, which are added in LDS in the order of the wavefronts.
//   forward: the piece is the same columns of G and of U, half of the stage's weight columns each;
//   input gradient: the units of 64 of both products, one after the other, are what the wavefronts split.
// What bounds it for a few tokens: the weights' bytes.  2048 x 5632 [F x K], 46 MB, out of the last-level cache: one token 8.5 us (5.4 TB/s; a large
// copy reaches 5.15), 27 tokens 9.4.  With more rows the operands that a compute unit takes out of its L2: input gradient of 1021 tokens, 768 x 2048,
// 13.9 us in 64 x 64 (192 workgroups, 1 MiB each), 12.4 in 64 x 48 (256, 0.875 MiB).
// Backward, the kept values requested first of all instead of when the sums are there: 1021 x 768 -> 2048 14.4 -> 12.5 us.
#include "gws_gated.h"
#include "gws_gemm_stream_core.h"

namespace gws {

namespace {

__device__ __forceinline__ f32x4 add4(const f32x4& a, const f32x4& b) {
  return f32x4{__fadd_rn(a[0], b[0]), __fadd_rn(a[1], b[1]), __fadd_rn(a[2], b[2]), __fadd_rn(a[3], b[3])};
}
__device__ __forceinline__ u32x2 pack4(const float (&v)[4]) { return u32x2{pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3])}; }

// Four columns of one row on their way out: sums[0] of G and sums[1] of U, or sums[0] alone.  All lanes of a wavefront come here, eight
// neighbouring ones with the 32 columns of a block; `here`: the row exists.
template <GatedOp OP, Kept KEPT>
__device__ __forceinline__ void four_out(const GatedArgs& g, uint32_t row, uint32_t col, bool here, const f32x4 (&sums)[2], const KeptFours<KEPT>& kept) {
  if (OP == GatedOp::kDx) {
    const float v[4] = {sums[0][0], sums[0][1], sums[0][2], sums[0][3]};
    if (here) *(u32x2*)(g.h + (size_t)row * g.ldh + col) = pack4(v);
  } else if (OP == GatedOp::kFwd) {
    float v[2][4], h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[0][e] = sums[0][e];
      v[1][e] = sums[1][e];
      h[e] = v[1][e];
    }
    with_gate(g.act, [&](auto gate) {
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] *= gate.a(v[0][e]);
    });
    if (here) *(u32x2*)(g.h + (size_t)row * g.ldh + col) = pack4(h);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint8_t* to = p == 0 ? g.kept.g : g.kept.u;
      const uint32_t ld = p == 0 ? g.kept.ldg : g.kept.ldu;
      if (KEPT == Kept::kBf16 && here) *(u32x2*)(to + ((size_t)row * ld + col) * 2) = pack4(v[p]);
      if (KEPT == Kept::kE4m3) {
        uint32_t m = __float_as_uint(act8_larger(act8_larger(0.0f, v[p][0], v[p][1]), v[p][2], v[p][3])) & 0x7FFFFFFFu;
        m = max(m, dpp_u32<0xB1>(m));    // lane ^ 1
        m = max(m, dpp_u32<0x4E>(m));    // lane ^ 2
        m = max(m, dpp_u32<0x141>(m));   // row_half_mirror: the other four of eight
        const uint32_t byte = act8_byte(m);
        if (byte == kAct8Max) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[p][e] = act8_clamp(v[p][e]);
        }
        if (here) *(uint32_t*)(to + (size_t)row * ld + col) = act8_codes(v[p], byte);
        if (here && (col & 31) == 0) (p == 0 ? g.kept.gs : g.kept.us)[(size_t)row * (p == 0 ? g.kept.lsg : g.kept.lsu) + (col >> 5)] = (uint8_t)byte;
      }
    }
  } else if (here) {
    float vg[4], vu[4], h[4], dg[4], du[4];
    kept.g.values(vg);
    kept.u.values(vu);
    with_gate(g.act, [&](auto gate) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float a, slope;
        gate.both(vg[e], a, slope);
        h[e] = a * vu[e];
        du[e] = sums[0][e] * a;
        dg[e] = sums[0][e] * vu[e] * slope;
      }
    });
    *(u32x2*)(g.dg + (size_t)row * g.ldd + col) = pack4(dg);
    *(u32x2*)(g.du + (size_t)row * g.ldd + col) = pack4(du);
    if (g.h != nullptr) *(u32x2*)(g.h + (size_t)row * g.ldh + col) = pack4(h);
  }
}

}  // namespace

// The tile: 16 MT rows (BM of them loaded and stored) and 16 NT columns of the stage.
template <GatedOp OP, int MT, int NT, int P, int D, bool W_NK, Kept KEPT, int BM = 16 * MT>
__global__ __launch_bounds__(64 * P) void gated_stream_kernel(const GatedArgs g) {
  using namespace stream;
  constexpr bool PAIR = OP == GatedOp::kFwd, TWO = OP == GatedOp::kDx;
  static_assert(BM == 16 * MT || (BM == 8 && MT == 1), "whole MFMA tiles or half a one");
  constexpr int T = PAIR ? NT / 2 : NT, BN = 16 * T;                   // column tiles and columns of one weight
  static_assert(W_NK || T == 2 || T == 4 || T == 8, "swizzle of the [K x N] stage");
  static_assert(KEPT != Kept::kE4m3 || T % 2 == 0, "whole blocks of 32");
  constexpr int XS = BM * 64, HS = BN * 64, WS = (PAIR ? 2 : 1) * HS, STG = XS + WS;   // elements of a stage
  constexpr int QX = BM / 8, QH = BN / 8, QW = WS / 512, LOADS = QX + QW;              // load instructions of a unit
  static_assert(LOADS * (D - 1) <= 63, "the wait for a unit counts the loads behind it");
  constexpr int MC = MT > 4 ? 4 : MT;                                   // row tiles of a pass of the reduction
  constexpr int kRing = P * D * STG * 2, kRed = red_bytes(MC, NT, P);
  __shared__ __attribute__((aligned(1024))) char lds[kRing > kRed ? kRing : kRed];
  const uint32_t lane = threadIdx.x & 63, li = lane & 15, grp = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* ring = (uint16_t*)lds + wave * (D * STG);
  const TileGrid t = {(g.M + BM - 1) / BM, (g.N + BN - 1) / BN, g.inv_band, g.inv_last};
  uint32_t m0, n0;
  if (t.joined()) tile_of_joined(t, blockIdx.x, m0, n0);
  else tile_of_groups(t, !W_NK && T == 2, blockIdx.x, m0, n0);
  m0 *= BM;
  n0 *= BN;
  // units of 64 of the contraction; with two products those of the second follow
  const uint32_t nu1 = (g.K + 63) >> 6, nu = TWO ? 2 * nu1 : nu1;
  const uint32_t u0 = (uint32_t)((uint64_t)nu * wave / P), u1 = (uint32_t)((uint64_t)nu * (wave + 1) / P);

  // lane offsets in bytes; rows and columns past the edge are read from the last ones and not stored
  uint32_t xo[QX], wo[W_NK ? QH : 1];
#pragma unroll
  for (int q = 0; q < QX; ++q) xo[q] = (umin(8u * q + (lane >> 3), g.M - 1 - m0) * g.lda + ((lane & 7) ^ (4 * (q & 1) + (lane >> 4))) * 8) * 2;
  if (W_NK) {
#pragma unroll
    for (int q = 0; q < QH; ++q) wo[q] = (umin(8u * q + (lane >> 3), g.N - 1 - n0) * g.ldb + ((lane & 7) ^ (4 * (q & 1) + (lane >> 4))) * 8) * 2;
  }
  // [K x N]: an instruction covers RPI k-rows of 2 T chunks
  constexpr uint32_t CPR = 2 * T, RPI = 64 / CPR;
  const uint32_t wk = lane / CPR, ws = lane % CPR;
  const uint32_t last_chunk = (g.N - n0) / 8 - 1;
  constexpr int NV = W_NK ? 1 : 16 / RPI;   // the swizzle depends on k % 16
  uint32_t wv[NV];
  if (!W_NK) {
#pragma unroll
    for (int v = 0; v < NV; ++v) wv[v] = (wk * g.ldb + umin(ws ^ oc_swizzle<W_NK ? 2 : T>(wk + RPI * v), last_chunk) * 8) * 2;
  }
  const size_t x_at = (size_t)m0 * g.lda * 2, w_at = (W_NK ? (size_t)n0 * g.ldb : (size_t)n0) * 2;
  auto load = [&](uint32_t u, uint32_t slot) {
    uint16_t* st = ring + slot * STG;
    const bool second = TWO && u >= nu1;   // uniform
    const uint32_t k0 = umin(64 * (second ? u - nu1 : u), g.K - 64);   // the half unit at the end of K is fetched as the second half of a whole one
    const GWS_GLOBAL char* xb = (const GWS_GLOBAL char*)(second ? g.a2 : g.a) + x_at;
#pragma unroll
    for (int p = 0; p < (PAIR ? 2 : 1); ++p) {
      const GWS_GLOBAL char* wb = (const GWS_GLOBAL char*)(p == 1 || second ? g.b2 : g.b) + w_at;
#pragma unroll
      for (int q = 0; q < QH; ++q) {
        if (W_NK) direct(wb + (size_t)k0 * 2, wo[q], st + XS + p * HS + q * 512);
        else direct(wb + (size_t)(k0 + RPI * q) * g.ldb * 2, wv[q % NV], st + XS + p * HS + q * 512);
      }
    }
#pragma unroll
    for (int q = 0; q < QX; ++q) direct(xb + (size_t)k0 * 2, xo[q], st + q * 512);
  };

  // Backward: what a thread needs of the kept G and U when the sums are there, four columns `fours` times a pass of the reduction, is
  // requested before anything else
  constexpr uint32_t PITCH = 4 * NT + 1, C4 = 4 * T;   // four-column groups of one weight
  constexpr int FOURS = (MC * 16 * C4 + P * 64 - 1) / (P * 64), PASSES = MT / MC;
  auto place = [&](int pass, int n, uint32_t& r, uint32_t& c, uint32_t& row, uint32_t& col) {
    const uint32_t it = threadIdx.x + n * P * 64;
    r = it / C4;
    c = it % C4;
    row = m0 + 16 * MC * pass + r;
    col = n0 + 4 * c;
    return row < g.M && col < g.N && r < 16 * MC && (BM == 16 * MT || r < BM);
  };
  KeptFours<KEPT> kept[PASSES][FOURS];
  if (OP == GatedOp::kBwd) {
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass)
#pragma unroll
      for (int n = 0; n < FOURS; ++n) {
        uint32_t r, c, row, col;
        if (place(pass, n, r, c, row, col)) kept[pass][n].load(g.kept, row, col);
      }
  }

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
  const uint32_t lx = BM == 8 ? li & 7 : li;
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
        const uint16_t* part = wsg + (j / T) * HS;
        if (W_NK) fw[h][j].u = *(const u32x4*)(part + (16 * (j % T) + li) * 64 + (((4 * h + grp) ^ ((li >> 1) & 7)) * 8));
        else fw[h][j] = read_oc<W_NK ? 2 : T>(part, h, j % T, li, grp);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read: the stage can be filled again
    __builtin_amdgcn_sched_barrier(0);
    if (i + D < n) load(u0 + i + D, slot);
    slot = slot + 1 == D ? 0 : slot + 1;
    const uint32_t u = u0 + i, in = TWO && u >= nu1 ? u - nu1 : u;
    const bool half = 64 * in + 64 > g.K;   // only the second half of the stage belongs to this unit
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 0 && half) continue;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < MT; ++r) acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[h][j].v, fx[h][r].v, acc[r][j], 0, 0, 0);
    }
  }

  // the partial sums, MC row tiles at a time, added in the order of the wavefronts
  f32x4* red = (f32x4*)lds;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    __syncthreads();   // what was in this memory is read
#pragma unroll
    for (int i = 0; i < MC; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) red[((wave * MC + i) * 16 + li) * PITCH + 4 * j + grp] = acc[MC * pass + i][j];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < FOURS; ++n) {
      if (threadIdx.x + n * P * 64 >= MC * 16 * C4) continue;   // whole wavefronts
      uint32_t r, c, row, col;
      const bool here = place(pass, n, r, c, row, col);
      f32x4 s[2];
#pragma unroll
      for (int p = 0; p < (PAIR ? 2 : 1); ++p) {
        s[p] = red[r * PITCH + p * C4 + c];
#pragma unroll
        for (int w = 1; w < P; ++w) s[p] = add4(s[p], red[(w * MC * 16 + r) * PITCH + p * C4 + c]);
      }
      four_out<OP, KEPT>(g, row, col, here, s, kept[pass][n]);
    }
  }
}

// The tile by an estimate in us: a launch and, per round of workgroups (one per compute unit: the rings fill its LDS), a fixed part, the gate
// and the bytes of the tile's operands at the rate (bytes per ns) that a compute unit takes them.  Narrow tiles only where few columns would leave
// compute units idle (the input gradient's K columns).  Over 120 drawn sizes of input gradients the choice takes 1.004 of the fastest tile's time.
// Measured and estimated:
//   forward, G and U not kept, [F x K]: 1 x 2048 -> 5632 9.1 us; 27 9.9, 9.9; 64 11.4, 9.7; 128 15.4, 15.4; [K x F], whose 64-byte pieces of rows
//   are half lines: 11.5; 12.3, 9.7; 14.5, 11.4; 19.3, 19.0
//   input gradient, [K x F]: 64 x 2 x 5632 -> 2048 25.5, 26.1; 1021 x 2 x 2048 -> 768 in 64 x 64 14.5, 15.0 (192 workgroups), in
//   64 x 48 13.2, 13.7 (256), in 128 x 64 21.5, 24.1 (96); 1978 x 2 x 1728 -> 928 24.7, 24.9, 31.1, 33.1 and 20.0, 21.5
GatedStreamPlan gated_stream_plan(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept) {
  GatedStreamPlan best = {0, 0, 0, 1e30};
  if (g.K < 64 || g.lda >= stream::kMaxLd || g.ldb >= stream::kMaxLd) return best;
  const uint64_t cus = compute_units() > 0 ? compute_units() : 256;
  const bool pair = op == GatedOp::kFwd, two = op == GatedOp::kDx;
  const double K = two ? 2.0 * g.K : (double)g.K;
  const struct { int mt, nt, p; double rate; } tiles[] = {{1, 1, 8, 130.0}, {1, 2, 8, 130.0}, {2, 2, 8, 130.0}, {1, 4, 8, 130.0},
                                                                 {2, 4, 4, 100.0}, {4, 3, 4, 100.0}, {4, 4, 4, 100.0}, {8, 4, 4, two ? 95.0 : 72.0}};
  for (const auto& t : tiles) {
    if (t.mt == 1 && g.M > 16) continue;
    if ((t.nt == 1 || (t.mt == 2 && t.nt == 2)) && !two) continue;
    if (t.nt == 1 && b_oc) continue;
    if (t.nt == 3 && (b_oc || !two)) continue;                          // 48 columns: not of a weight across the contraction, whose lines it would cut
    if (t.nt == 2 && pair && (b_oc || kept == Kept::kE4m3)) continue;   // 16 columns of each weight: half a block, a quarter of a line
    const uint64_t bn = 16 * t.nt / (pair ? 2 : 1), wgs = ((uint64_t)g.M + 16 * t.mt - 1) / (16 * t.mt) * ((g.N + bn - 1) / bn);
    // a weight across the contraction comes in pieces of lines; the kept values and the gate's results of a tile go through few wavefronts
    const double weight = t.nt * (b_oc && pair ? 1.8 : b_oc && two ? 1.35 : 1.0);
    const double beside = two && t.mt == 8 ? 3.0 : t.mt * t.nt * (op == GatedOp::kBwd ? 0.09 : pair && kept != Kept::kNone ? 0.06 : 0.0);
    const double rounds = (double)((wgs + cus - 1) / cus);
    // two wide operands of more than the L2s hold come from memory more slowly than the tiles ask for them: 5211 x 2 x 2944 -> 320 (61 MB) 51 us, 36
    // without this (128 x 128 tiles: 42); 6384 x 2 x 3968 -> 256 (101 MB) 78, 44
    const double rows_mb = (double)g.M * K * 2e-6, cold = two && rows_mb > 45.0 ? (rows_mb - 45.0) / 1.5 : 0.0;
    const double us = 1.8 + cold + rounds * (2.7 + beside + K * 2 * 16 * (t.mt + weight) / t.rate * 1e-3);
    if (wgs < 0x7FFFFFFFull && us < best.us) best = {t.mt, t.nt, t.p, us};
  }
  return best;
}

template <GatedOp OP, int MT, int NT, int P, int D, Kept KEPT, int BM = 16 * MT>
static int launch_tile(GatedArgs g, bool b_oc, hipStream_t s) {
  constexpr uint32_t BN = 16 * NT / (OP == GatedOp::kFwd ? 2 : 1);
  const uint64_t rows = ((uint64_t)g.M + BM - 1) / BM, columns = ((uint64_t)g.N + BN - 1) / BN;
  if (rows * columns >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  set_tile_grid(g, (uint32_t)rows, (uint32_t)columns, 8, columns >= (b_oc ? 6 : 4) && rows * columns >= 32 && (!b_oc || rows > 1));
  const dim3 grid((uint32_t)(rows * columns));
  if (!b_oc) {
    hipLaunchKernelGGL((gated_stream_kernel<OP, MT, NT, P, D, true, KEPT, BM>), grid, dim3(64 * P), 0, s, g);
  } else if constexpr (BN >= 32 && BN != 48) {
    hipLaunchKernelGGL((gated_stream_kernel<OP, MT, NT, P, D, false, KEPT, BM>), grid, dim3(64 * P), 0, s, g);
  } else {
    return GWS_ERR_SHAPE;
  }
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

template <GatedOp OP, Kept KEPT>
static int launch_plan(const GatedArgs& g, bool b_oc, const GatedStreamPlan& p, hipStream_t s) {
  if constexpr (OP == GatedOp::kDx) {
    if (p.nt == 1) return g.M <= 8 ? launch_tile<OP, 1, 1, 8, 2, KEPT, 8>(g, b_oc, s) : launch_tile<OP, 1, 1, 8, 2, KEPT>(g, b_oc, s);
    if (p.mt == 2 && p.nt == 2) return launch_tile<OP, 2, 2, 8, 2, KEPT>(g, b_oc, s);
    if (p.nt == 3) return launch_tile<OP, 4, 3, 4, 2, KEPT>(g, b_oc, s);
  }
  if constexpr (OP != GatedOp::kFwd || KEPT != Kept::kE4m3) {
    if (p.nt == 2) return g.M <= 8 ? launch_tile<OP, 1, 2, 8, 2, KEPT, 8>(g, b_oc, s) : launch_tile<OP, 1, 2, 8, 2, KEPT>(g, b_oc, s);
  }
  if (p.mt == 1) return g.M <= 8 ? launch_tile<OP, 1, 4, 8, 2, KEPT, 8>(g, b_oc, s) : launch_tile<OP, 1, 4, 8, 2, KEPT>(g, b_oc, s);
  if (p.mt == 2) return launch_tile<OP, 2, 4, 4, 3, KEPT>(g, b_oc, s);
  if (p.mt == 4) return launch_tile<OP, 4, 4, 4, 2, KEPT>(g, b_oc, s);
  return launch_tile<OP, 8, 4, 4, 1, KEPT>(g, b_oc, s);
}

int launch_gated_stream(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, const GatedStreamPlan& p, hipStream_t s) {
  if (op == GatedOp::kDx) return launch_plan<GatedOp::kDx, Kept::kNone>(g, b_oc, p, s);
  if (op == GatedOp::kBwd)
    return kept == Kept::kE4m3 ? launch_plan<GatedOp::kBwd, Kept::kE4m3>(g, b_oc, p, s) : launch_plan<GatedOp::kBwd, Kept::kBf16>(g, b_oc, p, s);
  return kept == Kept::kE4m3 ? launch_plan<GatedOp::kFwd, Kept::kE4m3>(g, b_oc, p, s)
         : kept == Kept::kBf16 ? launch_plan<GatedOp::kFwd, Kept::kBf16>(g, b_oc, p, s) : launch_plan<GatedOp::kFwd, Kept::kNone>(g, b_oc, p, s);
}

}  // namespace gws
