// The products of the gated block in 128 x 128 tiles (gfx950), for sizes with too few 256 x 256 tiles: the loop of gws_gemm128.hip (2 x 2
// wavefronts, K-steps of 64, operand tiles straight into a ring of four LDS stages, one barrier a K-step between its two halves), with
// 64 columns of two weights side by side (forward) or two products in one sum (input gradient).
// D: stages.  With four a workgroup has a compute unit for itself; with two a second one shares it, whose K-steps run under the other's way
// out: more tiles than compute units, 4096 x 768 -> 2048 backward from 8 bits 29 -> 22.5 us, forward 32 -> 26; 2048 x 2048 -> 5632 forward 99
// -> 82.  One workgroup alone waits longer for its loads: 256 x 2048 -> 5632 forward 17.4 and 23.0.
// What bounds it: a K-step takes 0.34 us alone and 0.41 with all compute units at work (the operands' 32 KiB out of the L2), a launch 2.7, the way
// out 2.6 (forward) to 10 us (backward).  1021 x 768 -> 2048, 256 tiles: forward 10.1 us, keeping G and U 11.4 (BF16) and 12.2 (8 bits).
//   forward: stage rows 32 w .. 32 w + 31 of [F x K] weights, one wavefront's loads, are columns 32 (w / 2) .. of Wg (w even) or Wu; of [K x F]
//   weights 64 k-rows of 64 columns of Wg and then of Wu, two wavefronts each.  Either way a wavefront multiplies 32 columns of both.
#include "gws_gated_out.h"
#include "gws_gemm_stream_core.h"

namespace gws {

namespace {
constexpr int T = 128, TK = 64, NJ = 4;              // rows and stage columns of a tile, depth of a K-step, column tiles of a wavefront
constexpr int OPERAND = T * TK, STG = 2 * OPERAND;   // elements of one operand's tile, of a stage
constexpr uint32_t kMaxLd128 = 1u << 24;             // 32-bit lane offsets: 127 rows x 2 bytes
}  // namespace

template <GatedOp OP, bool W_NK, Kept KEPT, int D>
__global__ __launch_bounds__(256, D == 2 ? 2 : 1) void gated128_kernel(const GatedArgs g) {
  using stream::umin;
  constexpr bool PAIR = OP == GatedOp::kFwd, TWO = OP == GatedOp::kDx;
  constexpr uint32_t TC = PAIR ? T / 2 : T;          // columns of a tile
  __shared__ __attribute__((aligned(1024))) uint16_t lds[D * STG];
  const uint32_t lane = threadIdx.x & 63, li = lane & 15, grp = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  uint32_t tile_m, tile_n;
  tile_of(TileGrid{(g.M + T - 1) / T, (g.N + TC - 1) / TC, g.inv_band, g.inv_last}, blockIdx.x, tile_m, tile_n);
  const uint32_t m0 = tile_m * T, n0 = tile_n * TC;

  // a wavefront's load instructions of an operand tile, four each; rows and columns past the edge are read from the last ones.  An
  // instruction's offset counts on both sides: 1 KiB a load in LDS, taken back here
  uint32_t xo[4], wo[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t row = 32 * wave + 8 * q + (lane >> 3), chunk = (lane & 7) ^ (4 * (q & 1) + (lane >> 4));
    xo[q] = (umin(row, g.M - 1 - m0) * g.lda + chunk * 8) * 2 + 1024 * (3 - q);
    if (W_NK) {
      const uint32_t col = PAIR ? 32 * (wave >> 1) + 8 * q + (lane >> 3) : row;
      wo[q] = (umin(col, g.N - 1 - n0) * g.ldb + chunk * 8) * 2;
    } else if (PAIR) {
      const uint32_t k = 32 * (wave & 1) + 8 * q + (lane >> 3), c = (lane & 7) ^ stream::oc_swizzle<4>(k);
      wo[q] = (k * g.ldb + umin(c, (g.N - n0) / 8 - 1) * 8) * 2;
    } else {
      const uint32_t k = 16 * wave + 4 * q + (lane >> 4), c = (lane & 15) ^ stream::oc_swizzle<8>(k);
      wo[q] = (k * g.ldb + umin(c, (g.N - n0) / 8 - 1) * 8) * 2;
    }
    wo[q] += 1024 * (3 - q);
  }
  const uint16_t* const mine = PAIR && (W_NK ? wave & 1 : wave >> 1) ? g.b2 : g.b;   // the wavefront's weight
  const size_t x_at = (size_t)m0 * g.lda, w_at = W_NK ? (size_t)n0 * g.ldb : n0;
  const GWS_GLOBAL char* xb = (const GWS_GLOBAL char*)(g.a + x_at) - 3072;
  const GWS_GLOBAL char* wb = (const GWS_GLOBAL char*)(mine + w_at) - 3072;
  const uint32_t nk1 = (g.K + TK - 1) / TK, nk = TWO ? 2 * nk1 : nk1;
  uint32_t k_next = 0, steps = 0;        // first k of the step that is fetched next; steps fetched
  const uint32_t lds_x = (uint32_t)(uintptr_t)(GWS_LDS void*)lds + wave * 4096, lds_w = lds_x + OPERAND * 2;
  // two of a step's loads (n = 0 .. 3): X, W, X, W, on one setting of M0
  auto load_n = [&](uint32_t stage, int n) {
    const uint32_t dst = (n & 1 ? lds_w : lds_x) + stage;
    const uint32_t v0 = n & 1 ? wo[n & 2] : xo[n & 2], v1 = n & 1 ? wo[(n & 2) + 1] : xo[(n & 2) + 1];
    const GWS_GLOBAL char* base = n & 1 ? wb : xb;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    if (n < 2)
      asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024"
                   ::"v"(v0), "v"(v1), "s"(base), "s"(dst) : "m0", "memory");
    else
      asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2 offset:2048\n\tglobal_load_lds_dwordx4 %1, %2 offset:3072"
                   ::"v"(v0), "v"(v1), "s"(base), "s"(dst) : "m0", "memory");
#pragma clang diagnostic pop
  };
  auto load_advance = [&]() {   // the half step at the end of K is fetched as the second half of a whole one
    const uint32_t k = umin(k_next + TK, g.K - TK), d = __builtin_amdgcn_readfirstlane(k - k_next);
    xb += d * 2;
    wb += W_NK ? (size_t)d * 2 : (size_t)d * (g.ldb * 2);
    k_next = k;
    if (TWO && ++steps == nk1) {   // on to the second product
      xb = (const GWS_GLOBAL char*)(g.a2 + x_at) - 3072;
      wb = (const GWS_GLOBAL char*)(g.b2 + w_at) - 3072;
      k_next = 0;
    }
  };
  Frag8 fx[2][4], fw[2][NJ];
  // read fragments of half h, step n of NR, in the order the MFMAs need them: X 0, W 0 .. 3, X 1 .. 3
  constexpr int RW = W_NK ? 1 : 2, NR = 4 + NJ * RW;
  uint32_t xr[2], wr[W_NK ? 2 : NJ];   // byte offsets in a stage
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t sl = ((4 * h + grp) ^ ((li >> 1) & 7)) * 16;
    xr[h] = (64 * wm + li) * 128 + sl;
    if (W_NK) wr[h] = OPERAND * 2 + (64 * wn + li) * 128 + sl;
  }
  constexpr uint32_t WROW = PAIR ? 128 : 256;   // bytes of a k-row
  if (!W_NK)
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint32_t k = 8 * grp + (li >> 2), c = 2 * (PAIR ? 2 * wn + (j & 1) : NJ * wn + j) + ((li >> 1) & 1);
      wr[j] = OPERAND * 2 + (PAIR ? (j >> 1) * 8192 : 0) + k * WROW + (c ^ stream::oc_swizzle<PAIR ? 4 : 8>(k)) * 16 + (li & 1) * 8;
    }
  auto read_n = [&](int h, uint32_t stage, int n) {
    const char* st = (const char*)lds + stage;
    if (n == 0 || n > NJ * RW) {
      const int i = n == 0 ? 0 : n - NJ * RW;
      fx[h][i].u = *(const u32x4*)(st + xr[h] + 2048 * i);
    } else if (W_NK) {
      fw[h][n - 1].u = *(const u32x4*)(st + wr[h] + 2048 * (n - 1));
    } else {
      const int j = (n - 1) >> 1, t = (n - 1) & 1;
      fw[h][j].h[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GWS_LDS i16x4*)(st + wr[j] + WROW * (32 * h + 4 * t)));
    }
  };
  f32x4 acc[4][NJ];   // row 16 i + lane % 16 of the wavefront's 64; columns: see gws_gated_out.h
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto mfma_n = [&](int h, int n) {
    const int i = n / NJ, j = n % NJ;
    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[h][j].v, fx[h][i].v, acc[i][j], 0, 0, 0);
  };
  const uint32_t p0 = m0 + 64 * wm, q0 = n0 + TC / 2 * wn;   // of the wavefront's part of the result
  [[maybe_unused]] KeptTile<KEPT == Kept::kNone ? Kept::kBf16 : KEPT, true, 4, 4> kept;
  if constexpr (OP == GatedOp::kBwd) kept.request(g, p0, q0, lane, 0);   // its first rows land under the loop
  constexpr int LOADS = 8;   // load instructions of a wavefront and K-step
#pragma unroll
  for (int s = 0; s < D; ++s)
    if ((uint32_t)s < nk) {
#pragma unroll
      for (int n = 0; n < 4; ++n) load_n(s * STG * 2, n);
      load_advance();
    }
  if (nk >= D) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS * (D - 1)) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int n = 0; n < NR; ++n) read_n(0, 0, n);
  // The order is written out and pinned: a read behind each of the first MFMAs of a half, two loads of the step four ahead
  // behind every fourth MFMA of the second half (into the stage that the barrier has just released).
  auto first_half = [&](uint32_t stage) {
#pragma unroll
    for (int n = 0; n < 4 * NJ; ++n) {
      mfma_n(0, n);
      __builtin_amdgcn_sched_barrier(0);
      if (n < NR) read_n(1, stage, n);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto second_half = [&](uint32_t stage, uint32_t next, bool more) {
#pragma unroll
    for (int n = 0; n < 4 * NJ; ++n) {
      mfma_n(1, n);
      __builtin_amdgcn_sched_barrier(0);
      if (n < NR) read_n(0, next, n);
      if (more && n % NJ == NJ - 1) load_n(stage, n / NJ);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) load_advance();
  };
  // half a step at the end of K: the stage's first half belongs to the step before
  auto half_step = [&](uint32_t kt) {
    if (TK * (TWO && kt >= nk1 ? kt - nk1 : kt) + TK > g.K) {
#pragma unroll
      for (int i = 0; i < 4; ++i) fx[0][i].u = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < NJ; ++j) fw[0][j].u = u32x4{0, 0, 0, 0};
    }
  };
  uint32_t kt = 0, stage = 0;   // of the ring, in bytes
  auto after = [](uint32_t s) { return (s + STG * 2) & (D * STG * 2 - 1); };
  for (; kt + D < nk; ++kt) {
    if (TWO) half_step(kt);
    first_half(stage);
    // this stage is read; the next step has landed when all but the two steps behind it have
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (D - 2)) : "memory");
    second_half(stage, after(stage), true);
    stage = after(stage);
  }
  // without this the register allocator passes the last accumulators on from register to register in the loop above
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm("" : "+a"(acc[i][j]));
  for (; kt < nk; ++kt) {   // everything is on its way: the reads past the last step fetch a stage that nobody multiplies
    half_step(kt);
    first_half(stage);
    if (kt + D == nk) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (D - 2)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    second_half(stage, after(stage), false);
    stage = after(stage);
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the ring is read

  uint16_t* cs = lds + wave * (D * STG / 4);
  if constexpr (OP == GatedOp::kFwd) {
    fwd_out<KEPT, true, 4, 2>(g, acc, (uint8_t*)cs, (uint8_t*)(lds + 2 * wm * (D * STG / 4)), wn, p0, q0, lane);
  } else if constexpr (OP == GatedOp::kBwd) {
    bwd_out<KEPT, true, 4, 4>(g, acc, kept, (float*)cs, p0, q0, lane);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        *(u32x2*)((uint8_t*)cs + (16 * i + li) * kPitch<4, 2> + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(acc[i][j][0], acc[i][j][1]), pack_bf16_rne(acc[i][j][2], acc[i][j][3])};
    own_lds_wait();
    rows_out<4, 2, true, false>((const uint8_t*)cs, (uint8_t*)(g.h + (size_t)p0 * g.ldh + q0), (size_t)g.ldh * 2, lane, (int)g.M - (int)p0, (int)g.N - (int)q0);
  }
}

bool gated128_applicable(const GatedArgs& g) { return g.K >= 64 && out_lds_ok(g) && g.lda < kMaxLd128 && g.ldb < kMaxLd128; }

template <GatedOp OP, Kept KEPT, int D>
static int launch_tiles(GatedArgs g, bool b_oc, hipStream_t stream) {
  constexpr uint32_t TC = OP == GatedOp::kFwd ? T / 2 : T;
  const uint32_t mt = (uint32_t)(((uint64_t)g.M + T - 1) / T), nt = (uint32_t)(((uint64_t)g.N + TC - 1) / TC);
  if ((uint64_t)mt * nt >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  set_tile_grid(g, mt, nt);
  if (b_oc) hipLaunchKernelGGL((gated128_kernel<OP, false, KEPT, D>), dim3(mt * nt), dim3(256), 0, stream, g);
  else hipLaunchKernelGGL((gated128_kernel<OP, true, KEPT, D>), dim3(mt * nt), dim3(256), 0, stream, g);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

int launch_gated128(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, bool two, hipStream_t stream) {
  constexpr GatedOp F = GatedOp::kFwd, B = GatedOp::kBwd;
  if (op == GatedOp::kDx) return launch_tiles<GatedOp::kDx, Kept::kNone, 4>(g, b_oc, stream);
  if (op == B && kept == Kept::kE4m3) return two ? launch_tiles<B, Kept::kE4m3, 2>(g, b_oc, stream) : launch_tiles<B, Kept::kE4m3, 4>(g, b_oc, stream);
  if (op == B) return two ? launch_tiles<B, Kept::kBf16, 2>(g, b_oc, stream) : launch_tiles<B, Kept::kBf16, 4>(g, b_oc, stream);
  if (kept == Kept::kE4m3) return two ? launch_tiles<F, Kept::kE4m3, 2>(g, b_oc, stream) : launch_tiles<F, Kept::kE4m3, 4>(g, b_oc, stream);
  if (kept == Kept::kBf16) return two ? launch_tiles<F, Kept::kBf16, 2>(g, b_oc, stream) : launch_tiles<F, Kept::kBf16, 4>(g, b_oc, stream);
  return two ? launch_tiles<F, Kept::kNone, 2>(g, b_oc, stream) : launch_tiles<F, Kept::kNone, 4>(g, b_oc, stream);
}

}  // namespace gws
