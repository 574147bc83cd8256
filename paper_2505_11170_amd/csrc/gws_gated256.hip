// The products of the gated block in 256 x 256 tiles (gfx950): the loop of gws_gemm256_core.h with two weights side by side
// (forward), with two products in one sum (input gradient), or as it is (backward), and the gate on the way out.
// The way out is in gws_gated_out.h.
// What bounds them: the matrix cores at the card's power limit while the loop runs, and then, with one wavefront a SIMD, the way out by itself.
//   input gradient: no way out to speak of, 8192 x 2 x 5632 -> 2048 in 263 - 278 us, 1.36 - 1.44 PFLOP/s (a large library product 1.35).
//   forward, 8192 x 2048 -> 5632 (two products of 167 - 173 us each without a gate): 287 - 298 us; the vector ALU takes 3 us a tile more for keeping
//   G and U (5.5 tiles a compute unit), and their bytes leave in bursts: 309 - 317 as BF16, 318 - 324 in 8 bits.  (With H past the caches 277 - 282,
//   304 - 312 and 307, at the cost of the product that reads it.)
//   backward of the same: 135 us of products, and 2.75 times all compute units at once ask for 134 MB: without the stores 171 us, without the
//   kept values 175, without the gate's arithmetic 200, with everything 196 - 206 (bf16 205 - 216).
// Less does not help where it was tried: three quarters of the kept values on their way instead of two (0.5 %, and registers to scratch), and
// two smaller tiles a compute unit, whose ways out fall under each other's loops but whose loops wait for the L2 (265 us).
#include "gws_gated_out.h"

namespace gws {

template <GatedOp OP, bool B_OC, Kept KEPT, bool EDGE>
__global__ __launch_bounds__(256, 1) void gated256_kernel(const GatedArgs g) {
  using namespace g256;
  constexpr uint32_t TC = OP == GatedOp::kFwd ? 128 : 256;   // columns of a tile
  uint32_t tile_m, tile_n;
  tile_of(TileGrid{(g.M + TM - 1) / TM, (g.N + TC - 1) / TC, g.inv_band, g.inv_last}, blockIdx.x, tile_m, tile_n);
  const uint32_t m0 = tile_m * TM, n0 = tile_n * TC, rows = g.M - m0 < TM ? g.M - m0 : TM, cols = g.N - n0 < TC ? g.N - n0 : TC;
  const uint32_t nk = (g.K + TK - 1) / TK;
  if constexpr (OP == GatedOp::kFwd) {
    gemm256_accumulate<false, B_OC, EDGE, 8, kPair>(g.a, g.lda, g.b, g.ldb, nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane, uint16_t* first) {
      fwd_out<KEPT, EDGE, 8, 4>(g, acc, (uint8_t*)cs, (uint8_t*)first, wave & 1, m0 + 128 * (wave >> 1), n0 + 64 * (wave & 1), lane);
    }, rows, cols, g.K, nullptr, g.b2);
  } else if constexpr (OP == GatedOp::kBwd) {
    const uint32_t wave0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    KeptTile<KEPT, EDGE, 8, 8> kept;   // its first rows land under the loop, in the registers that the loop leaves
    kept.request(g, m0 + 128 * (wave0 >> 1), n0 + 128 * (wave0 & 1), threadIdx.x & 63, 0);
    gemm256_accumulate<false, B_OC, EDGE>(g.a, g.lda, g.b, g.ldb, nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane) {
      bwd_out<KEPT, EDGE, 8, 8>(g, acc, kept, (float*)cs, m0 + 128 * (wave >> 1), n0 + 128 * (wave & 1), lane);
    }, rows, cols, g.K);
  } else {
    gemm256_accumulate<false, B_OC, EDGE, 8, kTwo>(g.a, g.lda, g.b, g.ldb, 2 * nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane) {
      uint16_t* yw = g.h + (size_t)(m0 + 128 * (wave >> 1)) * g.ldh + n0 + 128 * (wave & 1);
      const int wr = (int)rows - 128 * (int)(wave >> 1), wc = (int)cols - 128 * (int)(wave & 1);
      epilogue_bf16_half<EDGE>(*reinterpret_cast<const f32x4 (*)[4][8]>(&acc[0]), 0, cs, yw, g.ldh, lane, NoHook{}, wr, wc);
      epilogue_bf16_half<EDGE>(*reinterpret_cast<const f32x4 (*)[4][8]>(&acc[4]), 1, cs, yw, g.ldh, lane, NoHook{}, wr, wc);
    }, rows, cols, g.K, g.a2, g.b2);
  }
}

bool gated256_applicable(const GatedArgs& g) { return g.K >= 64 && out_lds_ok(g) && g.lda < g256::kMaxLdEdge && g.ldb < g256::kMaxLdEdge; }

template <GatedOp OP, Kept KEPT, bool EDGE>
static int launch_tiles(GatedArgs g, bool b_oc, hipStream_t stream) {
  constexpr uint32_t TC = OP == GatedOp::kFwd ? 128 : 256;
  const uint32_t mt = (uint32_t)(((uint64_t)g.M + 255) / 256), nt = (uint32_t)(((uint64_t)g.N + TC - 1) / TC);
  if ((uint64_t)mt * nt >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  set_tile_grid(g, mt, nt, tile_band(mt, nt));
  if (b_oc) hipLaunchKernelGGL((gated256_kernel<OP, true, KEPT, EDGE>), dim3(mt * nt), dim3(256), 0, stream, g);
  else hipLaunchKernelGGL((gated256_kernel<OP, false, KEPT, EDGE>), dim3(mt * nt), dim3(256), 0, stream, g);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

template <GatedOp OP, Kept KEPT>
static int launch_edge(const GatedArgs& g, bool b_oc, hipStream_t stream) {
  const bool whole = g.M % 256 == 0 && g.N % (OP == GatedOp::kFwd ? 128 : 256) == 0 && g.K % 64 == 0;
  return whole ? launch_tiles<OP, KEPT, false>(g, b_oc, stream) : launch_tiles<OP, KEPT, true>(g, b_oc, stream);
}

int launch_gated256(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream) {
  if (op == GatedOp::kDx) return launch_edge<GatedOp::kDx, Kept::kNone>(g, b_oc, stream);
  if (op == GatedOp::kBwd)
    return kept == Kept::kE4m3 ? launch_edge<GatedOp::kBwd, Kept::kE4m3>(g, b_oc, stream) : launch_edge<GatedOp::kBwd, Kept::kBf16>(g, b_oc, stream);
  return kept == Kept::kE4m3 ? launch_edge<GatedOp::kFwd, Kept::kE4m3>(g, b_oc, stream)
         : kept == Kept::kBf16 ? launch_edge<GatedOp::kFwd, Kept::kBf16>(g, b_oc, stream) : launch_edge<GatedOp::kFwd, Kept::kNone>(g, b_oc, stream);
}

}  // namespace gws
