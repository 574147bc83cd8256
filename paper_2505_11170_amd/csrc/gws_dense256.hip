// The dense layer's products in 256 x 256 and 256 x 192 tiles (gfx950): the loop of gws_gemm256_core.h, its sums through gws_dense_out.h.  Each of the four
// wavefronts has 128 x 16 NJ of the tile, and a row of partial sums.  8192 x 2048 -> 5632 GELU, Z kept 160 to 171 us by box (1.11 to 1.18 PFLOP/s; the plain product
// 142), backward with H and the bias gradient 182 to 190: the loop at the rate of the plain product's, then the way out, which all compute units reach together.
#include "gws_dense_out.h"

namespace gws {

template <DenseOp OP, bool W_NK, bool EDGE, int NJ>
__global__ __launch_bounds__(256, 1) void dense_gemm256_kernel(const GemmArgs g, const DenseArgs d) {
  using namespace g256;
  constexpr uint32_t TC = 32 * NJ;
  uint32_t tile_m, tile_n;
  tile_of(TileGrid{(g.M + TM - 1) / TM, (g.N + TC - 1) / TC, g.inv_band, g.inv_last}, blockIdx.x, tile_m, tile_n);
  const uint32_t m0 = tile_m * TM, n0 = tile_n * TC, rows = g.M - m0 < TM ? g.M - m0 : TM, cols = g.N - n0 < TC ? g.N - n0 : TC;
  const uint32_t wave0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  DenseHeld<OP, EDGE, 8, NJ> held;   // lands under the loop, in the registers that it leaves
  held.begin(g, d, m0 + 128 * (wave0 >> 1), n0 + 16 * NJ * (wave0 & 1), threadIdx.x & 63);
  gemm256_accumulate<false, !W_NK, EDGE, NJ>(g.x, g.ldx, g.w, g.ldw, (g.K + TK - 1) / TK, m0, n0,
                                             [&](f32x4 (&acc)[8][NJ], uint16_t* cs, uint32_t wave, uint32_t lane) {
    const uint32_t p0 = m0 + 128 * (wave >> 1);
    dense_out<OP, EDGE, 8, NJ>(g, d, acc, held, (float*)cs, p0, n0 + 16 * NJ * (wave & 1), lane, p0 / 128);
  }, rows, cols, g.K);
}

template <DenseOp OP, bool EDGE, int NJ>
static int launch_tiles(GemmArgs g, const DenseArgs& d, int w_is_nk, hipStream_t stream) {
  constexpr uint32_t TC = 32 * NJ;
  const uint32_t mt = (uint32_t)(((uint64_t)g.M + g256::TM - 1) / g256::TM), nt = (uint32_t)(((uint64_t)g.N + TC - 1) / TC);
  if ((uint64_t)mt * nt >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  set_tile_grid(g, mt, nt, NJ == 8 ? tile_band(mt, nt) : 8);
  if (w_is_nk) hipLaunchKernelGGL((dense_gemm256_kernel<OP, true, EDGE, NJ>), dim3(mt * nt), dim3(256), 0, stream, g, d);
  else hipLaunchKernelGGL((dense_gemm256_kernel<OP, false, EDGE, NJ>), dim3(mt * nt), dim3(256), 0, stream, g, d);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

template <DenseOp OP>
static int launch_form(const GemmArgs& g, const DenseArgs& d, int w_is_nk, GemmForm form, hipStream_t stream) {
  if (form == GemmForm::kNarrow) return launch_tiles<OP, true, 6>(g, d, w_is_nk, stream);
  return form == GemmForm::kLarge ? launch_tiles<OP, false, 8>(g, d, w_is_nk, stream) : launch_tiles<OP, true, 8>(g, d, w_is_nk, stream);
}
int launch_dense256(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, GemmForm form, hipStream_t stream) {
  return op == DenseOp::kFwd ? launch_form<DenseOp::kFwd>(g, d, w_is_nk, form, stream) : launch_form<DenseOp::kBwd>(g, d, w_is_nk, form, stream);
}

}  // namespace gws
