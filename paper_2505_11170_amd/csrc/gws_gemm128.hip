// Middle-tile BF16 MFMA GEMM for gfx950: Y[M x N] = X[M x K] * W (W stored [K x N] or [N x K]), any M, N and K of whole
// 32s.  For products with too few 256 x 256 tiles to fill the chip, or with edges that the large tile would pad.
//
// Workgroup = 2 x 2 wavefronts, tile 128 x 32 NJ (NJ 4 or 3), K-steps of 64; a wavefront owns 64 x 16 NJ of the output as 4 x NJ
// v_mfma_f32_16x16x32_bf16 tiles.  Both operand tiles (16 KiB, and 16 or 12) go global -> LDS directly into a ring of four stages,
// in the layouts of gws_gemm256_core.h (96 columns of a [K x N] weight as in gws_gemm_stream_core.h), three K-steps ahead; one
// barrier a K-step, between its two 32-deep halves: the second half's fragments are read under the first half's MFMAs, the next
// step's first ones under the second half's.
// What bounds it: a K-step of 128 x 128 takes 0.41 us (W [N x K]; 0.43 for [K x N]), of which the operands' 32 KiB from L2 alone 0.34, the
// MFMAs alone 0.25 and the LDS reads alone 0.17; misses in L2 are not it (0.39 without any).  A launch starts and
// ends in 5.7 us (6.0 with divisions in the tile numbering and the arguments in memory).
// 128 x 96 is for the sizes whose 128 x 128 tiles leave compute units idle in their rounds: 4096 x 3072 -> 768 is 256 tiles instead of
// 192, one round of either, 27.7 -> 23.7 us (816 TFLOP/s); 1000 x 768 -> 2304 8.7 -> 7.9; 3500 x 3008 -> 800 24.6 -> 21.2; 8192 x 2304
// -> 768, two rounds, 35.9 -> 32.8.  All of W [K x N]; [N x K] alike.  Each element's sum runs in the same order in both.
#include "gws_gemm128_core.h"

namespace gws {

bool gemm128_applicable(const GemmArgs& g) {
  return g.M > 0 && g.N > 0 && g.N % 32 == 0 && g.K % 32 == 0 && g.K >= 64 && g.ldx < g128::kMaxLd && g.ldw < g128::kMaxLd;
}

int launch_gemm128(const GemmArgs& g, int w_is_nk, int nj, hipStream_t stream) {
  return nj == 3 ? launch_middle_tiles<3>(g, w_is_nk, stream) : launch_middle_tiles<4>(g, w_is_nk, stream);
}

}  // namespace gws
