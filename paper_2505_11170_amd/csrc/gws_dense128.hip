// The dense layer's products in 128 x 128 and 128 x 96 tiles (gfx950): the loop of gemm128_kernel, its sums through gws_dense_out.h.  For some thousand rows and for
// up to one round of tiles: 4096 x 768 -> 2048 with Z kept 20.2 us, bound by the tiles' operands out of the L2 and the way out.  `shared`: two LDS stages
// instead of four, so two workgroups a compute unit, and one's way out runs under the other's loop (5469 x 5632 -> 800 104 -> 70 us).
#include "gws_dense_out.h"
#include "gws_gemm128_core.h"

namespace gws {

template <DenseOp OP>
static int launch_form(const GemmArgs& g, const DenseArgs& d, int w_is_nk, int nj, bool shared, hipStream_t stream) {
  const DenseWay<OP> way{d};
  if (shared) return launch_middle_tiles<4, 2>(g, w_is_nk, stream, way);
  return nj == 3 ? launch_middle_tiles<3>(g, w_is_nk, stream, way) : launch_middle_tiles<4>(g, w_is_nk, stream, way);
}
int launch_dense128(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, int nj, bool shared, hipStream_t stream) {
  return op == DenseOp::kFwd ? launch_form<DenseOp::kFwd>(g, d, w_is_nk, nj, shared, stream) : launch_form<DenseOp::kBwd>(g, d, w_is_nk, nj, shared, stream);
}

}  // namespace gws
