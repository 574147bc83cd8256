// The dense layer's products in 128 x 128 and 128 x 96 tiles (gfx950): the loop of gemm128_kernel, its sums through gws_dense_out.h.
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
