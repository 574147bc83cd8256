// The dense layer's products in 128 x 128 and 128 x 96 tiles (gfx950): the loop of gemm128_kernel, its sums through gws_dense_out.h.
#include "gws_dense_out.h"
#include "gws_gemm128_core.h"

namespace gws {

int launch_dense128(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, int nj, hipStream_t stream) {
  if (op == DenseOp::kFwd) {
    const DenseWay<DenseOp::kFwd> way{d};
    return nj == 3 ? launch_middle_tiles<3>(g, w_is_nk, stream, way) : launch_middle_tiles<4>(g, w_is_nk, stream, way);
  }
  const DenseWay<DenseOp::kBwd> way{d};
  return nj == 3 ? launch_middle_tiles<3>(g, w_is_nk, stream, way) : launch_middle_tiles<4>(g, w_is_nk, stream, way);
}

}  // namespace gws
