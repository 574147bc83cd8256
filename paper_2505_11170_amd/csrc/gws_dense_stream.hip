// The dense layer's products for few rows or few tiles (gfx950): the kernel of gws_gemm_stream_kernel.h, its partial sums through gws_dense_out.h.
#include "gws_dense_out.h"
#include "gws_gemm_stream_kernel.h"

namespace gws {

int launch_dense_stream(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, const StreamPlan& p, hipStream_t stream) {
  if (op == DenseOp::kFwd) return launch_stream_tiles(g, w_is_nk, p, stream, DenseWay<DenseOp::kFwd>{d});
  return launch_stream_tiles(g, w_is_nk, p, stream, DenseWay<DenseOp::kBwd>{d});
}

}  // namespace gws
