// The dense layer's products for few rows or few tiles (gfx950): the kernel of gws_gemm_stream_kernel.h, its partial sums through gws_dense_out.h.  One token, 2048 -> 5632: 4.0
// us, bound by the weight's bytes (5.8 TB/s); 64 tokens 8.3; 1021 x 2048 -> 768 with the residual 9.6, bound by latency: launch, first bytes, the wavefronts' sums.
#include "gws_dense_out.h"
#include "gws_gemm_stream_kernel.h"

namespace gws {

int launch_dense_stream(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, const StreamPlan& p, hipStream_t stream) {
  if (op == DenseOp::kFwd) return launch_stream_tiles(g, w_is_nk, p, stream, DenseWay<DenseOp::kFwd>{d});
  return launch_stream_tiles(g, w_is_nk, p, stream, DenseWay<DenseOp::kBwd>{d});
}

}  // namespace gws
