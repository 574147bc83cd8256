// The dense layer: launch arguments and the arithmetic on its sums, shared by its kernels (internal to csrc/).
#pragma once

#include "gws_gated.h"
#include "gws_norm.h"

namespace gws {

// What happens to the sums of a product (GemmArgs: x, w, y) on their way out.
//   forward : Z = sum + bias, kept in z; Y = a(Z) + r
//   backward: dZ = sum a'(Z) to y, H = a(Z) to h, and the columns' sums over the tile's rows to part[tile row][N]
struct DenseArgs {
  const float* bias;      // may be NULL
  const uint16_t* r;      // may be NULL
  uint16_t* z;            // forward: written, may be NULL; backward: read (NULL only without activation)
  uint16_t* h;            // may be NULL
  float* part;            // may be NULL
  uint32_t ldr, ldz, ldh;
  int act;
  bool past_caches;       // forward: Y, backward: dZ and H, of the large tiles
};
enum class DenseOp { kFwd = 0, kBwd = 1 };
// The way out of a product's kernels (gws_dense_out.h).
template <DenseOp OP>
struct DenseWay {
  DenseArgs d;
};

// The activation that is none.
struct NoGate {
  __device__ static __forceinline__ float a(float z) { return z; }
  __device__ static __forceinline__ void both(float z, float& a, float& slope) {
    a = z;
    slope = 1.0f;
  }
};
// GELU without the gate's bound on z^2: where z^2 is infinite, exp's argument is an infinity of the right sign, and q is 0 or 1 all the same.
struct GeluGate : Gate<GWS_ACT_GELU_TANH> {
  __device__ static __forceinline__ float a(float z) { return z * logistic(z * __fmaf_rn(-kLog2e * kGelu3, z * z, -kLog2e * kGelu1)); }
};
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {   // a uniform branch
  if (act == GWS_ACT_NONE) f(NoGate());
  else if (act == GWS_ACT_SILU) f(Gate<GWS_ACT_SILU>());
  else f(GeluGate());
}
inline bool known_dense_act(int act) { return act == GWS_ACT_NONE || known_act(act); }

// Which kernel, and how many rows of the result one row of partial sums stands for.
struct DensePlan {
  GemmForm form;         // kAnyShape: dense_any_kernel
  RoutePlan route;
  bool shared;           // kMiddle: two workgroups a compute unit
  uint32_t rows;
};
DensePlan plan_dense(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk);
// 256 x 256 tiles (whole, or with edges), 256 x 192
int launch_dense256(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, GemmForm form, hipStream_t stream);
// tiles of 128 x 32 nj; shared: of 128 x 128, two workgroups a compute unit
int launch_dense128(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, int nj, bool shared, hipStream_t stream);
int launch_dense_stream(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk, const StreamPlan& p, hipStream_t stream);
// every size
int launch_dense_any(const GemmArgs& g, const DenseArgs& e, DenseOp op, int w_is_nk, hipStream_t stream);
constexpr uint32_t kDenseAnyRows = 64;   // of its tiles, for the partial sums
// from a given dH (x, ldx): rows of tokens a workgroup takes
uint32_t dense_h_rows(uint64_t M, uint64_t F);
int launch_dense_bwd_h(const GemmArgs& g, const DenseArgs& e, hipStream_t stream);

}  // namespace gws
