// Launch arguments of the AdamW step and of the gradients' norm (internal to csrc/).
#pragma once

#include "gws_device.h"
#include "gws_launch.h"

namespace gws {

// A tensor as the kernels see it.
struct AdamwDesc {
  float* p;
  uint16_t* w;                 // may be NULL
  const void* g;
  void *m, *v;                 // fp32, or E4M3 codes with scales ms, vs
  uint8_t *ms, *vs;
  uint32_t rows, cols, ld, lds;
  float keep, rate;            // 1 - lr wd; lr / c1
  uint32_t seed_lo, seed_hi;
  uint32_t per_row, inv;       // groups of elements a row (of 4, whole blocks of 32 where the states are codes; the norm: of 8)
  uint32_t first_wg;           // this tensor's first workgroup within the launch
  uint32_t form;               // bit 0: g is fp32; bit 1: the states are codes; bit 2: fewer than 2^32 groups
};
static_assert(sizeof(AdamwDesc) == 104, "descriptor layout");
constexpr uint32_t kGradFp32 = 1, kCodes = 2, kFewGroups = 4;
constexpr int kAdamwTensors = 54;    // of a launch
struct AdamwArgs {
  uint32_t begin[kAdamwTensors];     // first workgroups; entries past the last tensor hold 0x7FFFFFFF
  AdamwDesc t[kAdamwTensors];
  float beta1, one1, beta2, one2, root2, eps;   // one1 = 1 - beta1, one2 = 1 - beta2, root2 = 1 / sqrt(c2)
  uint32_t step_lo, step_hi;
  const float* grad_scale;           // may be NULL
  double* part;                      // the norm's sums, one a workgroup of this launch
};
static_assert(sizeof(AdamwArgs) <= 6144, "kernel arguments: keep within the size verified on the device");

constexpr uint32_t kAdamwGroups = 512;    // groups of four that a workgroup updates
constexpr uint32_t kNormGroups = 2048;    // groups of eight whose squares a workgroup adds up
// all: codes in every tensor of the launch (2), in none (0), or in some (1)
int launch_adamw(const AdamwArgs& a, uint32_t wgs, int codes, hipStream_t stream);
int launch_grad_squares(const AdamwArgs& a, uint32_t wgs, hipStream_t stream);
int launch_grad_norm(const double* part, uint64_t n, double max_norm, float* out, hipStream_t stream);

}  // namespace gws
