// Launch arguments of the AdamW step and of the gradients' norm (internal to csrc/).
#pragma once

#include "gws_device.h"
#include "gws_launch.h"

namespace gws {

// What all tensors of a call share.
struct AdamwStep {
  float beta1, one1, beta2, one2, root2, eps;   // one1 = 1 - beta1, one2 = 1 - beta2, root2 = 1 / sqrt(c2)
  uint32_t step_lo, step_hi;
  const float* grad_scale;                      // may be NULL
};
constexpr uint32_t kGradFp32 = 1, kCodes = 2, kFewGroups = 4;   // bits of a descriptor's form: g is fp32; the states are codes; fewer than 2^32 groups

// A tensor with fp32 states and no gaps (one row, or rows that follow each other): a run of elements.
struct AdamwRun {
  float* p;
  uint16_t* w;                 // may be NULL
  const void* g;
  float *m, *v;
  uint64_t n;                  // elements; the highest bit: g is fp32
  float keep, rate;            // 1 - lr wd; lr / c1
};
constexpr uint64_t kRunGradFp32 = (uint64_t)1 << 63;
// Any other tensor.
struct AdamwMatrix {
  float* p;
  uint16_t* w;                 // may be NULL
  const void* g;
  void *m, *v;                 // fp32, or E4M3 codes with scales ms, vs
  uint8_t *ms, *vs;
  uint32_t rows, cols, ld, lds;
  float keep, rate;
  uint32_t seed_lo, seed_hi;
  uint32_t per_row, inv;       // groups of four elements a row (codes: of whole blocks of 32)
  uint32_t form, unused;
};
struct GradSquares {           // of the norm: a tensor's gradient
  const void* g;
  uint32_t rows, cols, ld;     // highest bit of rows: g is fp32; of cols: fewer than 2^32 groups
  uint32_t inv;                // of the groups of eight a row
};
constexpr uint32_t kHighBit = 0x80000000u;
// The tensors of a launch: first workgroups (entries past the last one hold 0x7FFFFFFF) and descriptors, as many as the kernel arguments hold.
template <class Desc, int N>
struct TensorList {
  static constexpr int kMax = N;
  uint32_t begin[N];
  Desc t[N];
};
using AdamwRuns = TensorList<AdamwRun, 100>;
using AdamwMatrices = TensorList<AdamwMatrix, 54>;
using GradList = TensorList<GradSquares, 216>;
constexpr size_t kArgumentBytes = 6144;   // verified on the device
static_assert(sizeof(AdamwRuns) + sizeof(AdamwStep) <= kArgumentBytes && sizeof(AdamwMatrices) + sizeof(AdamwStep) <= kArgumentBytes &&
              sizeof(GradList) + 8 <= kArgumentBytes, "kernel arguments");

constexpr uint32_t kAdamwGroups = 512;    // groups of four that a workgroup updates
constexpr uint32_t kNormGroups = 2048;    // groups of eight whose squares a workgroup adds up
int launch_adamw_runs(const AdamwRuns& t, const AdamwStep& s, uint32_t wgs, hipStream_t stream);
// codes: in every tensor of the launch (2), in none (0), or in some (1)
int launch_adamw_matrices(const AdamwMatrices& t, const AdamwStep& s, uint32_t wgs, int codes, hipStream_t stream);
int launch_grad_squares(const GradList& t, double* part, uint32_t wgs, hipStream_t stream);
int launch_grad_norm(const double* part, uint64_t n, double max_norm, float* out, hipStream_t stream);

}  // namespace gws
