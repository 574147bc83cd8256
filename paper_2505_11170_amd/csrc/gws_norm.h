// Launch arguments and device helpers of the norms, the dense layer and the sums over tokens (internal to csrc/).
#pragma once

#include "gws_device.h"
#include "gws_launch.h"

namespace gws {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef f4 f4_any __attribute__((aligned(4)));   // fp32 vectors may start at any element: global memory takes dword-aligned wide accesses

__device__ __forceinline__ float lo_of(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float hi_of(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// Eight BF16 values from column c (a multiple of eight) of a row of C; what lies past the row is not touched and reads as zeros.  Of a row's last C % 8 values four, two
// and one are an access each, chosen by uniform branches (backward 1021 x 999 23.9 -> 11.4 us, 4096 x 700 18.1 -> 14.8 beside an access a value).
__device__ __forceinline__ u32x4 load_eight(const GWS_GLOBAL uint16_t* row, uint32_t c, uint32_t C) {
  u32x4 v = {0, 0, 0, 0};
  if (c + 8 <= C) {
    v = *(const GWS_GLOBAL u32x4*)(row + c);
  } else if (c < C) {
    const GWS_GLOBAL uint16_t* p = row + c;
    if (C & 4) {
      const u32x2 w = *(const GWS_GLOBAL u32x2*)p;
      v[0] = w[0];
      v[1] = w[1];
      if (C & 2) {
        v[2] = *(const GWS_GLOBAL uint32_t*)(p + 4);
        if (C & 1) v[3] = p[6];
      } else if (C & 1) {
        v[2] = p[4];
      }
    } else if (C & 2) {
      v[0] = *(const GWS_GLOBAL uint32_t*)p;
      if (C & 1) v[1] = p[2];
    } else {
      v[0] = p[0];
    }
  }
  return v;
}
__device__ __forceinline__ void store_eight(GWS_GLOBAL uint16_t* row, uint32_t c, uint32_t C, const u32x4& v) {
  if (c + 8 <= C) {
    *(GWS_GLOBAL u32x4*)(row + c) = v;
  } else if (c < C) {
    GWS_GLOBAL uint16_t* p = row + c;
    if (C & 4) {
      *(GWS_GLOBAL u32x2*)p = u32x2{v[0], v[1]};
      if (C & 2) {
        *(GWS_GLOBAL uint32_t*)(p + 4) = v[2];
        if (C & 1) p[6] = (uint16_t)v[3];
      } else if (C & 1) {
        p[4] = (uint16_t)v[2];
      }
    } else if (C & 2) {
      *(GWS_GLOBAL uint32_t*)p = v[0];
      if (C & 1) p[2] = (uint16_t)v[1];
    } else {
      p[0] = (uint16_t)v[0];
    }
  }
}
__device__ __forceinline__ void widen(const u32x4& v, float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f[2 * k] = lo_of(v[k]);
    f[2 * k + 1] = hi_of(v[k]);
  }
}
__device__ __forceinline__ u32x4 narrow(const float (&f)[8]) {
  return u32x4{pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7])};
}
// Eight fp32 values of a vector of C; p == NULL: `other` in their place.
__device__ __forceinline__ void vector_eight(const float* p, uint32_t c, uint32_t C, float other, float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = other;
  if (p == nullptr) return;
  if (c + 8 <= C) {
    const f4 a = *(const GWS_GLOBAL f4_any*)global_ptr<float>(p + c), b = *(const GWS_GLOBAL f4_any*)global_ptr<float>(p + c + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[k] = a[k];
      f[4 + k] = b[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (c + k < C) f[k] = p[c + k];
  }
}

// The sum over L = 16, 32 or 64 neighbouring lanes, in each of them: DPP within rows of 16, then swaps.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  v += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(v)));    // lane ^ 1
  v += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(v)));    // lane ^ 2
  v += __uint_as_float(dpp_u32<0x141>(__float_as_uint(v)));   // the other four of eight
  v += __uint_as_float(dpp_u32<0x140>(__float_as_uint(v)));   // the other eight of sixteen
  if (L > 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (L > 32) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  return v;
}

// Workgroups in a grid of two dimensions: one has fewer than 2^32 threads.
constexpr uint32_t kGridWidth = 1u << 20;
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridWidth + blockIdx.x; }
inline dim3 grid_of(uint64_t workgroups) {
  return workgroups <= kGridWidth ? dim3((uint32_t)workgroups) : dim3(kGridWidth, (uint32_t)((workgroups + kGridWidth - 1) / kGridWidth));
}

// Columns of partial sums added up: out[c] = sum over p < P of part[p * n + c] for c < n, columns from n0 on to out1.
int launch_sum_partials(const float* part, uint32_t P, uint64_t n, uint64_t n0, float* out0, float* out1, hipStream_t stream);
int launch_zero(float* p, uint64_t n, hipStream_t stream);

struct NormArgs {
  const uint16_t *x, *dy, *r;
  uint16_t* y;                    // Y or dX
  const float *gamma, *beta;
  float *mean, *rstd;             // written forward, read backward
  float* part;                    // backward: partial dgamma and dbeta, [workgroups][wanted C]
  float* rows;                    // backward, wide rows: sum(t) / C and sum(t n) / C of every row
  uint32_t M, C, ldx, lddy, ldr, ldy;
  float eps;
  bool want_gamma, want_beta;
};
int launch_norm_fwd(const NormArgs& a, bool rms, hipStream_t stream);
uint32_t norm_bwd_parts(uint64_t M, uint64_t C);   // partial sums of dgamma and dbeta
bool norm_is_wide(uint64_t C);
int launch_norm_bwd(const NormArgs& a, bool rms, float* dgamma, float* dbeta, hipStream_t stream);

}  // namespace gws
