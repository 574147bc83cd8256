// The gate of the feed-forward block and the 8-bit form of activations: device arithmetic and launch arguments shared by
// their kernels (internal to csrc/).
//
//   gate: with q = 1 / (1 + exp(-w(g))), a(g) = g q and a'(g) = q + g q (1 - q) w'(g); w(g) is g itself for
//   SiLU (a = g times the logistic function of g) and 2 sqrt(2/pi) (g + 0.044715 g^3) for the tanh form of GELU, since
//   (1 + tanh z) / 2 is the logistic function of 2 z.
//   8 bits: 32 neighbouring values of a row share X = 2^(byte - 127), the smallest for which the largest of them rounds to at
//   most 448, the largest E4M3 value (1.8125 2^8 = 464 is the tie with what would be the next one and goes to 448), from 2^-117 to
//   2^119 (values saturate at 448 2^119): every decoded value is then zero or a finite normal BF16 value, so decoding is exact.
#pragma once

#include "gws_device.h"
#include "gws_launch.h"

namespace gws {

constexpr uint32_t kAct8Min = 10, kAct8Max = 246, kAct8Zero = 127, kAct8NaN = 255;

// The scale's byte from the fp32 bits of a block's largest magnitude.  A NaN or infinity in the block makes its scale NaN.
__device__ __forceinline__ uint32_t act8_byte(uint32_t amax) {
  const int b = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x680000u ? 1 : 0);
  const uint32_t byte = (uint32_t)(b < (int)kAct8Min ? (int)kAct8Min : b > (int)kAct8Max ? (int)kAct8Max : b);
  return amax == 0 ? kAct8Zero : amax >= 0x7F800000u ? kAct8NaN : byte;
}
// X for the converters (a NaN scale's blocks are written and read apart from them).
__device__ __forceinline__ float act8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// X for the converters from the same bits where no value is large: below 2^119, and what a block of zeros is divided by does not matter.
constexpr uint32_t kAct8Large = 0x7F000000u;   // from 2^127: the largest scale may be needed, or there is a NaN or an infinity
__device__ __forceinline__ float act8_small_scale(uint32_t amax) {
  const uint32_t e = (amax + 0x17FFFFu) >> 23;   // one more beyond 1.8125 2^x
  return __uint_as_float(((e < kAct8Min + 8 ? kAct8Min + 8 : e) << 23) - (8u << 23));
}
// The larger magnitude of m and two values; a NaN stays one.
__device__ __forceinline__ float act8_larger(float m, float a, float b) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(a)), __builtin_fabsf(b));
}
// The converter does not saturate: where a scale is the largest one (hardly ever), its values first.
__device__ __forceinline__ float act8_clamp(float v) { return fminf(fmaxf(v, -0x1.cp127f), 0x1.cp127f); }
// Four fp32 values to codes.
__device__ __forceinline__ uint32_t act8_convert(const float (&v)[4], float scale) {
  i16x2 c = {0, 0};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v[0], v[1], scale, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v[2], v[3], scale, true);
  uint32_t u;
  __builtin_memcpy(&u, &c, 4);
  return u;
}
// NaN codes under a NaN scale.
__device__ __forceinline__ uint32_t act8_codes(const float (&v)[4], uint32_t byte) {
  const uint32_t u = act8_convert(v, act8_scale(byte));
  return byte == kAct8NaN ? 0x7F7F7F7Fu : u;
}
// Codes as the converters take them: under a NaN scale NaN codes, whatever they are.
__device__ __forceinline__ uint32_t act8_read(uint32_t codes, uint32_t byte) { return byte == kAct8NaN ? 0x7F7F7F7Fu : codes; }
// Two of four codes (HI: the upper two) to fp32.
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <bool HI>
__device__ __forceinline__ f32x2 act8_values(uint32_t codes, uint32_t byte) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, act8_scale(byte), HI);
}
// The same to a packed BF16 pair.
template <bool HI>
__device__ __forceinline__ uint32_t act8_pair(uint32_t codes, uint32_t byte) {
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, act8_scale(byte), HI);
  uint32_t u;
  __builtin_memcpy(&u, &r, 4);
  return u;
}

// q, a(g) and a'(g) of an activation.  g^2 stays finite: beyond it q is 0 or 1 and what it is multiplied by is 0.
constexpr float kLog2e = 1.44269504088896340736f, kGelu1 = 1.5957691216057307118f, kGelu3 = 0.0713548162726009f;   // 2 sqrt(2/pi), that times 0.044715
template <int ACT>
struct Gate {
  __device__ static __forceinline__ float logistic(float minus_w_log2e) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(minus_w_log2e)); }
  __device__ static __forceinline__ float square(float g) { return fminf(g * g, 3.0e38f); }
  __device__ static __forceinline__ float a(float g) {
    if (ACT == GWS_ACT_SILU) return g * logistic(g * -kLog2e);
    return g * logistic(g * __fmaf_rn(-kLog2e * kGelu3, square(g), -kLog2e * kGelu1));
  }
  __device__ static __forceinline__ void both(float g, float& a, float& slope) {
    if (ACT == GWS_ACT_SILU) {
      const float q = logistic(g * -kLog2e);
      a = g * q;
      slope = q + __fmaf_rn(-a, q, a);
    } else {
      const float g2 = square(g), q = logistic(g * __fmaf_rn(-kLog2e * kGelu3, g2, -kLog2e * kGelu1));
      a = g * q;
      slope = __fmaf_rn(__fmaf_rn(-a, q, a), __fmaf_rn(3.0f * kGelu3, g2, kGelu1), q);
    }
  }
};
// f(Gate<act>()) for the activation of a call: a uniform branch, not a kernel for each.
template <class F>
__device__ __forceinline__ void with_gate(int act, F&& f) {
  if (act == GWS_ACT_SILU) f(Gate<GWS_ACT_SILU>());
  else f(Gate<GWS_ACT_GELU_TANH>());
}
inline bool known_act(int act) { return act == GWS_ACT_SILU || act == GWS_ACT_GELU_TANH; }
__device__ __forceinline__ float bf16_lo(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// G and U as they are kept between the passes.
enum class Kept { kNone = 0, kBf16 = 1, kE4m3 = 2 };
struct KeptArgs {
  uint8_t *g, *u;            // BF16 or codes
  uint8_t *gs, *us;          // block scales of codes
  uint32_t ldg, ldu;         // of g and u, in elements
  uint32_t lsg, lsu;         // of gs and us, in bytes
};

// Kept values of four columns, on their way and as fp32.
template <Kept KEPT>
struct KeptFour {
  uint32_t lo, hi, byte;   // BF16 pairs, or codes and their scale
  __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* s, uint32_t ld, uint32_t ls, uint32_t row, uint32_t col) {
    if (KEPT == Kept::kBf16) {
      const uint64_t w = *(const uint64_t*)(p + ((size_t)row * ld + col) * 2);
      lo = (uint32_t)w;
      hi = (uint32_t)(w >> 32);
    } else {
      lo = *(const uint32_t*)(p + (size_t)row * ld + col);
      byte = s[(size_t)row * ls + (col >> 5)];
    }
  }
  __device__ __forceinline__ void values(float (&v)[4]) const {
    if (KEPT == Kept::kBf16) {
      v[0] = bf16_lo(lo); v[1] = bf16_hi(lo); v[2] = bf16_lo(hi); v[3] = bf16_hi(hi);
    } else {
      const uint32_t c = act8_read(lo, byte);
      const f32x2 a = act8_values<false>(c, byte), b = act8_values<true>(c, byte);
      v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    }
  }
};
template <Kept KEPT>
struct KeptFours {
  KeptFour<KEPT> g, u;
  __device__ __forceinline__ void load(const KeptArgs& k, uint32_t row, uint32_t col) {
    g.load(k.g, k.gs, k.ldg, k.lsg, row, col);
    u.load(k.u, k.us, k.ldu, k.lsu, row, col);
  }
};

// One product of the block: C[M x N] = A * B over K (and A2 * B2 over as many more, or A * B2 beside it).
struct GatedArgs {
  const uint16_t *a, *a2, *b, *b2;   // A [M x K]; B [K x N] (B_OC) or [N x K]
  uint32_t M, N, K, lda, ldb;
  uint32_t inv_band, inv_last;       // of the kernel's tile grid (TileGrid)
  int act;
  bool past_caches;                  // forward: H, backward: dL/dG, dL/dU and H; 128 and 256 tiles
  KeptArgs kept;
  uint16_t *h, *dg, *du;             // results: H; dL/dG and dL/dU; (input gradient: h)
  uint32_t ldh, ldd;
};
enum class GatedOp { kFwd = 0, kBwd = 1, kDx = 2 };

// 256 x 256 tiles (a pair of weights: 256 x 128 of each)
bool gated256_applicable(const GatedArgs& g);
int launch_gated256(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream);
// 128 x 128 tiles (a pair of weights: 128 x 64 of each)
bool gated128_applicable(const GatedArgs& g);
// two: two workgroups a compute unit (not the input gradient)
int launch_gated128(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, bool two, hipStream_t stream);
// few tokens or few tiles: the wavefronts of a workgroup split the contraction; the tile in units of 16 rows and 16 columns (of a pair of
// weights: half of them of each), the parts, and the estimated time; p == 0: not a shape for it
struct GatedStreamPlan {
  int mt, nt, p;
  double us;
};
GatedStreamPlan gated_stream_plan(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept);
int launch_gated_stream(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, const GatedStreamPlan& p, hipStream_t stream);
int launch_gated_any(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream);
int launch_gated_bwd_h(const GatedArgs& g, Kept kept, hipStream_t stream);   // a = dL/dH, lda
int launch_act8(bool encode, const void* x, uint64_t M, uint64_t C, uint64_t ldx, const gws_act8& o, hipStream_t stream);

}  // namespace gws
