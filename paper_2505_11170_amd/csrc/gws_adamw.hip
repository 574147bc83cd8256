// The AdamW step over many tensors and the norm of their gradients (gfx950).
//
// One pass over memory, four elements a lane; the tensors of a launch are found in its arguments (up to 100 runs of elements, 54 other matrices or 216 gradients), so a model's update is a few launches.
// Bound by memory: 28 bytes a parameter with fp32 states and BF16 gradients (twelve layers of width 768, 66 million, with the gradients' norm 384 us: 4.8 TB/s), 16.1 with
// states in 8 bits (four layers of width 2048, 160 million, 491 us: 5.2 TB/s).  Few parameters are bound by the host's call, 97 vectors 17 us of which the kernels take 11.
// 512 groups of four a workgroup: two loads of each buffer on their way a lane, and a workgroup a vector of up to 2048.
//
// States in 8 bits.  What is held is m and r = sqrt(v): v's range in a block squared would not fit E4M3's 2^18, r's does, and the step divides by
// r anyway.  In one step m and r move by a tenth to a thousandth of themselves, an E4M3 spacing is a sixteenth to an eighth: rounded to nearest they would
// stand still.  So they are rounded at random, in proportion to where the value lies between its neighbours: t = |v| / X as fp32 bits
// has 20 bits below an E4M3 value's (below 2^-6 those of t + 2^-6, whose spacing there is E4M3's), to which 16 random bits are added at bits 4 .. 19, and
// a half of the lowest; the carry decides.  The random bits are a Philox call for every four elements: a tenth of the time that their bytes take.
// An r that became 0 would make the next step's quotient up to 1 / sqrt(1 - beta2) too large: a positive one stays at least E4M3's smallest.
#include "gws_adamw.h"
#include "gws_gated.h"

namespace gws {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// The tensor of workgroup `wg`: a lane compares with the first workgroup of one in 64, and the lanes whose tensors begin before it are counted.  One round
// trip to the arguments, which lie in memory; a search by parts takes several, and a small call is hardly more than such trips.
template <int N>
__device__ __forceinline__ uint32_t tensor_of(const uint32_t (&begin)[N], uint32_t wg) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t before = 0;
#pragma unroll
  for (int k = 0; k < N; k += 64) {
    const uint32_t i = k + lane;
    const uint32_t first = begin[i < N ? i : N - 1];
    before += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(i < N && wg >= first));
  }
  return __builtin_amdgcn_readfirstlane(before - 1);   // the first one begins at 0
}
// Row and group within it of a matrix's group `id`; false past its end.
__device__ __forceinline__ bool place(uint64_t id, uint32_t rows, uint32_t per_row, uint32_t inv, bool few, uint32_t& row, uint32_t& group) {
  if (few) {   // uniform
    row = divide((uint32_t)id, per_row, inv);
    group = (uint32_t)id - row * per_row;
  } else {
    row = (uint32_t)(id / per_row);
    group = (uint32_t)(id - (uint64_t)row * per_row);
  }
  return id < (uint64_t)rows * per_row;
}

// Four elements of which `n` exist (the others read as zeros).
__device__ __forceinline__ f4 load_four(const float* p, size_t at, int n) {
  const GWS_GLOBAL float* q = global_ptr<float>(p) + at;
  if (n == 4) return *(const GWS_GLOBAL f4*)q;
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) v[e] = q[e];
  return v;
}
__device__ __forceinline__ void store_four(float* p, size_t at, int n, const f4& v) {
  GWS_GLOBAL float* q = global_ptr<float>(p) + at;
  if (n == 4) {
    *(GWS_GLOBAL f4*)q = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) q[e] = v[e];
  }
}
__device__ __forceinline__ f4 load_four_bf16(const void* p, size_t at, int n) {
  const GWS_GLOBAL uint16_t* q = global_ptr<uint16_t>(p) + at;
  if (n == 4) {
    const u2 w = *(const GWS_GLOBAL u2*)q;
    return f4{bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1])};
  }
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) v[e] = __uint_as_float((uint32_t)q[e] << 16);
  return v;
}
__device__ __forceinline__ uint32_t load_codes(const void* p, size_t at, int n) {
  const GWS_GLOBAL uint8_t* q = global_ptr<uint8_t>(p) + at;
  if (n == 4) return *(const GWS_GLOBAL uint32_t*)q;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) c |= (uint32_t)q[e] << (8 * e);
  return c;
}
__device__ __forceinline__ void store_codes(void* p, size_t at, int n, uint32_t c) {
  GWS_GLOBAL uint8_t* q = global_ptr<uint8_t>(p) + at;
  if (n == 4) {
    *(GWS_GLOBAL uint32_t*)q = c;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) q[e] = (uint8_t)(c >> (8 * e));
  }
}
__device__ __forceinline__ f4 values(uint32_t codes, uint32_t byte) {
  const uint32_t c = act8_read(codes, byte);
  const f32x2 a = act8_values<false>(c, byte), b = act8_values<true>(c, byte);
  return f4{a[0], a[1], b[0], b[1]};
}

// The scale's byte from the fp32 bits of a block's largest magnitude: X the smallest power of two with max <= 448 X, so that nothing is rounded up
// past 448.
__device__ __forceinline__ uint32_t state_byte(uint32_t amax) {
  const int b = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  const uint32_t byte = (uint32_t)(b < (int)kAct8Min ? (int)kAct8Min : b > (int)kAct8Max ? (int)kAct8Max : b);
  return amax == 0 ? kAct8Zero : amax >= 0x7F800000u ? kAct8NaN : byte;
}
// Four values to codes under that scale, each rounded at random by 16 bits.
template <bool ROOT>
__device__ __forceinline__ uint32_t state_codes(const f4& v, uint32_t byte, const uint32_t (&bits)[4]) {
  if (byte == kAct8NaN) return 0x7F7F7F7Fu;
  const float inverse = __uint_as_float((254u - byte) << 23);
  uint32_t out = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float t = fminf(__builtin_fabsf(v[e]) * inverse, 448.0f);   // beyond it only under the largest scale
    const bool small = t < 0x1p-6f;
    const uint32_t raw = __float_as_uint(small ? t + 0x1p-6f : t) + ((ROOT ? bits[e] >> 16 : bits[e] & 0xFFFFu) << 4) + 8u;
    uint32_t c = (raw >> 20) - (small ? 968u : 960u);
    if (ROOT) c = c == 0 && v[e] > 0.0f ? 1u : c;
    else c |= (__float_as_uint(v[e]) >> 24) & 0x80u;
    out |= c << (8 * e);
  }
  return out;
}
__device__ __forceinline__ uint32_t largest(const f4& v) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  m = max(m, dpp_u32<0xB1>(m));     // lane ^ 1
  m = max(m, dpp_u32<0x4E>(m));     // lane ^ 2
  return max(m, dpp_u32<0x141>(m)); // row_half_mirror: the other four of eight
}

// Four elements on their way and their update: of a run of elements (fp32 states), or of a row of a matrix.
template <bool CODES>
struct Four {
  f4 p, g, m, v;
  uint32_t mc, vc, mb, vb;
  uint32_t row, group;
  int n;
  size_t at, block;

  template <class Desc>
  __device__ __forceinline__ void load_at(const Desc& t, bool grad_fp32) {
    p = g = m = v = f4{0.0f, 0.0f, 0.0f, 0.0f};
    mc = vc = 0;
    mb = vb = kAct8Zero;
    if (n == 0) return;
    p = load_four(t.p, at, n);
    g = grad_fp32 ? load_four((const float*)t.g, at, n) : load_four_bf16(t.g, at, n);
    if constexpr (CODES) {
      mc = load_codes(t.m, at, n);
      vc = load_codes(t.v, at, n);
      mb = global_ptr<uint8_t>(t.ms)[block];
      vb = global_ptr<uint8_t>(t.vs)[block];
    } else {
      m = load_four((const float*)t.m, at, n);
      v = load_four((const float*)t.v, at, n);
    }
  }
  __device__ __forceinline__ void load(const AdamwRun& t, uint64_t id) {
    const uint64_t count = t.n & ~kRunGradFp32;
    at = 4 * id;
    n = at >= count ? 0 : count - at < 4 ? (int)(count - at) : 4;
    load_at(t, (t.n & kRunGradFp32) != 0);
  }
  __device__ __forceinline__ void load(const AdamwMatrix& t, uint64_t id) {
    const bool in = place(id, t.rows, t.per_row, t.inv, (t.form & kFewGroups) != 0, row, group);
    const uint32_t c = 4 * group;
    n = !in || c >= t.cols ? 0 : t.cols - c < 4 ? (int)(t.cols - c) : 4;
    at = (size_t)row * t.ld + c;
    block = (size_t)row * t.lds + (c >> 5);
    load_at(t, (t.form & kGradFp32) != 0);
  }
  // all lanes come here: the eight of a block meet
  template <class Desc>
  __device__ __forceinline__ void update(const Desc& t, const AdamwStep& a, float scale) {
    if (CODES) {
      m = values(mc, mb);
      v = values(vc, vb);
      v *= v;
    }
    f4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gs = g[e] * scale;
      m[e] = a.beta1 * m[e] + a.one1 * gs;
      v[e] = a.beta2 * v[e] + a.one2 * (gs * gs);
      r[e] = sqrtf(v[e]);
      p[e] = p[e] * t.keep - (t.rate * m[e]) / (r[e] * a.root2 + a.eps);
    }
    uint32_t mbyte = 0, vbyte = 0;
    if (CODES) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e >= n) m[e] = r[e] = 0.0f;   // a NaN scale makes NaN of what does not exist
      mbyte = state_byte(largest(m));
      vbyte = state_byte(largest(r));
    }
    if (n == 0) return;
    store_four(t.p, at, n, p);
    if (t.w != nullptr) {
      const u2 w = {pack_bf16_rne(p[0], p[1]), pack_bf16_rne(p[2], p[3])};
      GWS_GLOBAL uint16_t* q = global_ptr<uint16_t>(t.w) + at;
      if (n == 4) {
        *(GWS_GLOBAL u2*)q = w;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < n) q[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
    if constexpr (CODES) {
      const Philox4 x = philox4x32_10(group, row, a.step_lo, a.step_hi ^ 0x47414457u, t.seed_lo, t.seed_hi);
      const uint32_t bits[4] = {x.x0, x.x1, x.x2, x.x3};
      store_codes(t.m, at, n, state_codes<false>(m, mbyte, bits));
      store_codes(t.v, at, n, state_codes<true>(r, vbyte, bits));
      if ((group & 7) == 0) {
        global_ptr<uint8_t>(t.ms)[block] = (uint8_t)mbyte;
        global_ptr<uint8_t>(t.vs)[block] = (uint8_t)vbyte;
      }
    } else {
      store_four((float*)t.m, at, n, m);
      store_four((float*)t.v, at, n, v);
    }
  }
};

template <bool CODES, class Desc>
__device__ __forceinline__ void update_groups(const AdamwStep& a, const Desc& t, uint32_t wg, float scale) {
  constexpr int U = kAdamwGroups / 256;
  const uint64_t first = (uint64_t)wg * kAdamwGroups + threadIdx.x;
  Four<CODES> f[U];
#pragma unroll
  for (int u = 0; u < U; ++u) f[u].load(t, first + 256 * u);
#pragma unroll
  for (int u = 0; u < U; ++u) f[u].update(t, a, scale);
}

// *grad_scale, or 1; false where it is not finite: a step without a finite gradient norm is none.
__device__ __forceinline__ bool scale_of(const AdamwStep& s, float& scale) {
  scale = s.grad_scale != nullptr ? *s.grad_scale : 1.0f;
  return (__float_as_uint(scale) & 0x7F800000u) != 0x7F800000u;
}

}  // namespace

__global__ __launch_bounds__(256) void adamw_runs_kernel(const AdamwRuns l, const AdamwStep s) {
  float scale;
  if (!scale_of(s, scale)) return;   // uniform
  const uint32_t i = tensor_of(l.begin, blockIdx.x);
  update_groups<false>(s, l.t[i], blockIdx.x - l.begin[i], scale);
}

template <int CODES>
__global__ __launch_bounds__(256) void adamw_matrices_kernel(const AdamwMatrices l, const AdamwStep s) {
  float scale;
  if (!scale_of(s, scale)) return;   // uniform
  const uint32_t i = tensor_of(l.begin, blockIdx.x), wg = blockIdx.x - l.begin[i];
  const AdamwMatrix& t = l.t[i];
  if (CODES == 2 || (CODES == 1 && (t.form & kCodes))) update_groups<true>(s, t, wg, scale);
  else update_groups<false>(s, t, wg, scale);
}

int launch_adamw_runs(const AdamwRuns& t, const AdamwStep& s, uint32_t wgs, hipStream_t stream) {
  hipLaunchKernelGGL(adamw_runs_kernel, dim3(wgs), dim3(256), 0, stream, t, s);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}
int launch_adamw_matrices(const AdamwMatrices& t, const AdamwStep& s, uint32_t wgs, int codes, hipStream_t stream) {
  if (codes == 0) hipLaunchKernelGGL(adamw_matrices_kernel<0>, dim3(wgs), dim3(256), 0, stream, t, s);
  else if (codes == 1) hipLaunchKernelGGL(adamw_matrices_kernel<1>, dim3(wgs), dim3(256), 0, stream, t, s);
  else hipLaunchKernelGGL(adamw_matrices_kernel<2>, dim3(wgs), dim3(256), 0, stream, t, s);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

// ---- the norm ----
// Squares are added in fp64: gradients of 1e-20 and sums of a billion of them keep all their bits.
namespace {
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = red[0];
  for (uint32_t w = 1; w < blockDim.x / 64; ++w) s += red[w];
  return s;
}
}  // namespace

// Eight elements of a gradient, group `id` of it, as they lie in memory (BF16: the first half); zeros past its end.
__device__ __forceinline__ void load_group(const GradSquares& t, bool fp32, uint64_t id, u32x4 (&raw)[2]) {
  const uint32_t cols = t.cols & ~kHighBit;
  uint32_t row, group;
  raw[0] = raw[1] = u32x4{0, 0, 0, 0};
  if (!place(id, t.rows & ~kHighBit, (cols + 7) / 8, t.inv, (t.cols & kHighBit) != 0, row, group)) return;
  const uint32_t c = 8 * group;
  const size_t at = (size_t)row * t.ld + c;
  if (fp32) {   // uniform
    const GWS_GLOBAL uint32_t* q = global_ptr<uint32_t>(t.g) + at;
    if (c + 8 <= cols) {
      raw[0] = *(const GWS_GLOBAL u32x4*)q;
      raw[1] = *(const GWS_GLOBAL u32x4*)(q + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c + e < cols) raw[e >> 2][e & 3] = q[e];
    }
  } else {
    const GWS_GLOBAL uint16_t* q = global_ptr<uint16_t>(t.g) + at;
    if (c + 8 <= cols) {
      raw[0] = *(const GWS_GLOBAL u32x4*)q;
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c + e < cols) raw[0][e >> 1] |= (uint32_t)q[e] << (16 * (e & 1));
    }
  }
}
__device__ __forceinline__ double add_squares(double s, bool fp32, const u32x4 (&raw)[2]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double a = (double)(fp32 ? __uint_as_float(raw[0][e]) : bf16_lo(raw[0][e])), b = (double)(fp32 ? __uint_as_float(raw[1][e]) : bf16_hi(raw[0][e]));
    s = __fma_rn(b, b, __fma_rn(a, a, s));
  }
  return s;
}
// Groups first, first + 256, ...: U loads are on their way before the first sum (48 gradients of 768 x 1760 BF16 30.0 us, one load after the other 37.1).
template <int U, bool FP32>
__device__ __forceinline__ double squares_of(const GradSquares& t, uint64_t first) {
  double s = 0.0;
  for (uint32_t k = 0; k < kNormGroups / 256; k += U) {
    u32x4 raw[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) load_group(t, FP32, first + 256 * (k + u), raw[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) s = add_squares(s, FP32, raw[u]);
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(const GradList l, double* part) {
  __shared__ double red[4];
  const uint32_t i = tensor_of(l.begin, blockIdx.x);
  const GradSquares& t = l.t[i];
  const uint64_t first = (uint64_t)(blockIdx.x - l.begin[i]) * kNormGroups + threadIdx.x;
  double s = t.rows & kHighBit ? squares_of<4, true>(t, first) : squares_of<8, false>(t, first);   // uniform
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* part, const uint64_t n, const double max_norm, float* out) {
  __shared__ double red[16];
  double s = 0.0;
  for (uint64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_sum(s, red);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(s);
  const bool finite = norm < __builtin_inf();
  const float nan = __uint_as_float(0x7FC00000u);
  out[0] = finite ? (float)norm : nan;
  out[1] = !finite ? nan : max_norm > 0.0 && norm > max_norm ? (float)(max_norm / norm) : 1.0f;
}

int launch_grad_squares(const GradList& t, double* part, uint32_t wgs, hipStream_t stream) {
  hipLaunchKernelGGL(grad_squares_kernel, dim3(wgs), dim3(256), 0, stream, t, part);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}
int launch_grad_norm(const double* part, uint64_t n, double max_norm, float* out, hipStream_t stream) {
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, stream, part, n, max_norm, out);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

}  // namespace gws
