// Layer norm and root-mean-square norm, forward and backward (gfx950).
//
// One pass over memory: a row is in the registers of L lanes (16 to 512), 8 V columns a lane, from its load to its store; mean, squares of the deviations
// and, backward, sum(t) and sum(t n) are sums over lanes (DPP) and, with more than a wavefront's 64, over the wavefronts through LDS.  The variance is the sum of (x - mean)^2,
// not the difference of two sums: the row is there, and nothing cancels.
// Bound by memory: 8192 x 2048 forward 12.4 us (5.4 TB/s), backward with both vectors 27.7 in a graph (23.6 for the rows, 4.0 for the workgroups' sums); few rows by
// latency, 1 x 2048 2.2 us.  Up to 2048 columns a row is one wavefront's, whose sums need no barrier; up to 256, and
// between 512 and 768, a wavefront has several (20000 x 128 forward 6.9 -> 3.5 us, backward 13.0 -> 8.7; 8192 x 768 8.1 -> 6.8, 16.4 -> 14.8; 512 and 1024 columns lose by it).
// dgamma and dbeta are sums over the rows: every lane adds up its own columns over the rows that its wavefronts take, the workgroup's rows meet in
// LDS, and what workgroups leave is added by a second kernel, always in one order.
#include <algorithm>

#include "gws_norm.h"

namespace gws {

namespace {

// Sums of N values over the L lanes of a row, in each of them; `red` holds 2 x N x (wavefronts of the workgroup) floats.  With more than a wavefront all of the
// workgroup comes here, and the two halves of `red` alternate, so that one barrier a sum is enough.
template <int L, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* red, uint32_t& turn) {
  constexpr int W = L / 64;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lanes_sum<(L < 64 ? L : 64)>(v[n]);
  if (W <= 1) return;
  const uint32_t waves = blockDim.x >> 6, wave = threadIdx.x >> 6, first = wave / (W > 0 ? W : 1) * W;
  float* half = red + turn * N * waves;
  turn ^= 1;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) half[n * waves + wave] = v[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float s = half[n * waves + first];
#pragma unroll
    for (int w = 1; w < W; ++w) s += half[n * waves + first + w];
    v[n] = s;
  }
}

}  // namespace

// A row's mean and rstd, and its deviations in f; times `unit` the numbers stay what they are, for rows whose sums or squares would pass fp32's range (beyond 10^19 or
// so) 2^-80 of them.  Returns the sum of the deviations' squares.
constexpr float kSmallUnit = 0x1p-80f;
template <int L, int V, bool RMS>
__device__ __forceinline__ float row_statistics(const NormArgs& a, const GWS_GLOBAL uint16_t* x, uint32_t lane, float unit, float (&f)[V][8], float& mean, float& rstd,
                                               float* red, uint32_t& turn) {
  const float count = (float)a.C;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    widen(load_eight(x, (lane + k * L) * 8, a.C), f[k]);
    if (unit != 1.0f)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[k][e] *= unit;
  }
  mean = 0.0f;
  if (!RMS) {
    float s[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += f[k][e];
    team_sum<L>(s, red, turn);
    mean = s[0] / count;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t c = (lane + k * L) * 8;
      if (c + 8 <= a.C) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[k][e] -= mean;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[k][e] = c + e < a.C ? f[k][e] - mean : 0.0f;
      }
    }
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < V; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) q[0] = __fmaf_rn(f[k][e], f[k][e], q[0]);
  team_sum<L>(q, red, turn);
  rstd = 1.0f / sqrtf(q[0] / count + a.eps * unit * unit);
  return q[0];
}
// A sum of squares past fp32's range leaves 0 (or NaN where the mean was past it too): such a row is done again in the small unit.
__device__ __forceinline__ bool out_of_range(float rstd) { return !(rstd > 0.0f); }
// There eps times 2^-160 may be 0, which is right beside squares, but a constant row whose sum was past the range has none: its rstd is that of eps alone, in the
// numbers' own unit.  (Its mean is exact, a value of eight bits times a count of up to fourteen.  Rows that are not constant keep squares: a sum past the range
// of up to 16384 values has one of 2^114 and more, and so two that are 2^106 apart.)
__device__ __forceinline__ float rstd_alone(float eps) { return 1.0f / sqrtf(eps); }

// L lanes a row, V groups of eight columns a lane, R rows a workgroup at a time.
template <int L, int V, int R, bool RMS>
__global__ __launch_bounds__(L * R) void norm_fwd_kernel(const NormArgs a) {
  static_assert(L <= 64 || R == 1, "all of a workgroup does a row again, or wavefronts that share nothing");
  __shared__ float red[2 * L * R / 64];
  const uint32_t team = threadIdx.x / L, lane = threadIdx.x % L;
  uint32_t turn = 0;
  float gamma[V][8], beta[V][8];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    vector_eight(a.gamma, (lane + k * L) * 8, a.C, 1.0f, gamma[k]);
    vector_eight(a.beta, (lane + k * L) * 8, a.C, 0.0f, beta[k]);
  }
  for (uint32_t row = blockIdx.x * R + team; row < a.M; row += gridDim.x * R) {
    const GWS_GLOBAL uint16_t* x = global_ptr<uint16_t>(a.x) + (size_t)row * a.ldx;
    float f[V][8], mean, rstd, kept_mean, kept_rstd;
    row_statistics<L, V, RMS>(a, x, lane, 1.0f, f, mean, rstd, red, turn);
    kept_mean = mean;
    kept_rstd = rstd;
    if (out_of_range(rstd)) {   // the same in all lanes of a row
      const float squares = row_statistics<L, V, RMS>(a, x, lane, kSmallUnit, f, mean, rstd, red, turn);
      kept_mean = mean / kSmallUnit;
      kept_rstd = rstd * kSmallUnit;
      if (squares == 0.0f) rstd = kept_rstd = rstd_alone(a.eps);
    }
    if (lane == 0) {
      if (a.mean != nullptr) a.mean[row] = kept_mean;
      if (a.rstd != nullptr) a.rstd[row] = kept_rstd;
    }
    GWS_GLOBAL uint16_t* y = global_ptr<uint16_t>(a.y) + (size_t)row * a.ldy;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __fmaf_rn(f[k][e] * rstd, gamma[k][e], beta[k][e]);
      store_eight(y, (lane + k * L) * 8, a.C, narrow(o));
    }
  }
}

// Rows of any length: the row is read three times (out of the caches).
template <bool RMS>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(const NormArgs a) {
  __shared__ float red[2 * 16];
  uint32_t turn = 0;
  const uint32_t row = workgroup();
  if (row >= a.M) return;
  const GWS_GLOBAL uint16_t* x = global_ptr<uint16_t>(a.x) + (size_t)row * a.ldx;
  const float count = (float)a.C;
  float mean, rstd, variance, unit = 1.0f;
  for (;;) {
    mean = 0.0f;
    if (!RMS) {
      float s[1] = {0.0f};
      for (uint32_t c = threadIdx.x * 8; c < a.C; c += 8192) {
        float f[8], t = 0.0f;
        widen(load_eight(x, c, a.C), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) t += f[e] * unit;
        s[0] += t;
      }
      team_sum<1024>(s, red, turn);
      mean = s[0] / count;
    }
    float q[1] = {0.0f};
    for (uint32_t c = threadIdx.x * 8; c < a.C; c += 8192) {
      float f[8], t = 0.0f;
      widen(load_eight(x, c, a.C), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = f[e] * unit - mean;
        t = c + e < a.C ? __fmaf_rn(d, d, t) : t;
      }
      q[0] += t;
    }
    team_sum<1024>(q, red, turn);
    variance = q[0] / count;
    rstd = 1.0f / sqrtf(variance + a.eps * unit * unit);
    if (!out_of_range(rstd) || unit != 1.0f) break;   // the same in all threads
    unit = kSmallUnit;
  }
  float kept_mean = mean / unit, kept_rstd = rstd * unit;
  // Deviations of less than a BF16 spacing in the mean: a constant row maybe, whose sum has more bits than fp32 holds from 65537 columns on (a value has eight, the count
  // seventeen), and whose mean is then not its value.
  if (!RMS && variance <= 0x1p-16f * mean * mean) {   // the same in all threads
    const uint32_t first = x[0];
    float others[1] = {0.0f};
    for (uint32_t c = threadIdx.x; c < a.C; c += 1024) others[0] = x[c] != first ? 1.0f : others[0];
    team_sum<1024>(others, red, turn);
    if (others[0] == 0.0f) {
      mean = lo_of(first) * unit;
      kept_mean = lo_of(first);
      rstd = kept_rstd = rstd_alone(a.eps);
    }
  }
  if (threadIdx.x == 0) {
    if (a.mean != nullptr) a.mean[row] = kept_mean;
    if (a.rstd != nullptr) a.rstd[row] = kept_rstd;
  }
  GWS_GLOBAL uint16_t* y = global_ptr<uint16_t>(a.y) + (size_t)row * a.ldy;
  for (uint32_t c = threadIdx.x * 8; c < a.C; c += 8192) {
    float f[8], gamma[8], beta[8];
    widen(load_eight(x, c, a.C), f);
    vector_eight(a.gamma, c, a.C, 1.0f, gamma);
    vector_eight(a.beta, c, a.C, 0.0f, beta);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __fmaf_rn((f[e] * unit - mean) * rstd, gamma[e], beta[e]);
    store_eight(y, c, a.C, narrow(f));
  }
}

// n = (x - mean) rstd by halves: x - mean itself may pass fp32's range.  Columns past the row are zeros with dY = 0, and their n = -mean rstd, which the sums multiply by that 0,
// has to be finite.  It is but in constant rows (in others two values are a BF16 spacing apart, and rstd is at most 2^8 sqrt(2 C) / mean), where n is 0 in the row's columns:
// there it is made 0 in all of them.
struct Normalise {
  float half_mean, twice_rstd;
  __device__ __forceinline__ Normalise(float mean, float rstd) : half_mean(0.5f * mean), twice_rstd(2.0f * rstd) {
    if (__builtin_fabsf(half_mean * twice_rstd) == __builtin_inff()) twice_rstd = 0.0f;
  }
  __device__ __forceinline__ float operator()(float x) const { return __fmaf_rn(x, 0.5f, -half_mean) * twice_rstd; }
};

// Backward: dX of the rows from row0 on, R at a time, `step` apart; with SUMS dgamma and dbeta of the lane's columns over them.
// n = (x - mean) rstd and t = dY gamma of a row.
template <int L, int V, int R, bool RMS, bool SUMS>
__device__ __forceinline__ void bwd_rows(const NormArgs& a, uint32_t row0, uint32_t step, float (&dgamma)[V][8], float (&dbeta)[V][8], float* red) {
  const uint32_t team = threadIdx.x / L, lane = threadIdx.x % L;
  uint32_t turn = 0;
  float gamma[V][8];
#pragma unroll
  for (int k = 0; k < V; ++k) vector_eight(a.gamma, (lane + k * L) * 8, a.C, 1.0f, gamma[k]);
  const float count = (float)a.C;
  for (; row0 < a.M; row0 += step) {
    const uint32_t row = row0 + team;
    const bool live = row < a.M;
    if (L == 64 && !live) break;   // with fewer lanes a row a wavefront has several
    const size_t at = live ? row : row0;   // past the last row a neighbour's is read, and nothing stored
    const GWS_GLOBAL uint16_t *x = global_ptr<uint16_t>(a.x) + at * a.ldx, *dy = global_ptr<uint16_t>(a.dy) + at * a.lddy;
    u32x4 xr[V], yr[V], rr[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      xr[k] = load_eight(x, (lane + k * L) * 8, a.C);
      yr[k] = load_eight(dy, (lane + k * L) * 8, a.C);
      if (a.r != nullptr) rr[k] = load_eight(global_ptr<uint16_t>(a.r) + at * a.ldr, (lane + k * L) * 8, a.C);
    }
    const float rstd = a.rstd[at];
    const Normalise normal(RMS ? 0.0f : a.mean[at], rstd);
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < V; ++k) {   // columns past the row have dY = 0: they add nothing
      float n[8], d[8];
      widen(xr[k], n);
      widen(yr[k], d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[e] = normal(n[e]);
        const float t = d[e] * gamma[k][e];
        s[0] += t;
        s[1] = __fmaf_rn(t, n[e], s[1]);
        if (SUMS && live) {
          dbeta[k][e] += d[e];
          dgamma[k][e] = __fmaf_rn(d[e], n[e], dgamma[k][e]);
        }
      }
    }
    team_sum<L>(s, red, turn);
    if (!live) continue;
    const float s0 = RMS ? 0.0f : s[0] / count, s1 = s[1] / count;
    GWS_GLOBAL uint16_t* dx = global_ptr<uint16_t>(a.y) + at * a.ldy;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float n[8], d[8], o[8], r[8];
      widen(xr[k], n);
      widen(yr[k], d);
      if (a.r != nullptr) widen(rr[k], r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[e] = normal(n[e]);
        o[e] = __fmaf_rn(-n[e], s1, __fmaf_rn(d[e], gamma[k][e], -s0)) * rstd;
        if (a.r != nullptr) o[e] += r[e];
      }
      store_eight(dx, (lane + k * L) * 8, a.C, narrow(o));
    }
  }
}

// Many rows: a workgroup's sums of its rows go to a.part, and a second kernel adds those up.
template <int L, int V, int R, bool RMS>
__global__ __launch_bounds__(L * R) void norm_bwd_kernel(const NormArgs a) {
  __shared__ float red[4 * L * R / 64];
  constexpr int TEAMS = L < 64 ? L * R / 64 : R;
  __shared__ float sums[TEAMS == 1 ? 1 : TEAMS * L * V * 8];
  const uint32_t team = threadIdx.x / L, lane = threadIdx.x % L;
  float dgamma[V][8], dbeta[V][8];
#pragma unroll
  for (int k = 0; k < V; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) dgamma[k][e] = dbeta[k][e] = 0.0f;
  bwd_rows<L, V, R, RMS, true>(a, blockIdx.x * R, gridDim.x * R, dgamma, dbeta, red);
  // the workgroup's sums: rows that share a wavefront by lanes, then its TEAMS of a wavefront or more in turn
  float* part = a.part + (size_t)blockIdx.x * ((a.want_gamma ? 1 : 0) + (a.want_beta ? 1 : 0)) * a.C;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which == 0 ? !a.want_gamma : !a.want_beta) continue;
    float(&mine)[V][8] = which == 0 ? dgamma : dbeta;
    if (L < 64)
#pragma unroll
      for (int n = 0; n < 8 * V; ++n) {
        float& m = mine[n / 8][n % 8];
        uint32_t v = __float_as_uint(m);
        if (L == 16) {
          const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
          v = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
        }
        const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        m = __uint_as_float(q[0]) + __uint_as_float(q[1]);
      }
    if (TEAMS > 1) {
      __syncthreads();
      if (L >= 64 || (threadIdx.x & 63) < L) {
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            *(f4*)(sums + (L < 64 ? threadIdx.x / 64 : team) * (L * V * 8) + (lane + k * L) * 8 + e) = f4{mine[k][e], mine[k][e + 1], mine[k][e + 2], mine[k][e + 3]};
      }
      __syncthreads();
      for (uint32_t c = threadIdx.x; c < a.C; c += L * R) {
        float s = sums[c];
#pragma unroll
        for (int t = 1; t < TEAMS; ++t) s += sums[t * (L * V * 8) + c];
        part[c] = s;
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t c = (lane + k * L) * 8 + e;
          if (c < a.C) part[c] = mine[k][e];
        }
    }
    part += a.C;
  }
}

// Few elements: one launch.  Its first workgroups add up dgamma and dbeta of 32 columns each over all rows (mean and rstd are given, so nothing has to wait for
// the rows' sums), the others make dX.  X and dY are read twice, out of a cache, where a second launch takes longer than that.
constexpr uint32_t kPairCols = 32, kPairThreads = 512;
template <int L, int V, bool RMS>
__global__ __launch_bounds__(kPairThreads) void norm_bwd_pair_kernel(const NormArgs a, const uint32_t column_wgs, float* out_gamma, float* out_beta) {
  constexpr int R = kPairThreads / L;
  __shared__ float red[2 * 8 * 32];   // more than the 4 x 8 of the rows' sums
  if (blockIdx.x >= column_wgs) {
    float none[V][8];
    bwd_rows<L, V, R, RMS, false>(a, (blockIdx.x - column_wgs) * R, (gridDim.x - column_wgs) * R, none, none, red);
    return;
  }
  // four lanes with eight columns each, 128 rows at a time
  const uint32_t c = blockIdx.x * kPairCols + (threadIdx.x & 3) * 8;
  float dgamma[8], dbeta[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dgamma[e] = dbeta[e] = 0.0f;
#pragma unroll 4
  for (uint32_t row = threadIdx.x >> 2; row < a.M; row += kPairThreads / 4) {
    float n[8], d[8];
    widen(load_eight(global_ptr<uint16_t>(a.x) + (size_t)row * a.ldx, c, a.C), n);
    widen(load_eight(global_ptr<uint16_t>(a.dy) + (size_t)row * a.lddy, c, a.C), d);
    const Normalise normal(RMS ? 0.0f : a.mean[row], a.rstd[row]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dbeta[e] += d[e];
      dgamma[e] = __fmaf_rn(d[e], normal(n[e]), dgamma[e]);
    }
  }
  // the sixteen lanes of a wavefront with the same columns, then the wavefronts
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float* const v[2] = {&dgamma[e], &dbeta[e]};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float s = *v[k];
      s += __uint_as_float(dpp_u32<0x124>(__float_as_uint(s)));   // row_ror 4 and 8: lanes l, l + 4, l + 8, l + 12 of sixteen
      s += __uint_as_float(dpp_u32<0x128>(__float_as_uint(s)));
      const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
      s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
      const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
      *v[k] = __uint_as_float(q[0]) + __uint_as_float(q[1]);
    }
  }
  const uint32_t wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < 4)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      red[wave * 32 + (threadIdx.x & 3) * 8 + e] = dgamma[e];
      red[256 + wave * 32 + (threadIdx.x & 3) * 8 + e] = dbeta[e];
    }
  __syncthreads();
  const uint32_t col = blockIdx.x * kPairCols + (threadIdx.x & 31), which = threadIdx.x >> 5;
  float* out = which == 0 ? out_gamma : out_beta;
  if (which < 2 && out != nullptr && col < a.C) {
    float s = red[256 * which + (threadIdx.x & 31)];
#pragma unroll
    for (int w = 1; w < 8; ++w) s += red[256 * which + 32 * w + (threadIdx.x & 31)];
    out[col] = s;
  }
}

// Rows of any length, in two steps: sum(t) / C and sum(t n) / C of every row; then dX by pieces of 2048 columns, with dgamma and dbeta of them.
template <bool RMS>
__global__ __launch_bounds__(1024) void norm_bwd_rows_kernel(const NormArgs a) {
  __shared__ float red[4 * 16];
  uint32_t turn = 0;
  const uint32_t row = workgroup();
  if (row >= a.M) return;
  const GWS_GLOBAL uint16_t *x = global_ptr<uint16_t>(a.x) + (size_t)row * a.ldx, *dy = global_ptr<uint16_t>(a.dy) + (size_t)row * a.lddy;
  const Normalise normal(RMS ? 0.0f : a.mean[row], a.rstd[row]);
  float s[2] = {0.0f, 0.0f};
  for (uint32_t c = threadIdx.x * 8; c < a.C; c += 8192) {
    float n[8], d[8], gamma[8], s0 = 0.0f, s1 = 0.0f;
    widen(load_eight(x, c, a.C), n);
    widen(load_eight(dy, c, a.C), d);
    vector_eight(a.gamma, c, a.C, 1.0f, gamma);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = d[e] * gamma[e];
      s0 += t;
      s1 = __fmaf_rn(t, normal(n[e]), s1);
    }
    s[0] += s0;
    s[1] += s1;
  }
  team_sum<1024>(s, red, turn);
  if (threadIdx.x == 0) {
    a.rows[2 * (size_t)row] = RMS ? 0.0f : s[0] / (float)a.C;
    a.rows[2 * (size_t)row + 1] = s[1] / (float)a.C;
  }
}

template <bool RMS>
__global__ __launch_bounds__(256) void norm_bwd_columns_kernel(const NormArgs a) {
  const uint32_t c = (blockIdx.x * 256 + threadIdx.x) * 8;
  float gamma[8], dgamma[8], dbeta[8];
  vector_eight(a.gamma, c, a.C, 1.0f, gamma);
#pragma unroll
  for (int e = 0; e < 8; ++e) dgamma[e] = dbeta[e] = 0.0f;
  for (uint32_t row = blockIdx.y; row < a.M; row += gridDim.y) {
    float n[8], d[8], o[8], r[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    widen(load_eight(global_ptr<uint16_t>(a.x) + (size_t)row * a.ldx, c, a.C), n);
    widen(load_eight(global_ptr<uint16_t>(a.dy) + (size_t)row * a.lddy, c, a.C), d);
    if (a.r != nullptr) widen(load_eight(global_ptr<uint16_t>(a.r) + (size_t)row * a.ldr, c, a.C), r);
    const float rstd = a.rstd[row];
    const Normalise normal(RMS ? 0.0f : a.mean[row], rstd);
    const float s0 = a.rows[2 * (size_t)row], s1 = a.rows[2 * (size_t)row + 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      n[e] = normal(n[e]);
      dbeta[e] += d[e];
      dgamma[e] = __fmaf_rn(d[e], n[e], dgamma[e]);
      o[e] = __fmaf_rn(-n[e], s1, __fmaf_rn(d[e], gamma[e], -s0)) * rstd;
      if (a.r != nullptr) o[e] += r[e];
    }
    store_eight(global_ptr<uint16_t>(a.y) + (size_t)row * a.ldy, c, a.C, narrow(o));
  }
  float* part = a.part + (size_t)blockIdx.y * ((a.want_gamma ? 1 : 0) + (a.want_beta ? 1 : 0)) * a.C;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (c + e >= a.C) break;
    if (a.want_gamma) part[c + e] = dgamma[e];
    if (a.want_beta) part[(a.want_gamma ? a.C : 0) + c + e] = dbeta[e];
  }
}

// ---- sums of partial sums ----
// A workgroup adds 32 columns, 8 lanes x 4 of them side by side and the P rows shared by 32 groups of lanes, eight loads of each on their way at once; the groups'
// sums meet in LDS.  Bound by that latency: 256 rows of 1536 columns 2.0 us (64 columns by 16 groups, one load after the other, 6.3), of 4096 4.0.
__global__ __launch_bounds__(256) void sum_partials_kernel(const float* part, const uint32_t P, const uint64_t n, const uint64_t n0, float* out0, float* out1) {
  __shared__ f4 red[32][8];
  const uint32_t group = threadIdx.x >> 3, at = threadIdx.x & 7;
  const uint64_t c = (uint64_t)workgroup() * 32 + 4 * at;
  f4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t p0 = group; p0 < P; p0 += 256) {
    f4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t p = p0 + 32 * k;
      const GWS_GLOBAL float* q = global_ptr<float>(part) + (p < P ? p : p0) * n + c;
      v[k] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if (c + 4 <= n) {
        v[k] = *(const GWS_GLOBAL f4_any*)q;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (c + e < n) v[k][e] = q[e];
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (p0 + 32 * k < P) s += v[k];
  }
  red[group][at] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const float* r = (const float*)red;
  float t = r[threadIdx.x];
#pragma unroll
  for (int g = 1; g < 32; ++g) t += r[32 * g + threadIdx.x];
  const uint64_t col = (uint64_t)workgroup() * 32 + threadIdx.x;
  if (col < n0) out0[col] = t;
  else if (col < n) out1[col - n0] = t;
}

int launch_sum_partials(const float* part, uint32_t P, uint64_t n, uint64_t n0, float* out0, float* out1, hipStream_t stream) {
  hipLaunchKernelGGL(sum_partials_kernel, grid_of((n + 31) / 32), dim3(256), 0, stream, part, P, n, n0, out0, out1);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

__global__ __launch_bounds__(256) void zero_kernel(float* p, const uint64_t n) {
  const uint64_t i = (uint64_t)workgroup() * 256 + threadIdx.x;
  if (i < n) p[i] = 0.0f;
}
int launch_zero(float* p, uint64_t n, hipStream_t stream) {
  hipLaunchKernelGGL(zero_kernel, grid_of((n + 255) / 256), dim3(256), 0, stream, p, n);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

// ---- launches ----
constexpr uint64_t kWide = 16384;
bool norm_is_wide(uint64_t C) { return C > kWide; }

namespace {
uint32_t cus() { return compute_units() > 0 ? (uint32_t)compute_units() : 256; }
uint32_t fewer(uint64_t a, uint64_t b) { return (uint32_t)(a < b ? a : b); }

template <int L, int V, int R>
int fwd(const NormArgs& a, bool rms, hipStream_t s) {
  const dim3 grid(fewer(((uint64_t)a.M + R - 1) / R, 8 * cus())), block(L * R);
  if (rms) hipLaunchKernelGGL((norm_fwd_kernel<L, V, R, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_fwd_kernel<L, V, R, false>), grid, block, 0, s, a);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}
template <int L, int V, int R>
int bwd(const NormArgs& a, bool rms, hipStream_t s) {
  const dim3 grid(norm_bwd_parts(a.M, a.C)), block(L * R);
  if (rms) hipLaunchKernelGGL((norm_bwd_kernel<L, V, R, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_bwd_kernel<L, V, R, false>), grid, block, 0, s, a);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}
// Rows a workgroup of the backward kernels takes at a time.
uint32_t bwd_rows_of(uint64_t C) { return C <= 128 ? 64 : C <= 256 ? 32 : C <= 768 ? 16 : C <= 1024 ? 12 : C <= 2048 ? 8 : C <= 8192 ? 2 : 1; }

template <int L, int V>
int pair(const NormArgs& a, bool rms, float* dgamma, float* dbeta, hipStream_t s) {
  constexpr uint32_t R = kPairThreads / L;
  const uint32_t columns = (a.C + kPairCols - 1) / kPairCols;
  const dim3 grid(columns + fewer(((uint64_t)a.M + R - 1) / R, 2 * cus())), block(kPairThreads);
  if (rms) hipLaunchKernelGGL((norm_bwd_pair_kernel<L, V, true>), grid, block, 0, s, a, columns, dgamma, dbeta);
  else hipLaunchKernelGGL((norm_bwd_pair_kernel<L, V, false>), grid, block, 0, s, a, columns, dgamma, dbeta);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}
// Whether one launch that reads twice beats two.  us of one and two in a graph (the host takes 3 more for a second launch): 512 x 768 3.9, 7.9; 1024 x 768 6.4, 8.2;
// 1280 x 768 7.8, 8.7; 2048 x 768 11.2, 9.4; 1024 x 2048 8.8, 10.9; 2048 x 2048 15.0, 13.5; 1280 x 4096 14.7, 16.0; 1024 x 6144 18.7, 19.1; 768 x 8192 20.0, 20.3; 1536 x 8192 34.8, 31.1; 256 x 16384
// 14.8, 35.4; 1536 x 16384 66.1, 69.4; 3000 x 16384 125, 105: with rows that long two launches write and read as much of partial sums as of X.
bool one_launch(uint64_t M, uint64_t C) {
  return !norm_is_wide(C) && M <= (C > 8192 ? 1536u : C > 6144 ? 768u : C > 4096 ? 1024u : 1280u);
}
}  // namespace

int launch_norm_fwd(const NormArgs& a, bool rms, hipStream_t s) {
  if (norm_is_wide(a.C)) {
    if (rms) hipLaunchKernelGGL(norm_fwd_wide_kernel<true>, grid_of(a.M), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL(norm_fwd_wide_kernel<false>, grid_of(a.M), dim3(1024), 0, s, a);
    return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
  }
  if (a.C <= 128) return fwd<16, 1, 16>(a, rms, s);
  if (a.C <= 256) return fwd<32, 1, 8>(a, rms, s);
  if (a.C <= 512) return fwd<64, 1, 4>(a, rms, s);
  if (a.C <= 768) return fwd<32, 3, 8>(a, rms, s);
  if (a.C <= 1024) return fwd<64, 2, 4>(a, rms, s);
  if (a.C <= 1536) return fwd<64, 3, 4>(a, rms, s);
  if (a.C <= 2048) return fwd<64, 4, 4>(a, rms, s);
  if (a.C <= 4096) return fwd<256, 2, 1>(a, rms, s);
  if (a.C <= 6144) return fwd<256, 3, 1>(a, rms, s);
  if (a.C <= 8192) return fwd<256, 4, 1>(a, rms, s);
  return fwd<512, 4, 1>(a, rms, s);
}

uint32_t norm_bwd_parts(uint64_t M, uint64_t C) {
  // Of long rows: parts enough for a workgroup a compute unit (64 x 32768 16 parts of four rows, few rows one each), more only where each keeps eight rows and more,
  // whose partial sums are then at most a quarter of what it reads, and no more than 64.  us with 8, 16, 32, 64 parts: 64 x 32768
  // 19.3, 18.1, 20.2, 26.1; 64 x 131072 38, 43, 81, 139; 300 x 20000 60, 39, 31, 29; 1000 x 32768 154,
  // 112, 92, 88, with 125 117.
  if (norm_is_wide(C)) {
    const uint64_t pieces = (C + 2047) / 2048, filled = (cus() + pieces - 1) / pieces;
    return fewer(M, fewer(std::max(filled, M / 8), 64));
  }
  return fewer((M + bwd_rows_of(C) - 1) / bwd_rows_of(C), cus());
}

int launch_norm_bwd(const NormArgs& a, bool rms, float* dgamma, float* dbeta, hipStream_t s) {
  int rc;
  if ((a.want_gamma || a.want_beta) && one_launch(a.M, a.C) && a.y != a.x && a.y != a.dy) {   // in place the rows would change what the columns read
    if (a.C <= 128) return pair<16, 1>(a, rms, dgamma, dbeta, s);
    if (a.C <= 256) return pair<32, 1>(a, rms, dgamma, dbeta, s);
    if (a.C <= 512) return pair<64, 1>(a, rms, dgamma, dbeta, s);
    if (a.C <= 768) return pair<32, 3>(a, rms, dgamma, dbeta, s);
    if (a.C <= 1024) return pair<64, 2>(a, rms, dgamma, dbeta, s);
    if (a.C <= 1536) return pair<64, 3>(a, rms, dgamma, dbeta, s);
    if (a.C <= 2048) return pair<64, 4>(a, rms, dgamma, dbeta, s);
    if (a.C <= 4096) return pair<256, 2>(a, rms, dgamma, dbeta, s);
    if (a.C <= 6144) return pair<256, 3>(a, rms, dgamma, dbeta, s);
    if (a.C <= 8192) return pair<256, 4>(a, rms, dgamma, dbeta, s);
    return pair<512, 4>(a, rms, dgamma, dbeta, s);
  }
  if (norm_is_wide(a.C)) {
    const dim3 pieces((uint32_t)(((uint64_t)a.C + 2047) / 2048), norm_bwd_parts(a.M, a.C));
    if (rms) {
      hipLaunchKernelGGL(norm_bwd_rows_kernel<true>, grid_of(a.M), dim3(1024), 0, s, a);
      hipLaunchKernelGGL(norm_bwd_columns_kernel<true>, pieces, dim3(256), 0, s, a);
    } else {
      hipLaunchKernelGGL(norm_bwd_rows_kernel<false>, grid_of(a.M), dim3(1024), 0, s, a);
      hipLaunchKernelGGL(norm_bwd_columns_kernel<false>, pieces, dim3(256), 0, s, a);
    }
    rc = hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
  } else if (a.C <= 128) rc = bwd<16, 1, 64>(a, rms, s);
  else if (a.C <= 256) rc = bwd<32, 1, 32>(a, rms, s);
  else if (a.C <= 512) rc = bwd<64, 1, 16>(a, rms, s);
  else if (a.C <= 768) rc = bwd<32, 3, 16>(a, rms, s);
  else if (a.C <= 1024) rc = bwd<64, 2, 12>(a, rms, s);
  else if (a.C <= 1536) rc = bwd<64, 3, 8>(a, rms, s);
  else if (a.C <= 2048) rc = bwd<64, 4, 8>(a, rms, s);
  else if (a.C <= 4096) rc = bwd<256, 2, 2>(a, rms, s);
  else if (a.C <= 6144) rc = bwd<256, 3, 2>(a, rms, s);
  else if (a.C <= 8192) rc = bwd<256, 4, 2>(a, rms, s);
  else rc = bwd<512, 4, 1>(a, rms, s);
  if (rc != GWS_OK || (!a.want_gamma && !a.want_beta)) return rc;
  const uint64_t n = a.want_gamma && a.want_beta ? 2 * (uint64_t)a.C : a.C;
  return launch_sum_partials(a.part, norm_bwd_parts(a.M, a.C), n, a.C, a.want_gamma ? dgamma : dbeta, dbeta, s);
}

}  // namespace gws
