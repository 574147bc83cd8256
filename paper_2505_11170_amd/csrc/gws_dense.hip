// The dense layer for any sizes (gfx950): the products of gws_dense_fwd and gws_dense_bwd by one small tile that reads its operands straight into the
// MFMA's registers, and gws_dense_bwd_h, a pass over memory.  The small tile is right for every size that the entry points take and there for
// those that the other kernels do not take (K = 32, very large leading dimensions).  Bound by its operands' latency (8192 x 2048 -> 5632 1550 us, ten times the large
// tiles).
#include "gws_dense.h"
#include "gws_gemm256_core.h"

namespace gws {

namespace {
constexpr uint32_t kRows = kDenseAnyRows, kCols = 64;   // of a workgroup: 4 wavefronts x 16 rows, four MFMA tiles of columns

// 8 consecutive k of row `row`
__device__ __forceinline__ Frag8 along(const uint16_t* p, uint32_t row, uint32_t ld, uint32_t k) {
  Frag8 f;
  f.u = *(const u32x4*)(p + (size_t)row * ld + k);
  return f;
}
// 8 consecutive k of column `col`
__device__ __forceinline__ Frag8 across(const uint16_t* p, uint32_t col, uint32_t ld, uint32_t k) {
  Frag8 f;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    f.u[e] = (uint32_t)p[(size_t)(k + 2 * e) * ld + col] | (uint32_t)p[(size_t)(k + 2 * e + 1) * ld + col] << 16;
  return f;
}
__device__ __forceinline__ u32x2 pack4(const float (&v)[4]) { return u32x2{pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3])}; }
__device__ __forceinline__ void four_of(const uint16_t* p, float (&v)[4]) {
  const u32x2 w = *(const u32x2*)p;
  v[0] = lo_of(w[0]); v[1] = hi_of(w[0]); v[2] = lo_of(w[1]); v[3] = hi_of(w[1]);
}
}  // namespace

// A lane's sums: row lane % 16 of its wavefront's 16, columns 16 j + 4 (lane / 16) .. + 3.
template <DenseOp OP, bool W_NK>
__global__ __launch_bounds__(256) void dense_any_kernel(const GemmArgs g, const DenseArgs d) {
  __shared__ float sums[4][kCols];
  const uint32_t lane = threadIdx.x & 63, li = lane & 15, grp = lane >> 4, wave = threadIdx.x >> 6;
  const uint32_t nt = (g.N + kCols - 1) / kCols, tile = workgroup(), tile_m = tile / nt, m0 = tile_m * kRows + 16 * wave, n0 = tile % nt * kCols;
  if (tile_m >= (g.M + kRows - 1) / kRows) return;   // uniform: past the last tile of a grid of two dimensions
  const bool live = m0 + li < g.M;
  const uint32_t row = live ? m0 + li : g.M - 1;   // past the edge the last ones are read, and nothing is stored
  uint32_t col[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) col[j] = n0 + 16 * j + li < g.N ? n0 + 16 * j + li : g.N - 1;
  f32x4 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t k = 8 * grp; k < g.K; k += 32) {
    const Frag8 fa = along(g.x, row, g.ldx, k);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Frag8 fb = W_NK ? along(g.w, col[j], g.ldw, k) : across(g.w, col[j], g.ldw, k);
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.v, fa.v, acc[j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t c = n0 + 16 * j + 4 * grp;
    const bool here = live && c < g.N;   // N is a multiple of 32: four columns exist or do not
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f}, o[4];
    if (here) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[j][e];
      if (OP == DenseOp::kFwd) {
        if (d.bias != nullptr)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += d.bias[c + e];
        if (d.z != nullptr) *(u32x2*)(d.z + (size_t)row * d.ldz + c) = pack4(v);
        with_act(d.act, [&](auto gate) {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = gate.a(v[e]);
        });
        if (d.r != nullptr) {
          float r[4];
          four_of(d.r + (size_t)row * d.ldr + c, r);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += r[e];
        }
        *(u32x2*)(g.y + (size_t)row * g.ldy + c) = pack4(o);
      } else {
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f}, h[4];
        if (d.z != nullptr) four_of(d.z + (size_t)row * d.ldz + c, z);
        with_act(d.act, [&](auto gate) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float slope;
            gate.both(z[e], h[e], slope);
            v[e] *= slope;
          }
        });
        *(u32x2*)(g.y + (size_t)row * g.ldy + c) = pack4(v);
        if (d.h != nullptr) *(u32x2*)(d.h + (size_t)row * d.ldh + c) = pack4(h);
      }
    }
    if (OP == DenseOp::kBwd && d.part != nullptr) {   // uniform
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // over the 16 rows of the wavefront
        float s = v[e];
        s += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(s)));
        s += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(s)));
        s += __uint_as_float(dpp_u32<0x141>(__float_as_uint(s)));
        s += __uint_as_float(dpp_u32<0x140>(__float_as_uint(s)));
        if (li == 0) sums[wave][16 * j + 4 * grp + e] = s;
      }
    }
  }
  if (OP == DenseOp::kBwd && d.part != nullptr) {
    __syncthreads();
    const uint32_t c = threadIdx.x;
    if (c < kCols && n0 + c < g.N) d.part[(size_t)tile_m * g.N + n0 + c] = ((sums[0][c] + sums[1][c]) + sums[2][c]) + sums[3][c];
  }
}

int launch_dense_any(const GemmArgs& g, const DenseArgs& e, DenseOp op, int w_is_nk, hipStream_t stream) {
  const uint64_t tiles = (((uint64_t)g.M + kRows - 1) / kRows) * (((uint64_t)g.N + kCols - 1) / kCols);
  if (tiles >= (uint64_t)1 << 31) return GWS_ERR_SHAPE;   // results of 8 TB and more
  const dim3 grid = grid_of(tiles), block(256);
  if (op == DenseOp::kFwd) {
    if (w_is_nk) hipLaunchKernelGGL((dense_any_kernel<DenseOp::kFwd, true>), grid, block, 0, stream, g, e);
    else hipLaunchKernelGGL((dense_any_kernel<DenseOp::kFwd, false>), grid, block, 0, stream, g, e);
  } else {
    if (w_is_nk) hipLaunchKernelGGL((dense_any_kernel<DenseOp::kBwd, true>), grid, block, 0, stream, g, e);
    else hipLaunchKernelGGL((dense_any_kernel<DenseOp::kBwd, false>), grid, block, 0, stream, g, e);
  }
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

// ---- the activation's backward pass from a given dL/dH ----
// A workgroup takes 256 columns, eight a lane, and `rows` rows, eight at a time; the eight rows' sums of a column meet in LDS.  Bound by memory: 8192 x 5632 with H 77 us
// (4.8 TB/s).  Its stores are ordinary ones: past the caches the call takes 74, but it and the products that read dZ and H 1 to 6 % more (4096 tokens 325 and 317 us).
__global__ __launch_bounds__(256) void dense_bwd_h_kernel(const GemmArgs g, const DenseArgs d, const uint32_t rows) {
  __shared__ float sums[8][256];
  const uint32_t lane = threadIdx.x & 31, first = threadIdx.x >> 5, c = blockIdx.x * 256 + 8 * lane;
  const uint32_t end = g.M - blockIdx.y * rows < rows ? g.M : (blockIdx.y + 1) * rows;
  float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < g.N) {   // N is a multiple of 8
    with_act(d.act, [&](auto gate) {
#pragma unroll 2
      for (uint32_t row = blockIdx.y * rows + first; row < end; row += 8) {
        float v[8], z[8] = {0, 0, 0, 0, 0, 0, 0, 0}, h[8];
        widen(*(const u32x4*)(g.x + (size_t)row * g.ldx + c), v);
        if (d.z != nullptr) widen(*(const u32x4*)(d.z + (size_t)row * d.ldz + c), z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float slope;
          gate.both(z[e], h[e], slope);
          v[e] *= slope;
          total[e] += v[e];
        }
        if (g.y != nullptr) *(u32x4*)(g.y + (size_t)row * g.ldy + c) = narrow(v);
        if (d.h != nullptr) *(u32x4*)(d.h + (size_t)row * d.ldh + c) = narrow(h);
      }
    });
  }
  if (d.part == nullptr) return;   // uniform
#pragma unroll
  for (int e = 0; e < 8; e += 4) *(f4*)&sums[first][8 * lane + e] = f4{total[e], total[e + 1], total[e + 2], total[e + 3]};
  __syncthreads();
  float s = sums[0][threadIdx.x];
#pragma unroll
  for (int k = 1; k < 8; ++k) s += sums[k][threadIdx.x];
  const uint32_t col = blockIdx.x * 256 + threadIdx.x;
  if (col < g.N) d.part[(size_t)blockIdx.y * g.N + col] = s;
}

// 32, or 16 where that leaves less than four workgroups a compute unit.  8192 x 5632 GELU with H and the bias gradient, 32, 64, 128, 256 rows: 77.1, 79.6, 83.9, 83.7 us.
uint32_t dense_h_rows(uint64_t M, uint64_t F) {
  const uint64_t cus = compute_units() > 0 ? compute_units() : 256, columns = (F + 255) / 256;
  uint64_t rows = 32;
  while (rows > 16 && columns * ((M + rows - 1) / rows) < 4 * cus) rows /= 2;
  while ((M + rows - 1) / rows > 65535) rows *= 2;   // of a grid
  return (uint32_t)rows;
}

int launch_dense_bwd_h(const GemmArgs& g, const DenseArgs& e, hipStream_t stream) {
  const uint32_t rows = dense_h_rows(g.M, g.N);
  const dim3 grid((uint32_t)(((uint64_t)g.N + 255) / 256), (uint32_t)(((uint64_t)g.M + rows - 1) / rows));
  hipLaunchKernelGGL(dense_bwd_h_kernel, grid, dim3(256), 0, stream, g, e, rows);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

}  // namespace gws
