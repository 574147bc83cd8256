// The gated feed-forward block for any sizes (gfx950): the products of gws_gated_fwd, gws_gated_bwd and gws_gated_bwd_x by one
// small tile that reads its operands straight into the MFMA's registers.  Right for every size the entry points take, and there for
// those that the other kernels do not take (K = 32, leading dimensions of 2^24 elements and more, of results 2^28).  Bound by those reads, 16 rows of 64 bytes
// an instruction: 1021 x 768 -> 2048 forward 84 us (11.2 in 128 x 128 tiles).
#include "gws_gated.h"
#include "gws_gemm256_core.h"

namespace gws {

namespace {
constexpr uint32_t kRows = 64, kCols = 64;   // of a workgroup: 4 wavefronts x 16 rows, four MFMA tiles of columns

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
}  // namespace

// A lane's sums: row lane % 16 of its wavefront's 16, columns 16 j + 4 (lane / 16) .. + 3.
template <GatedOp OP, bool B_OC, Kept KEPT>
__global__ __launch_bounds__(256) void gated_any_kernel(const GatedArgs g) {
  const uint32_t lane = threadIdx.x & 63, li = lane & 15, grp = lane >> 4, wave = threadIdx.x >> 6;
  const uint32_t nt = (g.N + kCols - 1) / kCols, m0 = blockIdx.x / nt * kRows + 16 * wave, n0 = blockIdx.x % nt * kCols;
  const uint32_t row = m0 + li < g.M ? m0 + li : g.M - 1;   // past the edge the last ones are read, and nothing is stored
  uint32_t col[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) col[j] = n0 + 16 * j + li < g.N ? n0 + 16 * j + li : g.N - 1;
  constexpr int P = OP == GatedOp::kFwd ? 2 : 1;            // products side by side
  f32x4 acc[P][4];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[p][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int part = 0; part < (OP == GatedOp::kDx ? 2 : 1); ++part) {
    const uint16_t* a = part == 0 ? g.a : g.a2;
    for (uint32_t k = 8 * grp; k < g.K; k += 32) {
      const Frag8 fa = along(a, row, g.lda, k);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const uint16_t* b = p + part == 0 ? g.b : g.b2;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Frag8 fb = B_OC ? across(b, col[j], g.ldb, k) : along(b, col[j], g.ldb, k);
          acc[p][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.v, fa.v, acc[p][j], 0, 0, 0);
        }
      }
    }
  }
  const bool live = m0 + li < g.M;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t c = n0 + 16 * j + 4 * grp;
    const bool here = live && c < g.N;   // N is a multiple of 32: four columns exist or do not
    if (OP == GatedOp::kDx) {
      if (here) *(u32x2*)(g.h + (size_t)row * g.ldh + c) = u32x2{pack_bf16_rne(acc[0][j][0], acc[0][j][1]), pack_bf16_rne(acc[0][j][2], acc[0][j][3])};
    } else if (OP == GatedOp::kFwd) {
      float h[4], v[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[0][e] = acc[0][j][e];
        v[1][e] = acc[P - 1][j][e];
        h[e] = v[1][e];
      }
      with_gate(g.act, [&](auto gate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] *= gate.a(v[0][e]);
      });
      if (here) *(u32x2*)(g.h + (size_t)row * g.ldh + c) = u32x2{pack_bf16_rne(h[0], h[1]), pack_bf16_rne(h[2], h[3])};
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint8_t* to = p == 0 ? g.kept.g : g.kept.u;
        const uint32_t ld = p == 0 ? g.kept.ldg : g.kept.ldu;
        if (KEPT == Kept::kBf16 && here) *(u32x2*)(to + ((size_t)row * ld + c) * 2) = u32x2{pack_bf16_rne(v[p][0], v[p][1]), pack_bf16_rne(v[p][2], v[p][3])};
        if (KEPT == Kept::kE4m3) {
          // a block of 32 columns: MFMA tiles 2 (j / 2) and the next, the four lanes lane % 16 + 16 x
          float top = 0.0f;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const f32x4& s = acc[p == 0 ? 0 : P - 1][(j & 2) + (t >> 1)];
            top = act8_larger(top, s[2 * (t & 1)], s[2 * (t & 1) + 1]);
          }
          uint32_t m = __float_as_uint(top) & 0x7FFFFFFFu;
          m = max(m, (uint32_t)__shfl_xor((int)m, 16));
          m = max(m, (uint32_t)__shfl_xor((int)m, 32));
          const uint32_t byte = act8_byte(m);
          if (byte == kAct8Max) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[p][e] = act8_clamp(v[p][e]);
          }
          if (here) *(uint32_t*)(to + (size_t)row * ld + c) = act8_codes(v[p], byte);
          if (here && grp == 0 && (j & 1) == 0) (p == 0 ? g.kept.gs : g.kept.us)[(size_t)row * (p == 0 ? g.kept.lsg : g.kept.lsu) + (c >> 5)] = (uint8_t)byte;
        }
      }
    } else if (here) {
      float vg[4], vu[4], h[4], dg[4], du[4];
      KeptFours<KEPT> kept;
      kept.load(g.kept, row, c);
      kept.g.values(vg);
      kept.u.values(vu);
      with_gate(g.act, [&](auto gate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float a, slope;
          gate.both(vg[e], a, slope);
          h[e] = a * vu[e];
          du[e] = acc[0][j][e] * a;
          dg[e] = acc[0][j][e] * vu[e] * slope;
        }
      });
      *(u32x2*)(g.dg + (size_t)row * g.ldd + c) = u32x2{pack_bf16_rne(dg[0], dg[1]), pack_bf16_rne(dg[2], dg[3])};
      *(u32x2*)(g.du + (size_t)row * g.ldd + c) = u32x2{pack_bf16_rne(du[0], du[1]), pack_bf16_rne(du[2], du[3])};
      if (g.h != nullptr) *(u32x2*)(g.h + (size_t)row * g.ldh + c) = u32x2{pack_bf16_rne(h[0], h[1]), pack_bf16_rne(h[2], h[3])};
    }
  }
}

template <GatedOp OP, Kept KEPT>
static int launch_any(const GatedArgs& g, bool b_oc, uint32_t tiles, hipStream_t stream) {
  if (b_oc) hipLaunchKernelGGL((gated_any_kernel<OP, true, KEPT>), dim3(tiles), dim3(256), 0, stream, g);
  else hipLaunchKernelGGL((gated_any_kernel<OP, false, KEPT>), dim3(tiles), dim3(256), 0, stream, g);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

int launch_gated_any(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream) {
  const uint64_t tiles = (uint64_t)((g.M + kRows - 1) / kRows) * ((g.N + kCols - 1) / kCols);
  if (tiles >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  const uint32_t n = (uint32_t)tiles;
  if (op == GatedOp::kDx) return launch_any<GatedOp::kDx, Kept::kNone>(g, b_oc, n, stream);
  if (op == GatedOp::kBwd)
    return kept == Kept::kE4m3 ? launch_any<GatedOp::kBwd, Kept::kE4m3>(g, b_oc, n, stream) : launch_any<GatedOp::kBwd, Kept::kBf16>(g, b_oc, n, stream);
  return kept == Kept::kE4m3 ? launch_any<GatedOp::kFwd, Kept::kE4m3>(g, b_oc, n, stream)
         : kept == Kept::kBf16 ? launch_any<GatedOp::kFwd, Kept::kBf16>(g, b_oc, n, stream) : launch_any<GatedOp::kFwd, Kept::kNone>(g, b_oc, n, stream);
}

// ---- the gate's backward pass from a given dL/dH: one pass over memory, eight columns a lane ----
// Bound by memory: 8192 x 5632 with H, kept in 8 bits 85 us (5.5 TB/s of 464 MB), as BF16 103 us (5.4 TB/s of 554 MB).
template <Kept KEPT>
__global__ __launch_bounds__(256) void gated_bwd_h_kernel(const GatedArgs g, const uint32_t per_row, const uint32_t inv) {
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t total = (uint64_t)g.M * per_row;
  if (id >= total) return;
  uint32_t row, c;
  if (total < 0x80000000ull) {   // uniform
    row = divide((uint32_t)id, per_row, inv);
    c = ((uint32_t)id - row * per_row) * 8;
  } else {
    row = (uint32_t)(id / per_row);
    c = (uint32_t)(id - (uint64_t)row * per_row) * 8;
  }
  const u32x4 d = *(const u32x4*)(g.a + (size_t)row * g.lda + c);
  float vg[2][4], vu[2][4];
  KeptFours<KEPT> kept[2];
  kept[0].load(g.kept, row, c);
  kept[1].load(g.kept, row, c + 4);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    kept[t].g.values(vg[t]);
    kept[t].u.values(vu[t]);
  }
  u32x4 odg, odu, oh;
  with_gate(g.act, [&](auto gate) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      float a[2], slope[2], u[2], dh[2] = {bf16_lo(d[p]), bf16_hi(d[p])};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        gate.both(vg[p >> 1][2 * (p & 1) + e], a[e], slope[e]);
        u[e] = vu[p >> 1][2 * (p & 1) + e];
      }
      odg[p] = pack_bf16_rne(dh[0] * u[0] * slope[0], dh[1] * u[1] * slope[1]);
      odu[p] = pack_bf16_rne(dh[0] * a[0], dh[1] * a[1]);
      oh[p] = pack_bf16_rne(a[0] * u[0], a[1] * u[1]);
    }
  });
  *(u32x4*)(g.dg + (size_t)row * g.ldd + c) = odg;
  *(u32x4*)(g.du + (size_t)row * g.ldd + c) = odu;
  if (g.h != nullptr) *(u32x4*)(g.h + (size_t)row * g.ldh + c) = oh;
}

int launch_gated_bwd_h(const GatedArgs& g, Kept kept, hipStream_t stream) {
  const uint32_t per_row = g.N / 8;
  const uint64_t wgs = ((uint64_t)g.M * per_row + 255) / 256;
  if (wgs >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  if (kept == Kept::kE4m3) hipLaunchKernelGGL(gated_bwd_h_kernel<Kept::kE4m3>, dim3((uint32_t)wgs), dim3(256), 0, stream, g, per_row, reciprocal(per_row));
  else hipLaunchKernelGGL(gated_bwd_h_kernel<Kept::kBf16>, dim3((uint32_t)wgs), dim3(256), 0, stream, g, per_row, reciprocal(per_row));
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

}  // namespace gws
