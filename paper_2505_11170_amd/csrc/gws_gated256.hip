// The products of the gated block in 256 x 256 tiles (gfx950): the loop of gws_gemm256_core.h with two weights side by side
// (forward), with two products in one sum (input gradient), or as it is (backward), and the gate on the way out.
//
// Forward: a wavefront holds the same 64 columns of G and of U for its 128 rows, so a lane has both halves of an element of H, and
// the four lanes of a block of 32 that is kept in 8 bits meet in two cross-lane steps.  Everything leaves through LDS by rows.
// Backward: dL/dH leaves the accumulators through LDS as fp32, 32 rows at a time, and meets the kept G and U, which were
// requested before, 8 columns of a row a lane.
#include "gws_gated.h"
#include "gws_gemm256_core.h"

namespace gws {

namespace {

// This wavefront's LDS writes have landed / its reads are done.
__device__ __forceinline__ void own_lds_wait() {
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  __builtin_amdgcn_wave_barrier();
}

constexpr int PH = 64 + 8;    // pitch of a staged row of 64 BF16 values (elements)
constexpr int PB = 64 + 16;   // of 64 codes (bytes)

// 64 staged rows of 64 BF16 values (of 64 codes) to rows of `ld` bytes at `to`; of them `rows` and, of the columns, `cols` exist
// (cols a multiple of 32).
template <int BYTES, bool EDGE>
__device__ __forceinline__ void rows_out(const uint8_t* cs, uint8_t* to, size_t ld, uint32_t lane, int rows, int cols) {
  constexpr int PITCH = BYTES == 2 ? PH * 2 : PB, LANES = 4 * BYTES, ROWS = 64 / LANES;   // lanes of a row, rows of an instruction
  const uint32_t r = lane / LANES, c = (lane % LANES) * 16;
  const bool col_in = !EDGE || (int)c < cols * BYTES;
#pragma unroll 4
  for (int it = 0; it < 64 / ROWS; ++it) {
    const uint32_t row = it * ROWS + r;
    if (!EDGE || ((int)row < rows && col_in)) *(u32x4*)(to + row * ld + c) = *(const u32x4*)(cs + row * PITCH + c);
  }
}

// H, and G and U as they are kept, of a wavefront's 128 rows x 64 columns from (p0, q0).
template <Kept KEPT, bool EDGE>
__device__ __forceinline__ void fwd_out(const GatedArgs& g, const f32x4 (&acc)[8][8], uint8_t* cs, uint32_t p0, uint32_t q0, uint32_t lane) {
  const uint32_t li = lane & 15, grp = lane >> 4;
  uint8_t* const hs = cs;                                    // 64 rows of H, then of G and of U
  uint8_t* const ks[2] = {cs + 64 * PH * 2, cs + 64 * PH * 2 + 64 * (KEPT == Kept::kE4m3 ? PB : PH * 2)};
  const int rows = (int)g.M - (int)p0, cols = (int)g.N - (int)q0;   // EDGE: what exists, may be <= 0
  // 8 bits: lane group 0, 1 stores the scales of G's two blocks, 2, 3 those of U's
  uint8_t* sp = nullptr;
  size_t ls = 0;
  if (KEPT == Kept::kE4m3) {
    ls = grp < 2 ? g.kept.lsg : g.kept.lsu;
    sp = (grp < 2 ? g.kept.gs : g.kept.us) + (size_t)(p0 + li) * ls + (q0 >> 5) + (grp & 1);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2) {
      const int i = 4 * h + i2;
      uint32_t byte[2][2] = {{0, 0}, {0, 0}};   // [G, U][block]
      if (KEPT == Kept::kE4m3) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            uint32_t m = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(acc[i][4 * p + 2 * b + t][e]) & 0x7FFFFFFFu);
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            byte[p][b] = act8_byte(m);
          }
        const uint32_t mine = grp & 2 ? (grp & 1 ? byte[1][1] : byte[1][0]) : (grp & 1 ? byte[0][1] : byte[0][0]);
        if (!EDGE || (16 * i + (int)li < rows && 32 * (int)(grp & 1) < cols)) sp[(size_t)(16 * i) * ls] = (uint8_t)mine;
      }
      const uint32_t row = 16 * i2 + li;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[2][4], o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[0][e] = acc[i][j][e];
          v[1][e] = acc[i][j + 4][e];
          o[e] = gate_a(g.gate, v[0][e]) * v[1][e];
        }
        *(u32x2*)(hs + row * PH * 2 + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3])};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (KEPT == Kept::kBf16)
            *(u32x2*)(ks[p] + row * PH * 2 + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(v[p][0], v[p][1]), pack_bf16_rne(v[p][2], v[p][3])};
          if (KEPT == Kept::kE4m3) *(uint32_t*)(ks[p] + row * PB + 16 * j + 4 * grp) = act8_codes(v[p], byte[p][j >> 1]);
        }
      }
    }
    own_lds_wait();
    const uint32_t r0 = p0 + 64 * h;
    rows_out<2, EDGE>(hs, (uint8_t*)(g.h + (size_t)r0 * g.ldh + q0), (size_t)g.ldh * 2, lane, rows - 64 * h, cols);
    if (KEPT == Kept::kBf16) {
      rows_out<2, EDGE>(ks[0], g.kept.g + ((size_t)r0 * g.kept.ldg + q0) * 2, (size_t)g.kept.ldg * 2, lane, rows - 64 * h, cols);
      rows_out<2, EDGE>(ks[1], g.kept.u + ((size_t)r0 * g.kept.ldu + q0) * 2, (size_t)g.kept.ldu * 2, lane, rows - 64 * h, cols);
    }
    if (KEPT == Kept::kE4m3) {
      rows_out<1, EDGE>(ks[0], g.kept.g + (size_t)r0 * g.kept.ldg + q0, g.kept.ldg, lane, rows - 64 * h, cols);
      rows_out<1, EDGE>(ks[1], g.kept.u + (size_t)r0 * g.kept.ldu + q0, g.kept.ldu, lane, rows - 64 * h, cols);
    }
    own_lds_wait();
  }
}

// Kept values of eight columns on their way, and as fp32 pairs.
template <Kept KEPT>
struct KeptEight {
  u32x4 w;          // BF16, or codes in the first two
  uint32_t byte;
  __device__ __forceinline__ void load(const uint8_t* p, const uint8_t* s, uint32_t ld, uint32_t ls, uint32_t row, uint32_t col) {
    if (KEPT == Kept::kBf16) {
      w = *(const u32x4*)(p + ((size_t)row * ld + col) * 2);
    } else {
      const u32x2 c = *(const u32x2*)(p + (size_t)row * ld + col);
      w = u32x4{c[0], c[1], 0, 0};
      byte = s[(size_t)row * ls + (col >> 5)];
    }
  }
  __device__ __forceinline__ uint32_t pair(int d) const {
    if (KEPT == Kept::kBf16) return w[d];
    return d & 1 ? act8_pair<true>(w[d >> 1], byte) : act8_pair<false>(w[d >> 1], byte);
  }
};

// dL/dG, dL/dU and H of a wavefront's 128 x 128 part from (p0, q0).
template <Kept KEPT, bool EDGE>
__device__ __forceinline__ void bwd_out(const GatedArgs& g, const f32x4 (&acc)[8][8], float* cs, uint32_t p0, uint32_t q0, uint32_t lane) {
  constexpr int PF = 128 + 4;   // pitch of a staged row of fp32 (32 of them)
  const uint32_t li = lane & 15, grp = lane >> 4;
  const uint32_t r = lane >> 4, c = (lane & 15) * 8;   // on the way out: row % 4, column
  const int rows = (int)g.M - (int)p0, cols = (int)g.N - (int)q0;
  const bool col_in = !EDGE || (int)c < cols;
  KeptEight<KEPT> vg[8], vu[8];
  auto request = [&](int quarter) {
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const uint32_t row = 32 * quarter + 4 * it + r;
      if (!EDGE || ((int)row < rows && col_in)) {
        vg[it].load(g.kept.g, g.kept.gs, g.kept.ldg, g.kept.lsg, p0 + row, q0 + c);
        vu[it].load(g.kept.u, g.kept.us, g.kept.ldu, g.kept.lsu, p0 + row, q0 + c);
      }
    }
  };
  request(0);
#pragma unroll
  for (int quarter = 0; quarter < 4; ++quarter) {
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
      for (int j = 0; j < 8; ++j) *(f32x4*)(cs + (16 * i2 + li) * PF + 16 * j + 4 * grp) = acc[2 * quarter + i2][j];
    own_lds_wait();
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const uint32_t row = 4 * it + r;
      const f32x4 d0 = *(const f32x4*)(cs + row * PF + c), d1 = *(const f32x4*)(cs + row * PF + c + 4);
      if (!EDGE || (32 * quarter + (int)row < rows && col_in)) {
        u32x4 odg, odu, oh;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const uint32_t pg = vg[it].pair(p), pu = vu[it].pair(p);
          const float u0 = bf16_lo(pu), u1 = bf16_hi(pu);
          const float h0 = p < 2 ? d0[2 * p] : d1[2 * p - 4], h1 = p < 2 ? d0[2 * p + 1] : d1[2 * p - 3];
          float a0, a1, s0, s1;
          gate_both(g.gate, bf16_lo(pg), a0, s0);
          gate_both(g.gate, bf16_hi(pg), a1, s1);
          odg[p] = pack_bf16_rne(h0 * u0 * s0, h1 * u1 * s1);
          odu[p] = pack_bf16_rne(h0 * a0, h1 * a1);
          oh[p] = pack_bf16_rne(a0 * u0, a1 * u1);
        }
        const size_t at = p0 + 32 * quarter + row;
        *(u32x4*)(g.dg + at * g.ldd + q0 + c) = odg;
        *(u32x4*)(g.du + at * g.ldd + q0 + c) = odu;
        if (g.h != nullptr) *(u32x4*)(g.h + at * g.ldh + q0 + c) = oh;
      }
    }
    if (quarter < 3) request(quarter + 1);
    own_lds_wait();
  }
}

}  // namespace

template <GatedOp OP, bool B_OC, Kept KEPT, bool EDGE>
__global__ __launch_bounds__(256, 1) void gated256_kernel(const GatedArgs g) {
  using namespace g256;
  constexpr uint32_t TC = OP == GatedOp::kFwd ? 128 : 256;   // columns of a tile
  uint32_t tile_m, tile_n;
  tile_of(TileGrid{(g.M + TM - 1) / TM, (g.N + TC - 1) / TC, g.inv_band, g.inv_last}, blockIdx.x, tile_m, tile_n);
  const uint32_t m0 = tile_m * TM, n0 = tile_n * TC, rows = g.M - m0 < TM ? g.M - m0 : TM, cols = g.N - n0 < TC ? g.N - n0 : TC;
  const uint32_t nk = (g.K + TK - 1) / TK;
  if constexpr (OP == GatedOp::kFwd) {
    gemm256_accumulate<false, B_OC, EDGE, 8, kPair>(g.a, g.lda, g.b, g.ldb, nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane) {
      fwd_out<KEPT, EDGE>(g, acc, (uint8_t*)cs, m0 + 128 * (wave >> 1), n0 + 64 * (wave & 1), lane);
    }, rows, cols, g.K, nullptr, g.b2);
  } else if constexpr (OP == GatedOp::kBwd) {
    gemm256_accumulate<false, B_OC, EDGE>(g.a, g.lda, g.b, g.ldb, nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane) {
      bwd_out<KEPT, EDGE>(g, acc, (float*)cs, m0 + 128 * (wave >> 1), n0 + 128 * (wave & 1), lane);
    }, rows, cols, g.K);
  } else {
    gemm256_accumulate<false, B_OC, EDGE, 8, kTwo>(g.a, g.lda, g.b, g.ldb, 2 * nk, m0, n0, [&](f32x4 (&acc)[8][8], uint16_t* cs, uint32_t wave, uint32_t lane) {
      uint16_t* yw = g.h + (size_t)(m0 + 128 * (wave >> 1)) * g.ldh + n0 + 128 * (wave & 1);
      const int wr = (int)rows - 128 * (int)(wave >> 1), wc = (int)cols - 128 * (int)(wave & 1);
      epilogue_bf16_half<EDGE>(*reinterpret_cast<const f32x4 (*)[4][8]>(&acc[0]), 0, cs, yw, g.ldh, lane, NoHook{}, wr, wc);
      epilogue_bf16_half<EDGE>(*reinterpret_cast<const f32x4 (*)[4][8]>(&acc[4]), 1, cs, yw, g.ldh, lane, NoHook{}, wr, wc);
    }, rows, cols, g.K, g.a2, g.b2);
  }
}

bool gated256_applicable(const GatedArgs& g) { return g.K >= 64 && g.lda < g256::kMaxLdEdge && g.ldb < g256::kMaxLdEdge; }

template <GatedOp OP, Kept KEPT, bool EDGE>
static int launch_tiles(GatedArgs g, bool b_oc, hipStream_t stream) {
  constexpr uint32_t TC = OP == GatedOp::kFwd ? 128 : 256;
  const uint32_t mt = (uint32_t)(((uint64_t)g.M + 255) / 256), nt = (uint32_t)(((uint64_t)g.N + TC - 1) / TC);
  if ((uint64_t)mt * nt >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  set_tile_grid(g, mt, nt, tile_band(mt, nt));
  if (b_oc) hipLaunchKernelGGL((gated256_kernel<OP, true, KEPT, EDGE>), dim3(mt * nt), dim3(256), 0, stream, g);
  else hipLaunchKernelGGL((gated256_kernel<OP, false, KEPT, EDGE>), dim3(mt * nt), dim3(256), 0, stream, g);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

template <GatedOp OP, Kept KEPT>
static int launch_edge(const GatedArgs& g, bool b_oc, hipStream_t stream) {
  const bool whole = g.M % 256 == 0 && g.N % (OP == GatedOp::kFwd ? 128 : 256) == 0 && g.K % 64 == 0;
  return whole ? launch_tiles<OP, KEPT, false>(g, b_oc, stream) : launch_tiles<OP, KEPT, true>(g, b_oc, stream);
}

int launch_gated256(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream) {
  if (op == GatedOp::kDx) return launch_edge<GatedOp::kDx, Kept::kNone>(g, b_oc, stream);
  if (op == GatedOp::kBwd)
    return kept == Kept::kE4m3 ? launch_edge<GatedOp::kBwd, Kept::kE4m3>(g, b_oc, stream) : launch_edge<GatedOp::kBwd, Kept::kBf16>(g, b_oc, stream);
  return kept == Kept::kE4m3 ? launch_edge<GatedOp::kFwd, Kept::kE4m3>(g, b_oc, stream)
         : kept == Kept::kBf16 ? launch_edge<GatedOp::kFwd, Kept::kBf16>(g, b_oc, stream) : launch_edge<GatedOp::kFwd, Kept::kNone>(g, b_oc, stream);
}

}  // namespace gws
