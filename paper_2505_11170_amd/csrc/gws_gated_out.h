// The way out of the gated block's products (internal to csrc/): the gate on the sums of a wavefront, for the tiles that walk the
// contraction from end to end.  acc[i][j][e]: row 16 i + lane % 16, column 16 j + 4 (lane / 16) + e of the wavefront's part; cs: LDS of the
// wavefront's own.  EDGE: only rows below g.M and columns below g.N exist.
#pragma once

#include "gws_gated.h"
#include "gws_gemm256_core.h"

namespace gws {

// This wavefront's LDS writes have landed / its reads are done.
__device__ __forceinline__ void own_lds_wait() {
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  __builtin_amdgcn_wave_barrier();
}

// Pitch in bytes of a staged row of 16 NG values, BF16 or codes.
template <int NG, int BYTES>
constexpr int kPitch = 16 * NG * BYTES + 16;

// 64 staged rows of 16 NG BF16 values (codes) to rows of `ld` bytes at `to`; of them `rows` and, of the columns, `cols` exist
// (cols a multiple of 32).
template <int NG, int BYTES, bool EDGE>
__device__ __forceinline__ void rows_out(const uint8_t* cs, uint8_t* to, size_t ld, uint32_t lane, int rows, int cols) {
  constexpr int PITCH = kPitch<NG, BYTES>, LANES = NG * BYTES, ROWS = 64 / LANES;   // lanes of a row, rows of an instruction
  const uint32_t r = lane / LANES, c = (lane % LANES) * 16;
  const bool col_in = !EDGE || (int)c < cols * BYTES;
#pragma unroll 4
  for (int it = 0; it < 64 / ROWS; ++it) {
    const uint32_t row = it * ROWS + r;
    if (!EDGE || ((int)row < rows && col_in)) *(u32x4*)(to + row * ld + c) = *(const u32x4*)(cs + row * PITCH + c);
  }
}

// H, and G and U as they are kept, of a wavefront's 16 NI rows x 16 NG columns from (p0, q0): a lane has both halves of an element
// (acc[i][j] with j < NG is G, acc[i][j + NG] U), and the four lanes of a block of 32 that is kept in 8 bits meet in two cross-lane
// steps.  Everything leaves through LDS by rows, 64 rows at a time.
template <Kept KEPT, bool EDGE, int NI, int NG>
__device__ __forceinline__ void fwd_out(const GatedArgs& g, const f32x4 (&acc)[NI][2 * NG], uint8_t* cs, uint32_t p0, uint32_t q0, uint32_t lane) {
  const uint32_t li = lane & 15, grp = lane >> 4;
  uint8_t* const hs = cs;                                    // 64 rows of H, then of G and of U
  constexpr int PH = kPitch<NG, 2>, PB = kPitch<NG, 1>;
  uint8_t* const ks[2] = {cs + 64 * PH, cs + 64 * PH + 64 * (KEPT == Kept::kE4m3 ? PB : PH)};
  const int rows = (int)g.M - (int)p0, cols = (int)g.N - (int)q0;   // EDGE: what exists, may be <= 0
  // 8 bits: the lane groups store the scales, of G's NG / 2 blocks and then of U's
  constexpr uint32_t NB = NG / 2;
  static_assert(NG == 2 || NG == 4, "");
  uint8_t* sp = nullptr;
  size_t ls = 0;
  if (KEPT == Kept::kE4m3) {
    ls = grp < NB ? g.kept.lsg : g.kept.lsu;
    sp = (grp < NB ? g.kept.gs : g.kept.us) + (size_t)(p0 + li) * ls + (q0 >> 5) + grp % NB;
  }
#pragma unroll
  for (int h = 0; h < NI / 4; ++h) {
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2) {
      const int i = 4 * h + i2;
      uint32_t byte[2][NB] = {};   // [G, U][block]
      if (KEPT == Kept::kE4m3) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int b = 0; b < (int)NB; ++b) {
            uint32_t m = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(acc[i][NG * p + 2 * b + t][e]) & 0x7FFFFFFFu);
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            byte[p][b] = act8_byte(m);
          }
        uint32_t mine = byte[0][0];
#pragma unroll
        for (uint32_t n = 1; n < 2 * NB; ++n) mine = grp == n ? byte[n / NB][n % NB] : mine;
        if (grp < 2 * NB && (!EDGE || (16 * i + (int)li < rows && 32 * (int)(grp % NB) < cols))) sp[(size_t)(16 * i) * ls] = (uint8_t)mine;
      }
      const uint32_t row = 16 * i2 + li;
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        float v[2][4], o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[0][e] = acc[i][j][e];
          v[1][e] = acc[i][j + NG][e];
          o[e] = gate_a(g.gate, v[0][e]) * v[1][e];
        }
        *(u32x2*)(hs + row * PH + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3])};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (KEPT == Kept::kBf16)
            *(u32x2*)(ks[p] + row * PH + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(v[p][0], v[p][1]), pack_bf16_rne(v[p][2], v[p][3])};
          if (KEPT == Kept::kE4m3) *(uint32_t*)(ks[p] + row * PB + 16 * j + 4 * grp) = act8_codes(v[p], byte[p][j >> 1]);
        }
      }
    }
    own_lds_wait();
    const uint32_t r0 = p0 + 64 * h;
    rows_out<NG, 2, EDGE>(hs, (uint8_t*)(g.h + (size_t)r0 * g.ldh + q0), (size_t)g.ldh * 2, lane, rows - 64 * h, cols);
    if (KEPT == Kept::kBf16) {
      rows_out<NG, 2, EDGE>(ks[0], g.kept.g + ((size_t)r0 * g.kept.ldg + q0) * 2, (size_t)g.kept.ldg * 2, lane, rows - 64 * h, cols);
      rows_out<NG, 2, EDGE>(ks[1], g.kept.u + ((size_t)r0 * g.kept.ldu + q0) * 2, (size_t)g.kept.ldu * 2, lane, rows - 64 * h, cols);
    }
    if (KEPT == Kept::kE4m3) {
      rows_out<NG, 1, EDGE>(ks[0], g.kept.g + (size_t)r0 * g.kept.ldg + q0, g.kept.ldg, lane, rows - 64 * h, cols);
      rows_out<NG, 1, EDGE>(ks[1], g.kept.u + (size_t)r0 * g.kept.ldu + q0, g.kept.ldu, lane, rows - 64 * h, cols);
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

// dL/dG, dL/dU and H of a wavefront's 16 NI x 16 NJ part from (p0, q0): dL/dH leaves the accumulators through LDS as fp32, 32 rows at
// a time, and meets the kept G and U, which were requested before, 8 columns of a row a lane.
template <Kept KEPT, bool EDGE, int NI, int NJ>
__device__ __forceinline__ void bwd_out(const GatedArgs& g, const f32x4 (&acc)[NI][NJ], float* cs, uint32_t p0, uint32_t q0, uint32_t lane) {
  constexpr int PF = 16 * NJ + 4;   // pitch of a staged row of fp32 (32 of them)
  constexpr uint32_t LANES = 2 * NJ, ROWS = 64 / LANES, IT = 32 / ROWS;
  const uint32_t li = lane & 15, grp = lane >> 4;
  const uint32_t r = lane / LANES, c = lane % LANES * 8;   // on the way out: row % ROWS, column
  const int rows = (int)g.M - (int)p0, cols = (int)g.N - (int)q0;
  const bool col_in = !EDGE || (int)c < cols;
  KeptEight<KEPT> vg[IT], vu[IT];
  auto request = [&](int quarter) {
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row = 32 * quarter + ROWS * it + r;
      if (!EDGE || ((int)row < rows && col_in)) {
        vg[it].load(g.kept.g, g.kept.gs, g.kept.ldg, g.kept.lsg, p0 + row, q0 + c);
        vu[it].load(g.kept.u, g.kept.us, g.kept.ldu, g.kept.lsu, p0 + row, q0 + c);
      }
    }
  };
  request(0);
#pragma unroll
  for (int quarter = 0; quarter < NI / 2; ++quarter) {
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)(cs + (16 * i2 + li) * PF + 16 * j + 4 * grp) = acc[2 * quarter + i2][j];
    own_lds_wait();
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row = ROWS * it + r;
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
    if (quarter + 1 < NI / 2) request(quarter + 1);
    own_lds_wait();
  }
}

}  // namespace gws
