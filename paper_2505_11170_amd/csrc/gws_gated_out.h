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

// The same of every wavefront of the workgroup.
__device__ __forceinline__ void both_lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Each m's largest of the four lanes lane % 16 + 16 x: v_permlane16_swap and v_permlane32_swap of m with itself leave a lane's own value in
// one result and its partner's in the other.  Together, so that one's steps fill the waits between another's.
template <int N>
__device__ __forceinline__ void max_over_rows(uint32_t (&m)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const auto a = __builtin_amdgcn_permlane16_swap(m[n], m[n], false, false);
    m[n] = max((uint32_t)a[0], (uint32_t)a[1]);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const auto b = __builtin_amdgcn_permlane32_swap(m[n], m[n], false, false);
    m[n] = max((uint32_t)b[0], (uint32_t)b[1]);
  }
}

// Pitch in bytes of a staged row of 16 NG values, BF16 or codes.
template <int NG, int BYTES>
constexpr int kPitch = 16 * NG * BYTES + 16;

// 64 staged rows of 16 NG BF16 values (codes) to rows of `ld` bytes at `to`; of them `rows` and, of the columns, `cols` exist
// (cols a multiple of 32).
template <int NG, int BYTES, bool EDGE, bool STREAM>
__device__ __forceinline__ void rows_out(const uint8_t* cs, uint8_t* to, size_t ld, uint32_t lane, int rows, int cols) {
  constexpr int PITCH = kPitch<NG, BYTES>, LANES = NG * BYTES, ROWS = 64 / LANES;   // lanes of a row, rows of an instruction
  const uint32_t r = lane / LANES, c = (lane % LANES) * 16;
  const bool col_in = !EDGE || (int)c < cols * BYTES;
#pragma unroll 4
  for (int it = 0; it < 64 / ROWS; ++it) {
    const uint32_t row = it * ROWS + r;
    if (!EDGE || ((int)row < rows && col_in)) {
      const u32x4 v = *(const u32x4*)(cs + row * PITCH + c);
      if (STREAM) __builtin_nontemporal_store(v, (u32x4*)(to + row * ld + c));
      else *(u32x4*)(to + row * ld + c) = v;
    }
  }
}

// H, and G and U as they are kept, of a wavefront's 16 NI rows x 16 NG columns from (p0, q0): a lane has both halves of an element
// (acc[i][j] with j < NG is G, acc[i][j + NG] U), and the four lanes of a block of 32 that is kept in 8 bits meet in two cross-lane
// steps.  Everything leaves through LDS by rows, 64 rows at a time; codes, of which a wavefront's columns are half a line or less, by the two
// wavefronts that share the rows (`odd`: this is the one with the later columns; first: the other's cs) together, G's by the one and U's by the
// other (8192 tokens, 2048 -> 5632: 1 % of 320 us; in 128 x 128 tiles 1021 x 768 -> 2048 12.8 -> 12.2).
template <Kept KEPT, bool EDGE, int NI, int NG, class G>
__device__ __forceinline__ void fwd_out_by(G gate, const GatedArgs& g, const f32x4 (&acc)[NI][2 * NG], uint8_t* cs, uint8_t* first, bool odd, uint32_t p0,
                                        uint32_t q0, uint32_t lane) {
  const uint32_t li = lane & 15, grp = lane >> 4;
  uint8_t* const hs = cs;                                    // 64 rows of H, then of G and of U
  constexpr int PH = kPitch<NG, 2>, PB = kPitch<2 * NG, 1>;
  constexpr int KS = 64 * (KEPT == Kept::kE4m3 ? PB : PH);   // bytes of staged G, of U
  uint8_t* const ks = (KEPT == Kept::kE4m3 ? first + 16 * NG * odd : cs) + 64 * PH;
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
      const uint32_t row = 16 * i2 + li;
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const f32x4 vg = acc[i][j], vu = acc[i][j + NG];
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = gate.a(vg[e]) * vu[e];
        *(u32x2*)(hs + row * PH + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3])};
        if (KEPT == Kept::kBf16) {
          *(u32x2*)(ks + row * PH + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(vg[0], vg[1]), pack_bf16_rne(vg[2], vg[3])};
          *(u32x2*)(ks + KS + row * PH + (16 * j + 4 * grp) * 2) = u32x2{pack_bf16_rne(vu[0], vu[1]), pack_bf16_rne(vu[2], vu[3])};
        }
      }
      if (KEPT == Kept::kE4m3) {
        uint32_t m[2 * NB];   // largest magnitudes of G's blocks, then of U's
#pragma unroll
        for (uint32_t b = 0; b < 2 * NB; ++b) {
          float top = 0.0f;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const f32x4& v = acc[i][2 * b + (t >> 1)];
            top = act8_larger(top, v[2 * (t & 1)], v[2 * (t & 1) + 1]);
          }
          m[b] = __float_as_uint(top) & 0x7FFFFFFFu;
        }
        max_over_rows(m);
        uint32_t mine = m[0], most = m[0];
#pragma unroll
        for (uint32_t b = 1; b < 2 * NB; ++b) {
          mine = grp == b ? m[b] : mine;
          most = max(most, m[b]);
        }
        if (grp < 2 * NB && (!EDGE || (16 * i + (int)li < rows && 32 * (int)(grp % NB) < cols))) sp[(size_t)(16 * i) * ls] = (uint8_t)act8_byte(mine);
        auto codes = [&](auto&& four) {
#pragma unroll
          for (int j = 0; j < 2 * NG; ++j) {
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            *(uint32_t*)(ks + j / NG * KS + row * PB + 16 * (j % NG) + 4 * grp) = four(v, j / 2);
          }
        };
        if (__builtin_amdgcn_ballot_w64(most >= kAct8Large) == 0) {   // uniform
          float scale[2 * NB];
#pragma unroll
          for (uint32_t b = 0; b < 2 * NB; ++b) scale[b] = act8_small_scale(m[b]);
          codes([&](const float (&v)[4], int b) { return act8_convert(v, scale[b]); });
        } else {
          codes([&](const float (&v)[4], int b) {
            const float w[4] = {act8_clamp(v[0]), act8_clamp(v[1]), act8_clamp(v[2]), act8_clamp(v[3])};   // under a smaller scale nothing is that large
            return act8_codes(w, act8_byte(m[b]));
          });
        }
      }
    }
    own_lds_wait();
    if (KEPT == Kept::kE4m3) both_lds_wait();
    const uint32_t r0 = p0 + 64 * h;
    // What is kept is wanted again a pass later: past the caches.  H is read at once, by the product that follows: so too only where it is
    // too large for the caches to keep until then (past_caches in gws_gated_api.hip).
    // (Two loops: of one with both stores the compiler makes ordinary ones.)
    uint8_t* const hp = (uint8_t*)(g.h + (size_t)r0 * g.ldh + q0);
    if (g.past_caches) rows_out<NG, 2, EDGE, true>(hs, hp, (size_t)g.ldh * 2, lane, rows - 64 * h, cols);
    else rows_out<NG, 2, EDGE, false>(hs, hp, (size_t)g.ldh * 2, lane, rows - 64 * h, cols);
    if (KEPT == Kept::kBf16) {
      rows_out<NG, 2, EDGE, true>(ks, g.kept.g + ((size_t)r0 * g.kept.ldg + q0) * 2, (size_t)g.kept.ldg * 2, lane, rows - 64 * h, cols);
      rows_out<NG, 2, EDGE, true>(ks + KS, g.kept.u + ((size_t)r0 * g.kept.ldu + q0) * 2, (size_t)g.kept.ldu * 2, lane, rows - 64 * h, cols);
    }
    if (KEPT == Kept::kE4m3) {
      const uint32_t c0 = q0 - 16 * NG * odd;
      const uint32_t ld = odd ? g.kept.ldu : g.kept.ldg;
      rows_out<2 * NG, 1, EDGE, true>(first + 64 * PH + KS * odd, (odd ? g.kept.u : g.kept.g) + (size_t)r0 * ld + c0, ld, lane, rows - 64 * h, (int)g.N - (int)c0);
      if (h + 1 < NI / 4) both_lds_wait();
    }
    own_lds_wait();
  }
}

// Kept values of eight columns on their way, and as fp32 pairs.
template <Kept KEPT>
struct KeptEight {
  u32x4 w;          // BF16, or codes in the first two
  uint32_t byte;
  // p, s: uniform; off, soff: the lane's bytes from there
  __device__ __forceinline__ void load(const GWS_GLOBAL uint8_t* p, const GWS_GLOBAL uint8_t* s, uint32_t off, uint32_t soff) {
    if (KEPT == Kept::kBf16) {
      w = __builtin_nontemporal_load((const GWS_GLOBAL u32x4*)(p + off));
    } else {
      const u32x2 c = __builtin_nontemporal_load((const GWS_GLOBAL u32x2*)(p + off));
      w = u32x4{c[0], c[1], 0, 0};
      byte = s[soff];
    }
  }
  __device__ __forceinline__ void landed() {
    if (KEPT == Kept::kE4m3) {
      w[0] = act8_read(w[0], byte);
      w[1] = act8_read(w[1], byte);
    }
  }
  __device__ __forceinline__ f32x2 pair(int d) const {
    if (KEPT == Kept::kBf16) return f32x2{bf16_lo(w[d]), bf16_hi(w[d])};
    return d & 1 ? act8_values<true>(w[d >> 1], byte) : act8_values<false>(w[d >> 1], byte);
  }
};

// A uniform pointer into row p0, byte `col` of a matrix; the rest of an address is uniform too but for a 32-bit lane offset of up to
// seven rows.
__device__ __forceinline__ GWS_GLOBAL uint8_t* at_row(const void* p, uint32_t row, size_t row_bytes, size_t col) {
  return (GWS_GLOBAL uint8_t*)(uintptr_t)p + (size_t)row * row_bytes + col;
}
constexpr uint32_t kMaxLdOut = 1u << 28;   // leading dimensions (elements) that reaches

// The kept G and U of a wavefront's 16 NI x 16 NJ part from (p0, q0), 32 rows at a time in two buffers; lane = (row % ROWS, 8 columns).
template <Kept KEPT, bool EDGE, int NI, int NJ>
struct KeptTile {
  static constexpr uint32_t LANES = 2 * NJ, ROWS = 64 / LANES, IT = 32 / ROWS, E = KEPT == Kept::kBf16 ? 2 : 1;
  KeptEight<KEPT> g[2][IT], u[2][IT];
  __device__ __forceinline__ void request(const GatedArgs& a, uint32_t p0, uint32_t q0, uint32_t lane, int quarter) {
    const uint32_t r = lane / LANES, c = lane % LANES * 8;
    const int rows = (int)a.M - (int)p0, cols = (int)a.N - (int)q0;
    const uint32_t g_off = (r * a.kept.ldg + c) * E, u_off = (r * a.kept.ldu + c) * E, gs_off = r * a.kept.lsg + (c >> 5), us_off = r * a.kept.lsu + (c >> 5);
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row0 = 32 * quarter + ROWS * it;
      if (!EDGE || ((int)(row0 + r) < rows && (int)c < cols)) {
        g[quarter & 1][it].load(at_row(a.kept.g, p0 + row0, (size_t)a.kept.ldg * E, (size_t)q0 * E), at_row(a.kept.gs, p0 + row0, a.kept.lsg, q0 >> 5), g_off, gs_off);
        u[quarter & 1][it].load(at_row(a.kept.u, p0 + row0, (size_t)a.kept.ldu * E, (size_t)q0 * E), at_row(a.kept.us, p0 + row0, a.kept.lsu, q0 >> 5), u_off, us_off);
      }
    }
  }
};

// dL/dG, dL/dU and H of a wavefront's 16 NI x 16 NJ part from (p0, q0): dL/dH leaves the accumulators through LDS as fp32, 32 rows at
// a time, and meets the kept G and U, which were requested before (the first 32 rows by the caller), 8 columns of a row a lane.
template <bool STREAM>
__device__ __forceinline__ void store_out(const u32x4& v, GWS_GLOBAL uint8_t* to) {
  if (STREAM) __builtin_nontemporal_store(v, (GWS_GLOBAL u32x4*)to);
  else *(GWS_GLOBAL u32x4*)to = v;
}
template <bool STREAM, Kept KEPT, bool EDGE, int NI, int NJ, class G>
__device__ __forceinline__ void bwd_out_by(G gate, const GatedArgs& g, const f32x4 (&acc)[NI][NJ], KeptTile<KEPT, EDGE, NI, NJ>& kept, float* cs, uint32_t p0,
                                           uint32_t q0, uint32_t lane) {
  constexpr int PF = 16 * NJ + 4;   // pitch of a staged row of fp32 (32 of them)
  constexpr uint32_t LANES = 2 * NJ, ROWS = 64 / LANES, IT = 32 / ROWS;
  const uint32_t li = lane & 15, grp = lane >> 4;
  const uint32_t r = lane / LANES, c = lane % LANES * 8;   // on the way out: row % ROWS, column
  const int rows = (int)g.M - (int)p0, cols = (int)g.N - (int)q0;
  const bool col_in = !EDGE || (int)c < cols;
  GWS_GLOBAL uint8_t *dgp = at_row(g.dg, p0, (size_t)g.ldd * 2, (size_t)q0 * 2), *dup = at_row(g.du, p0, (size_t)g.ldd * 2, (size_t)q0 * 2);
  GWS_GLOBAL uint8_t* hp = at_row(g.h, p0, (size_t)g.ldh * 2, (size_t)q0 * 2);
  const uint32_t d_off = (r * g.ldd + c) * 2, h_off = (r * g.ldh + c) * 2;
#pragma unroll
  for (int quarter = 0; quarter < NI / 2; ++quarter) {
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)(cs + (16 * i2 + li) * PF + 16 * j + 4 * grp) = acc[2 * quarter + i2][j];
    // before this quarter's stores: loads and stores complete in one order, and a wait for loads behind stores is one for those too
    if (quarter + 1 < NI / 2) kept.request(g, p0, q0, lane, quarter + 1);
    __builtin_amdgcn_sched_barrier(0);
    own_lds_wait();
    KeptEight<KEPT> (&vg)[IT] = kept.g[quarter & 1], (&vu)[IT] = kept.u[quarter & 1];
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row = ROWS * it + r;
      const f32x4 d0 = *(const f32x4*)(cs + row * PF + c), d1 = *(const f32x4*)(cs + row * PF + c + 4);
      if (!EDGE || (32 * quarter + (int)row < rows && col_in)) {
        u32x4 odg, odu, oh;
        vg[it].landed();
        vu[it].landed();
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const f32x2 pg = vg[it].pair(p), pu = vu[it].pair(p);
          const float u0 = pu[0], u1 = pu[1];
          const float h0 = p < 2 ? d0[2 * p] : d1[2 * p - 4], h1 = p < 2 ? d0[2 * p + 1] : d1[2 * p - 3];
          float a0, a1, s0, s1;
          gate.both(pg[0], a0, s0);
          gate.both(pg[1], a1, s1);
          odg[p] = pack_bf16_rne(h0 * u0 * s0, h1 * u1 * s1);
          odu[p] = pack_bf16_rne(h0 * a0, h1 * a1);
          oh[p] = pack_bf16_rne(a0 * u0, a1 * u1);
        }
        const uint32_t row0 = 32 * quarter + ROWS * it;
        store_out<STREAM>(odg, dgp + (size_t)row0 * g.ldd * 2 + d_off);
        store_out<STREAM>(odu, dup + (size_t)row0 * g.ldd * 2 + d_off);
        if (g.h != nullptr) store_out<STREAM>(oh, hp + (size_t)row0 * g.ldh * 2 + h_off);
      }
    }
    own_lds_wait();
  }
}

template <Kept KEPT, bool EDGE, int NI, int NG>
__device__ __forceinline__ void fwd_out(const GatedArgs& g, const f32x4 (&acc)[NI][2 * NG], uint8_t* cs, uint8_t* first, bool odd, uint32_t p0,
                                        uint32_t q0, uint32_t lane) {
  with_gate(g.act, [&](auto gate) { fwd_out_by<KEPT, EDGE, NI, NG>(gate, g, acc, cs, first, odd, p0, q0, lane); });
}
template <Kept KEPT, bool EDGE, int NI, int NJ>
__device__ __forceinline__ void bwd_out(const GatedArgs& g, const f32x4 (&acc)[NI][NJ], KeptTile<KEPT, EDGE, NI, NJ>& kept, float* cs, uint32_t p0, uint32_t q0,
                                        uint32_t lane) {
  with_gate(g.act, [&](auto gate) {
    if (g.past_caches) bwd_out_by<true, KEPT, EDGE, NI, NJ>(gate, g, acc, kept, cs, p0, q0, lane);   // uniform
    else bwd_out_by<false, KEPT, EDGE, NI, NJ>(gate, g, acc, kept, cs, p0, q0, lane);
  });
}
inline bool out_lds_ok(const GatedArgs& g) {
  const KeptArgs& k = g.kept;
  return g.ldd < kMaxLdOut && g.ldh < kMaxLdOut && k.ldg < kMaxLdOut && k.ldu < kMaxLdOut && k.lsg < kMaxLdOut && k.lsu < kMaxLdOut;
}

}  // namespace gws
