// The way out of the dense layer's products (internal to csrc/): bias, activation and residual, or the activation's backward pass, on the sums of a wavefront.
//   tiles that walk the contraction from end to end: acc[i][j][e] is row 16 i + lane % 16, column 16 j + 4 (lane / 16) + e of the wavefront's part.  The sums
//   leave the accumulators through the wavefront's own LDS as fp32, 32 rows at a time, and meet what is read there (the residual or Z, requested before),
//   eight columns of a row a lane.  A lane keeps its columns, so it keeps their bias and adds up their sums.
//   tiles whose wavefronts split the contraction: four columns of a row a thread, as the partial sums meet.
// With one wavefront a SIMD nothing hides the way out, so what it reads is on its way before the loop (the first rows) and before the stores of
// the rows before (a wait for loads behind stores waits for the stores too).
// Bound by vector instructions: GELU takes an exponential, a reciprocal and seven others an element, its slope five more.  8192 x 2048 -> 5632 in us, beside the plain product's
// 142: bias 5, GELU 12 to 15, keeping Z nothing that shows, a residual 12; backward the slope with Z's bytes 27, H 10, the bias gradient 4.  (Two quarters of Z or of
// the residual on their way instead of one brought nothing.)
#pragma once

#include "gws_dense.h"
#include "gws_gated_out.h"
#include "gws_gemm_stream_core.h"

namespace gws {

// ---- tiles that walk the contraction ----
template <DenseOp OP, bool EDGE, int NI, int NJ>
struct DenseHeld {
  // 2 NJ lanes a row; rows of an instruction: as many whole ones as divide 32 (NJ 3 and 6: 16 lanes idle)
  static constexpr uint32_t LANES = 2 * NJ, ROWS = NJ == 8 ? 4 : NJ == 4 ? 8 : NJ == 3 ? 8 : 4, IT = 32 / ROWS;
  static_assert(LANES * ROWS <= 64 && ROWS * IT == 32, "");
  u32x4 v[2][IT];    // residual or Z, 32 rows in each half
  float bias[8];
  __device__ __forceinline__ static bool column_in(const GemmArgs& g, uint32_t q0, uint32_t lane) {
    return (LANES * ROWS == 64 || lane < LANES * ROWS) && (!EDGE || (int)(lane % LANES * 8) < (int)g.N - (int)q0);
  }
  __device__ __forceinline__ void request(const GemmArgs& g, const DenseArgs& d, uint32_t p0, uint32_t q0, uint32_t lane, int quarter) {
    const uint16_t* p = OP == DenseOp::kFwd ? d.r : d.z;
    if (p == nullptr) return;   // uniform
    const uint32_t ld = OP == DenseOp::kFwd ? d.ldr : d.ldz, r = lane / LANES, off = (r * ld + lane % LANES * 8) * 2;
    const int rows = (int)g.M - (int)p0;
    const bool col_in = column_in(g, q0, lane);
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row0 = 32 * quarter + ROWS * it;
      if ((!EDGE || (int)(row0 + r) < rows) && col_in)
        v[quarter & 1][it] = __builtin_nontemporal_load((const GWS_GLOBAL u32x4*)(at_row(p, p0 + row0, (size_t)ld * 2, (size_t)q0 * 2) + off));
    }
  }
  __device__ __forceinline__ void begin(const GemmArgs& g, const DenseArgs& d, uint32_t p0, uint32_t q0, uint32_t lane) {
    if (OP == DenseOp::kFwd) vector_eight(d.bias, column_in(g, q0, lane) ? q0 + lane % LANES * 8 : g.N, g.N, 0.0f, bias);
    request(g, d, p0, q0, lane, 0);
  }
};

template <DenseOp OP, bool STREAM, bool EDGE, int NI, int NJ, class G>
__device__ __forceinline__ void dense_out_by(G gate, const GemmArgs& g, const DenseArgs& d, const f32x4 (&acc)[NI][NJ], DenseHeld<OP, EDGE, NI, NJ>& held, float* cs,
                                             uint32_t p0, uint32_t q0, uint32_t lane, uint32_t part_row) {
  using Held = DenseHeld<OP, EDGE, NI, NJ>;
  constexpr int PF = 16 * NJ + 4;   // pitch of a staged row of fp32 (32 of them)
  constexpr uint32_t LANES = Held::LANES, ROWS = Held::ROWS, IT = Held::IT;
  const uint32_t li = lane & 15, grp = lane >> 4, r = lane / LANES, c = lane % LANES * 8;
  const int rows = (int)g.M - (int)p0;
  const bool col_in = Held::column_in(g, q0, lane);
  GWS_GLOBAL uint8_t *yp = at_row(g.y, p0, (size_t)g.ldy * 2, (size_t)q0 * 2);
  const uint32_t y_off = (r * g.ldy + c) * 2;
  uint16_t* const second = OP == DenseOp::kFwd ? d.z : d.h;   // the other output
  const uint32_t ld2 = OP == DenseOp::kFwd ? d.ldz : d.ldh, off2 = (r * ld2 + c) * 2;
  GWS_GLOBAL uint8_t* p2 = at_row(second, p0, (size_t)ld2 * 2, (size_t)q0 * 2);
  const bool reads = (OP == DenseOp::kFwd ? d.r : d.z) != nullptr, sums = OP == DenseOp::kBwd && d.part != nullptr;
  float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int quarter = 0; quarter < NI / 2; ++quarter) {
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)(cs + (16 * i2 + li) * PF + 16 * j + 4 * grp) = acc[2 * quarter + i2][j];
    if (quarter + 1 < NI / 2) held.request(g, d, p0, q0, lane, quarter + 1);
    __builtin_amdgcn_sched_barrier(0);
    own_lds_wait();
    u32x4(&in)[IT] = held.v[quarter & 1];
#pragma unroll
    for (uint32_t it = 0; it < IT; ++it) {
      const uint32_t row = ROWS * it + r;
      if ((!EDGE || 32 * quarter + (int)row < rows) && col_in) {
        const f32x4 s0 = *(const f32x4*)(cs + row * PF + c), s1 = *(const f32x4*)(cs + row * PF + c + 4);
        float s[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]}, o[8], other[8], e[8];
        const uint32_t row0 = 32 * quarter + ROWS * it;
        // uniform branches around what a call leaves out: a vector instruction an element is 1 % of a large tile's time
        if (OP == DenseOp::kFwd) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            other[k] = s[k] + held.bias[k];
            o[k] = gate.a(other[k]);
          }
          if (reads) {
            widen(in[it], e);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] += e[k];
          }
        } else {
          if (reads) widen(in[it], e);
          else widen(u32x4{0, 0, 0, 0}, e);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float slope;
            gate.both(e[k], other[k], slope);
            o[k] = s[k] * slope;
          }
          if (sums) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              total[k] += o[k];
              asm volatile("" : "+v"(total[k]));   // here: put off to the end of it all, the additions keep every row's values (to scratch)
            }
          }
        }
        store_out<STREAM>(narrow(o), yp + (size_t)row0 * g.ldy * 2 + y_off);
        // Z is wanted again a pass later: past the caches
        if (second != nullptr) store_out<OP == DenseOp::kFwd || STREAM>(narrow(other), p2 + (size_t)row0 * ld2 * 2 + off2);
      }
      if (it % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // two rows' arithmetic together; all of them is more than the registers hold
    }
    own_lds_wait();
  }
  if (sums && rows > 0) {   // uniform: the sums of the wavefront's rows
    if (LANES * ROWS == 64 || lane < LANES * ROWS) {
      *(f32x4*)(cs + r * (16 * NJ) + c) = f32x4{total[0], total[1], total[2], total[3]};
      *(f32x4*)(cs + r * (16 * NJ) + c + 4) = f32x4{total[4], total[5], total[6], total[7]};
    }
    own_lds_wait();
#pragma unroll
    for (uint32_t col = lane; col < 16 * NJ; col += 64) {
      float s = cs[col];
#pragma unroll
      for (uint32_t k = 1; k < ROWS; ++k) s += cs[k * (16 * NJ) + col];
      if (q0 + col < g.N) d.part[(size_t)part_row * g.N + q0 + col] = s;
    }
  }
}
template <DenseOp OP, bool EDGE, int NI, int NJ>
__device__ __forceinline__ void dense_out(const GemmArgs& g, const DenseArgs& d, const f32x4 (&acc)[NI][NJ], DenseHeld<OP, EDGE, NI, NJ>& held, float* cs, uint32_t p0,
                                          uint32_t q0, uint32_t lane, uint32_t part_row) {
  with_act(d.act, [&](auto gate) {
    if (d.past_caches) dense_out_by<OP, true, EDGE, NI, NJ>(gate, g, d, acc, held, cs, p0, q0, lane, part_row);   // uniform
    else dense_out_by<OP, false, EDGE, NI, NJ>(gate, g, d, acc, held, cs, p0, q0, lane, part_row);
  });
}

// of gemm128_kernel: a wavefront has 64 x 16 NJ of the tile, and a row of partial sums
template <int NJ, DenseOp OP>
__device__ __forceinline__ DenseHeld<OP, true, 4, NJ> before128(const GemmArgs& g, uint32_t m0, uint32_t n0, uint32_t wave, uint32_t lane, const DenseWay<OP>& way) {
  DenseHeld<OP, true, 4, NJ> held;
  held.begin(g, way.d, m0 + 64 * (wave >> 1), n0 + 16 * NJ * (wave & 1), lane);
  return held;
}
template <int NJ, int D, DenseOp OP>
__device__ __forceinline__ void finish128(const GemmArgs& g, const f32x4 (&acc)[4][NJ], DenseHeld<OP, true, 4, NJ>& held, uint16_t* lds, uint32_t wave, uint32_t lane,
                                          uint32_t m0, uint32_t n0, const DenseWay<OP>& way) {
  constexpr uint32_t SHARE = D * (128 + 32 * NJ) * 64 / 4;   // elements of the ring that are a wavefront's
  static_assert(SHARE * 2 >= 32 * (16 * NJ + 4) * 4, "32 rows are staged in it");
  const uint32_t p0 = m0 + 64 * (wave >> 1);
  dense_out<OP, true, 4, NJ>(g, way.d, acc, held, (float*)(lds + wave * SHARE), p0, n0 + 16 * NJ * (wave & 1), lane, p0 / 64);
}

// ---- tiles whose wavefronts split the contraction ----
template <DenseOp OP, int MT, int NT, int P, int BM, int BN>
struct DenseHeldFours {
  static constexpr int MC = MT > 4 ? 4 : MT, PASSES = MT / MC;
  static constexpr uint32_t C4 = 4 * NT, FOURS = (MC * 16 * C4 + P * 64 - 1) / (P * 64);
  static_assert(P * 64 % C4 == 0, "a thread keeps its columns");
  u32x2 v[PASSES][FOURS];
  f4 bias;
  // four columns of a row of pass `pass`, the n-th of a thread
  __device__ __forceinline__ static bool place(const GemmArgs& g, uint32_t m0, uint32_t n0, int pass, uint32_t n, uint32_t& r, uint32_t& row, uint32_t& col) {
    const uint32_t c = threadIdx.x % C4;
    r = (threadIdx.x + n * P * 64) / C4;
    row = m0 + 16 * MC * pass + r;
    col = n0 + 4 * c;
    return row < g.M && col < g.N && r < 16 * MC && (BM == 16 * MT || r < BM) && (BN == 16 * NT || 4 * c < BN);
  }
};
template <int MT, int NT, int P, int BM, int BN, DenseOp OP>
__device__ __forceinline__ DenseHeldFours<OP, MT, NT, P, BM, BN> before_stream(const GemmArgs& g, uint32_t m0, uint32_t n0, const DenseWay<OP>& way) {
  using Held = DenseHeldFours<OP, MT, NT, P, BM, BN>;
  Held held;
  const DenseArgs& d = way.d;
  const uint16_t* p = OP == DenseOp::kFwd ? d.r : d.z;
  const uint32_t ld = OP == DenseOp::kFwd ? d.ldr : d.ldz;
  held.bias = f4{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t c = n0 + 4 * (threadIdx.x % Held::C4);
  if (OP == DenseOp::kFwd && d.bias != nullptr && c < g.N) held.bias = *(const GWS_GLOBAL f4_any*)global_ptr<float>(d.bias + c);
#pragma unroll
  for (int pass = 0; pass < Held::PASSES; ++pass)
#pragma unroll
    for (uint32_t n = 0; n < Held::FOURS; ++n) {
      uint32_t r, row, col;
      held.v[pass][n] = u32x2{0, 0};
      if (p != nullptr && Held::place(g, m0, n0, pass, n, r, row, col)) held.v[pass][n] = *(const GWS_GLOBAL u32x2*)(global_ptr<uint16_t>(p) + (size_t)row * ld + col);
    }
  return held;
}
template <int MT, int NT, int P, int BM, int BN, DenseOp OP>
__device__ __forceinline__ void finish_stream(const GemmArgs& g, const f32x4 (&acc)[MT][NT], const DenseHeldFours<OP, MT, NT, P, BM, BN>& held, char* lds, uint32_t m0,
                                              uint32_t n0, const DenseWay<OP>& way) {
  using Held = DenseHeldFours<OP, MT, NT, P, BM, BN>;
  constexpr uint32_t PITCH = 4 * NT + 1, C4 = Held::C4;
  constexpr int MC = Held::MC;
  const DenseArgs& d = way.d;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = threadIdx.x % C4;
  f32x4* red = (f32x4*)lds;
  float total[4] = {0, 0, 0, 0};
#pragma unroll
  for (int pass = 0; pass < Held::PASSES; ++pass) {
    __syncthreads();   // what was in this memory is read
#pragma unroll
    for (int i = 0; i < MC; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) red[((wave * MC + i) * 16 + (lane & 15)) * PITCH + 4 * j + (lane >> 4)] = acc[MC * pass + i][j];
    __syncthreads();
#pragma unroll
    for (uint32_t n = 0; n < Held::FOURS; ++n) {
      uint32_t r, row, col;
      if (!Held::place(g, m0, n0, pass, n, r, row, col)) continue;
      f32x4 s = red[r * PITCH + c];
#pragma unroll
      for (int w = 1; w < P; ++w) {
        const f32x4 v = red[(w * MC * 16 + r) * PITCH + c];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = __fadd_rn(s[e], v[e]);
      }
      const u32x2 in = held.v[pass][n];
      const float x[4] = {lo_of(in[0]), hi_of(in[0]), lo_of(in[1]), hi_of(in[1])};
      float o[4], other[4];
      with_act(d.act, [&](auto gate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (OP == DenseOp::kFwd) {
            other[e] = s[e] + held.bias[e];
            o[e] = gate.a(other[e]) + x[e];
          } else {
            float slope;
            gate.both(x[e], other[e], slope);
            o[e] = s[e] * slope;
            total[e] += o[e];
          }
        }
      });
      *(u32x2*)(g.y + (size_t)row * g.ldy + col) = u32x2{pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3])};
      uint16_t* const second = OP == DenseOp::kFwd ? d.z : d.h;
      if (second != nullptr)
        *(u32x2*)(second + (size_t)row * (OP == DenseOp::kFwd ? d.ldz : d.ldh) + col) = u32x2{pack_bf16_rne(other[0], other[1]), pack_bf16_rne(other[2], other[3])};
    }
  }
  if (OP == DenseOp::kBwd && d.part != nullptr) {   // uniform: the tile's rows
    constexpr uint32_t GROUPS = P * 64 / C4, USED = GROUPS < 16 * MC ? GROUPS : 16 * MC;   // threads of a column, and those that had rows
    __syncthreads();
    if (threadIdx.x / C4 < USED) red[threadIdx.x / C4 * C4 + c] = f32x4{total[0], total[1], total[2], total[3]};
    __syncthreads();
    const uint32_t col = threadIdx.x;
    if (col < BN && n0 + col < g.N) {
      const float* t = (const float*)red;
      float s = t[col];
#pragma unroll
      for (uint32_t k = 1; k < USED; ++k) s += t[k * 16 * NT + col];
      d.part[(size_t)(m0 / BM) * g.N + n0 + col] = s;
    }
  }
}

}  // namespace gws
