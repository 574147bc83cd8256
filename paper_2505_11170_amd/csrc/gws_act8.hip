// Activations kept in 8 bits (gfx950): BF16 [M x C] to E4M3 codes with an E8M0 scale for every 32 of a row, and back.
// One pass over memory: a lane takes eight values, the four lanes of a block meet in two cross-lane steps, the scaled converters do the rest.
// Bound by memory: 8192 x 5632 to codes 26.3 us, 5.3 TB/s of the 3 bytes a value (a large copy reaches 5.15); 8192 x 2048 back 10.4 us, 4.9 TB/s
// where the codes come from memory.  301 x 1000 back is a launch, 2.1 us.
#include "gws_gated.h"

namespace gws {

struct Act8Args {
  uint16_t* x;
  uint8_t *codes, *scales;
  uint32_t M, C, ldx, ldc, lds;
  uint32_t per_row, inv;   // lanes a row: 4 ceil(C / 32)
};

// Row and first column of lane `id`; false past the end.
__device__ __forceinline__ bool act8_place(const Act8Args& a, uint32_t& row, uint32_t& c) {
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, total = (uint64_t)a.M * a.per_row;
  if (total < 0x80000000ull) {   // uniform
    row = divide((uint32_t)id, a.per_row, a.inv);
    c = ((uint32_t)id - row * a.per_row) * 8;
  } else {
    row = (uint32_t)(id / a.per_row);
    c = (uint32_t)(id - (uint64_t)row * a.per_row) * 8;
  }
  return id < total;
}

__global__ __launch_bounds__(256) void act8_encode_kernel(const Act8Args a) {
  uint32_t row, c;
  const bool in = act8_place(a, row, c);
  const int nv = !in || c >= a.C ? 0 : a.C - c < 8 ? (int)(a.C - c) : 8;
  u32x4 x = {0, 0, 0, 0};
  if (nv > 0) x = *(const u32x4*)(a.x + (size_t)row * a.ldx + c);   // ldx is a multiple of 8: never past the row's end
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k >= nv) x[k >> 1] &= k & 1 ? 0x0000FFFFu : 0xFFFF0000u;
    const uint32_t bits = k & 1 ? x[k >> 1] >> 16 : x[k >> 1] & 0xFFFFu;
    m = max(m, bits & 0x7FFFu);
  }
  m = max(m, dpp_u32<0xB1>(m));   // lane ^ 1
  m = max(m, dpp_u32<0x4E>(m));   // lane ^ 2
  const uint32_t byte = act8_byte(m << 16);
  uint32_t code[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float v[4] = {bf16_lo(x[2 * t]), bf16_hi(x[2 * t]), bf16_lo(x[2 * t + 1]), bf16_hi(x[2 * t + 1])};
    if (byte == kAct8Max) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = act8_clamp(v[e]);
    }
    code[t] = act8_codes(v, byte);
  }
  uint8_t* to = a.codes + (size_t)row * a.ldc + c;
  if (nv == 8) {
    *(uint64_t*)to = (uint64_t)code[1] << 32 | code[0];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < nv) to[k] = (uint8_t)(code[k >> 2] >> (8 * (k & 3)));
  }
  if (nv > 0 && (c & 31) == 0) a.scales[(size_t)row * a.lds + (c >> 5)] = (uint8_t)byte;
}

__global__ __launch_bounds__(256) void act8_decode_kernel(const Act8Args a) {
  uint32_t row, c;
  if (!act8_place(a, row, c) || c >= a.C) return;
  const uint64_t code = *(const uint64_t*)(a.codes + (size_t)row * a.ldc + c);   // ldc is a multiple of 8
  const uint32_t byte = a.scales[(size_t)row * a.lds + (c >> 5)], lo = act8_read((uint32_t)code, byte), hi = act8_read((uint32_t)(code >> 32), byte);
  const u32x4 v = {act8_pair<false>(lo, byte), act8_pair<true>(lo, byte), act8_pair<false>(hi, byte), act8_pair<true>(hi, byte)};
  uint16_t* to = a.x + (size_t)row * a.ldx + c;
  if (c + 8 <= a.C) {
    *(u32x4*)to = v;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k < a.C) to[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
  }
}

int launch_act8(bool encode, const void* x, uint64_t M, uint64_t C, uint64_t ldx, const gws_act8& o, hipStream_t stream) {
  const uint32_t per_row = (uint32_t)((C + 31) / 32) * 4;
  const uint64_t wgs = (M * per_row + 255) / 256;
  if (wgs >= 0x7FFFFFFFull) return GWS_ERR_SHAPE;
  const Act8Args a = {(uint16_t*)x, (uint8_t*)o.codes, o.xscale, (uint32_t)M, (uint32_t)C, (uint32_t)ldx, (uint32_t)o.ldc, (uint32_t)o.lds, per_row, reciprocal(per_row)};
  if (encode) hipLaunchKernelGGL(act8_encode_kernel, dim3((uint32_t)wgs), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(act8_decode_kernel, dim3((uint32_t)wgs), dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? GWS_OK : GWS_ERR_LAUNCH;
}

}  // namespace gws
