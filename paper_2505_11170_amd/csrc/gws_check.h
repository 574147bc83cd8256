// What the C entry points ask of their buffers (host code, internal to csrc/).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "gws.h"

namespace gws {

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline bool overlap2(const void* a, size_t abytes, const void* b, size_t bbytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + bbytes && y < x + abytes;
}

// A matrix in memory: rows of `width` bytes, `pitch` bytes apart.
struct Span2 {
  const void* p;
  size_t rows, width, pitch;
  size_t bytes() const { return rows == 0 ? 0 : (rows - 1) * pitch + width; }
};

// Whether two matrices share no byte.  Columns of one buffer, as halves of wider rows, lie between each other's rows.
inline bool apart(const Span2& a, const Span2& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes() == 0 || b.bytes() == 0) return true;
  if (!overlap2(a.p, a.bytes(), b.p, b.bytes())) return true;
  if (a.pitch != b.pitch || a.pitch == 0) return false;
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  const size_t d = y >= x ? (y - x) % a.pitch : (a.pitch - (x - y) % a.pitch) % a.pitch;   // where b's rows begin in a's
  return d >= a.width && a.pitch - d >= b.width;
}

// Sizes and leading dimensions.
constexpr int64_t kMaxDim = (int64_t)1 << 31;

inline bool size_ok(int64_t n) { return n >= 0 && n < kMaxDim; }
// A BF16 matrix's leading dimension.
inline bool ld_ok(int64_t ld, int64_t cols) { return ld >= cols && ld < kMaxDim && (ld & 7) == 0; }
// By leading dimensions the kernel is chosen: of a matrix that is not there any number may stand in the call.
inline uint32_t ld_of(const void* p, int64_t ld) { return p ? (uint32_t)ld : 0; }
inline Span2 span16(const void* p, int64_t rows, int64_t cols, int64_t ld) { return Span2{p, (size_t)rows, (size_t)cols * 2, (size_t)ld * 2}; }
inline bool same_place(const Span2& a, const Span2& b) { return a.p == b.p && a.pitch == b.pitch && a.width == b.width && a.rows == b.rows; }

inline int check_act8(const gws_act8& a, int64_t M, int64_t C) {
  if (!a.codes || !a.xscale) return GWS_ERR_NULL;
  if (a.ldc < C || a.ldc >= kMaxDim || (a.ldc & 7) != 0 || a.lds < (C + 31) / 32 || a.lds >= kMaxDim) return GWS_ERR_SHAPE;
  return aligned(a.codes, 8) ? GWS_OK : GWS_ERR_ALIGN;
}

// A list of matrices of which some are written.
struct Buffers {
  Span2 in[8], out[8];
  int ins = 0, outs = 0;
  void reads(const Span2& s) { if (s.p) in[ins++] = s; }
  void writes(const Span2& s) { if (s.p) out[outs++] = s; }
  // No output on another one; none on an input, but for the ones at the very same place where `in_place` allows those.
  bool apart_all(bool in_place) const {
    for (int i = 0; i < outs; ++i) {
      for (int j = 0; j < i; ++j)
        if (!apart(out[i], out[j])) return false;
      for (int j = 0; j < ins; ++j)
        if (!apart(out[i], in[j]) && !(in_place && same_place(out[i], in[j]))) return false;
    }
    return true;
  }
};

// From a matrix's first byte to behind its last.
struct Range {
  uintptr_t from, to;
};
inline Range range_of(const Span2& s) { return Range{(uintptr_t)s.p, s.p ? (uintptr_t)s.p + s.bytes() : (uintptr_t)s.p}; }
inline bool ranges_apart(const Range& a, const Range& b) { return a.to <= b.from || b.to <= a.from; }

}  // namespace gws
