// What the C entry points ask of their buffers (host code, internal to csrc/).
#pragma once

#include <stddef.h>
#include <stdint.h>

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

}  // namespace gws
