// Argument checks that the C entry points share.
#pragma once
#include <cstdint>

#include "rosaq_internal.h"

namespace rosaq {

// Sets the error text, where there is memory for it: nothing throws through a C entry.
inline int fail(int code, const char* msg) {
  try { set_error(msg); } catch (...) {}
  return code;
}

inline bool misaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// Whether two matrices of M rows, leading dimensions and widths in bytes, share memory.  With one leading dimension they may be columns of one buffer.
inline bool overlap_bytes(const void* x, int64_t ldx, int64_t wx, const void* y, int64_t ldy, int64_t wy, int M) {
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), x1 = x0 + (static_cast<uint64_t>(M - 1) * ldx + wx);
  const uintptr_t y0 = reinterpret_cast<uintptr_t>(y), y1 = y0 + (static_cast<uint64_t>(M - 1) * ldy + wy);
  if (!(x0 < y1 && y0 < x1)) return false;
  if (ldx != ldy) return true;
  const uint64_t row = static_cast<uint64_t>(ldx);
  const uint64_t at = y0 >= x0 ? (y0 - x0) % row : (row - (x0 - y0) % row) % row;     // of y's rows within x's
  return !(at >= static_cast<uint64_t>(wx) && at + static_cast<uint64_t>(wy) <= row);
}

}  // namespace rosaq
