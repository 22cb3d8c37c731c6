// Whether two arrays of rows share a byte. Host code only.
#pragma once

#include <cstdint>

namespace bo {

// Rows of `width` bytes, `pitch` apart; none where p is null. A vector is one row.
struct Span {
  const void* p;
  int64_t rows, width, pitch;
};

// False only where they share nothing. Rows at a and b modulo a number that divides
// both pitches lie in the same columns throughout, so that column ranges of one buffer
// are told apart, also where one side is a single row (its pitch does not count) or
// takes every so-many'th row. Ranges that interleave in other ways count as shared.
inline bool share(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t step_a = a.rows > 1 ? static_cast<uint64_t>(a.pitch) : 0;
  const uint64_t step_b = b.rows > 1 ? static_cast<uint64_t>(b.pitch) : 0;
  const uint64_t wa = static_cast<uint64_t>(a.width), wb = static_cast<uint64_t>(b.width);
  if (pa >= pb + (static_cast<uint64_t>(b.rows) - 1) * step_b + wb) return false;
  if (pb >= pa + (static_cast<uint64_t>(a.rows) - 1) * step_a + wa) return false;
  uint64_t common = step_a;
  for (uint64_t r = step_b; r;) {
    const uint64_t t = common % r;
    common = r;
    r = t;
  }
  if (!common) return true;                        // a row each
  const uint64_t off = pb >= pa ? (pb - pa) % common : (common - (pa - pb) % common) % common;
  return off < wa || common - off < wb;
}

}  // namespace bo
