// Whether two operands share memory: host code alone.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace grpo {

typedef __int128 wide;  // any stride times any number of rows

// n rows of `length` bytes, `step` bytes apart (>= length).
struct ByteRows {
  const void* p;
  wide n, length, step;
  ByteRows(const void* p_, int64_t rows, int64_t cols, int64_t ld, size_t esz)
      : p(p_), n(rows), length((wide)cols * (wide)esz), step((wide)(rows > 1 ? ld : cols) * (wide)esz) {
    if (step == length) {  // one row
      length *= n;
      step = length;
      n = 1;
    }
  }
};

// Rows i of a and j of b share a byte where (i - j) steps of equal size, or i steps alone, come close enough; rows of different
// steps are gone through one by one, those of the side that has fewer.  NULL shares nothing.
inline bool rows_share(const ByteRows& a, const ByteRows& b) {
  if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.length < 1 || b.length < 1) return false;
  if (a.n > b.n) return rows_share(b, a);
  const wide a0 = (wide)(uintptr_t)a.p, b0 = (wide)(uintptr_t)b.p;
  if (a0 + (a.n - 1) * a.step + a.length <= b0 || b0 + (b.n - 1) * b.step + b.length <= a0) return false;
  if (b.n == 1) return true;
  // whether d - a.length < k step < d + b.length for a k of lo .. hi
  auto meets = [&](wide d, wide step, wide lo, wide hi) {
    auto floor_div = [](wide x, wide y) { return x / y - (x % y < 0 ? 1 : 0); };
    lo = std::max(lo, floor_div(d - a.length, step) + 1);
    hi = std::min(hi, floor_div(d + b.length - 1, step));
    return lo <= hi;
  };
  if (a.step == b.step) return meets(b0 - a0, a.step, 1 - b.n, a.n - 1);
  for (wide i = 0; i < a.n; ++i)
    if (meets(b0 - (a0 + i * a.step), b.step, 1 - b.n, 0)) return true;
  return false;
}

}  // namespace grpo
