// Whether two arrays of rows have bytes in common: the host's check of outputs
// against inputs.
#pragma once

#include <algorithm>
#include <cstdint>

namespace tim {

// Rows of `width` bytes, `ld` bytes (at least `width`) apart.
struct Rows {
  const void* p;
  int64_t rows, width, ld;
};
inline Rows rows_of(const void* p, int64_t rows, int64_t n, int64_t ld, int bytes) {
  return {p, rows, n * bytes, ld * bytes};
}
// Bytes next to each other.
inline Rows flat(const void* p, int64_t rows, int64_t bytes) { return {p, rows, bytes, bytes}; }

// Whether the two have a byte in common. Rows beside each other in one buffer do not.
inline bool share_bytes(Rows a, Rows b) {
  typedef __int128 wide;
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
  const wide at = (wide)(uintptr_t)b.p - (wide)(uintptr_t)a.p;  // of b's first byte from a's
  if (at >= (wide)(a.rows - 1) * a.ld + a.width || -at >= (wide)(b.rows - 1) * b.ld + b.width) return false;
  auto one_row = [](Rows& r) {
    if (r.ld == r.width) r.width *= r.rows, r.rows = 1;
  };
  one_row(a), one_row(b);
  auto down = [](wide x, wide y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
  if (a.rows == 1 || b.rows == 1 || a.ld == b.ld) {
    // row i of a and row j of b do where -b.width < at + (j - i) ld < a.width
    const wide ld = a.rows == 1 ? (b.rows == 1 ? std::max(a.width, b.width) : b.ld) : a.ld;
    const wide least = std::max<wide>(down(-at - b.width, ld) + 1, 1 - a.rows);
    return least <= std::min<wide>(down(a.width - 1 - at, ld), b.rows - 1);
  }
  for (int64_t i = 0; i < a.rows; ++i) {
    // the last row of b that begins before row i of a ends
    const wide from = i * (wide)a.ld - at, j = std::min<wide>(down(from + a.width - 1, b.ld), b.rows - 1);
    if (j >= 0 && j * b.ld + b.width > from) return true;
  }
  return false;
}

}  // namespace tim
