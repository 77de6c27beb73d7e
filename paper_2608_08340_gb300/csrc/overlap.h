// Whether memory that a call writes overlaps memory that it reads.  Host code without CUDA.
#pragma once

#include <cstdint>
#include <utility>

namespace oprag {

// `rows` rows of `bytes` bytes, `stride` bytes apart (at least `bytes`).
struct Rows {
  uintptr_t at;
  int64_t rows, bytes, stride;
  uintptr_t end() const { return at + static_cast<uintptr_t>((rows - 1) * stride + bytes); }
};

// Exact: rows that lie between the other's are apart from them.
inline bool overlap(Rows a, Rows b) {
  if (a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
  if (b.at < a.at) std::swap(a, b);
  // Rows of one stride meet at b's first row or nowhere: it lies between the ends of a, so
  // that a has the rows on both sides of it, and further rows lie to a's as it does.
  const int64_t n = a.stride == b.stride ? 1 : b.rows;
  for (int64_t i = 0; i < n; ++i) {
    const uintptr_t from = b.at + static_cast<uintptr_t>(i * b.stride);
    if (from >= a.end()) return false;
    // The last row of a that begins before this one ends.
    int64_t r = static_cast<int64_t>(from + static_cast<uintptr_t>(b.bytes) - 1 - a.at) / a.stride;
    if (r > a.rows - 1) r = a.rows - 1;
    if (a.at + static_cast<uintptr_t>(r * a.stride + a.bytes) > from) return true;
  }
  return false;
}

}  // namespace oprag
