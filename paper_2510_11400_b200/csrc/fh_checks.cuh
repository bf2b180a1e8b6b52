// Checks of arguments that the host sides of the matrix and head functions share.
#pragma once

#include "../../include/fh.h"

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace fh {

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
inline size_t esize_of(int dtype) { return dtype == FH_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == FH_F32 || dtype == FH_BF16; }

inline int check_matrix(const fh_matrix* m) {
  if (!m || !is_dtype(m->dtype) || m->rows < 1 || m->cols < 1 || m->reserved != 0) return FH_ERR_ARG;
  // (addresses are formed in 64 bits of bytes)
  if (m->ld < m->cols || m->ld > (INT64_MAX >> 3) / m->rows) return FH_ERR_ARG;
  return FH_OK;
}

// Whether two pieces of memory have a byte in common (a null pointer has none).
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + b_bytes && y < x + a_bytes;
}
// Bytes from the first to the last of a matrix.
inline size_t extent(int64_t rows, int64_t cols, int64_t ld, int dtype) { return ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * esize_of(dtype); }

// Rows of `width` bytes, `step` apart (a vector, a container: one).
struct Rows {
  uintptr_t at;
  uint64_t rows, step, width;  // width <= step
  Rows(const void* p, uint64_t bytes) : at((uintptr_t)p), rows(1), step(bytes), width(bytes) {}
  Rows(const void* p, int64_t r, int64_t cols, int64_t ld, int dtype) : at((uintptr_t)p), rows(r), step((uint64_t)ld * esize_of(dtype)), width((uint64_t)cols * esize_of(dtype)) {}
  uint64_t end() const { return at + (rows - 1) * step + width; }
};
// Whether they have a byte in common; rows that lie between one another's have none.
inline bool meet(const Rows& a, const Rows& b) {
  if (!a.at || !b.at || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.rows > b.rows) return meet(b, a);
  if (a.rows > 1 && a.step == b.step) {
    // row j of b begins d + (j - i) * step behind row i of a: only the two distances next to zero, `near` and `near - step`, can be too small
    const int64_t step = (int64_t)a.step, d = (int64_t)(b.at - a.at), less = d >= 0 ? d / step : -((-d + step - 1) / step);
    const uint64_t near = (uint64_t)(d - less * step);
    auto there = [&](int64_t rows) { return rows > -(int64_t)a.rows && rows < (int64_t)b.rows; };  // j - i
    return (near < a.width && there(-less)) || (a.step - near < b.width && there(-less - 1));
  }
  for (uint64_t i = 0; i < a.rows; ++i) {
    const uint64_t x = a.at + i * a.step, j = x > b.at ? std::min<uint64_t>((x - b.at) / b.step, b.rows - 1) : 0, y = b.at + j * b.step;
    if (x < y + b.width && y < x + a.width) return true;
    if (j + 1 < b.rows && y + b.step < x + a.width) return true;
  }
  return false;
}
// Whether the first of them meets one of the others.
template <typename... T>
inline bool meets(const Rows& a, const T&... others) {
  return (meet(a, others) || ...);
}

}  // namespace fh
