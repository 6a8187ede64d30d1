// Checks of arguments that several entry points share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "ml2.h"

namespace ml2 {

inline bool element_size(int32_t dtype, size_t *size) {
  if (dtype != ML2_F32 && dtype != ML2_BF16 && dtype != ML2_F16) return false;
  *size = dtype == ML2_F32 ? 4 : 2;
  return true;
}

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool size_ok(int64_t v) { return v >= 0 && v <= (int64_t)INT32_MAX; }

// Whether two matrices of `rows` rows of n elements of `size` bytes, lda and ldb
// elements apart and aligned to their elements, have one in common.  Columns of
// one buffer lie between one another without that.
inline bool overlap(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, int64_t n,
             size_t size) {
  if (!a || !b || rows <= 0 || n <= 0) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  if (pa > pb) return overlap(b, ldb, a, lda, rows, n, size);
  const uint64_t d = (pb - pa) / size;  // b's first element, counted from a's
  const uint64_t la = (uint64_t)lda, lb = (uint64_t)ldb, len = (uint64_t)n;
  if (d >= (uint64_t)(rows - 1) * la + len) return false;
  if (la == lb) {
    // row r of b begins in row r + d / la of a, or behind its end and reaches on
    // into the next
    const uint64_t at = d % la, row = d / la;
    return at < len || (row + 1 < (uint64_t)rows && at + len > la);
  }
  for (uint64_t i = 0, j = 0; i < (uint64_t)rows && j < (uint64_t)rows;) {
    const uint64_t x = i * la, y = d + j * lb;
    if (x < y + len && y < x + len) return true;
    if (x < y) ++i; else ++j;
  }
  return false;
}

}  // namespace ml2
