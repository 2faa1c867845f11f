// Checks of arguments that the entry points of row-major tensors share.
#pragma once

#include "poetx_common.h"

namespace poetx {

inline bool dtype_ok(int dtype) { return dtype == POETX_F32 || dtype == POETX_BF16; }
inline size_t esize(int dtype) { return dtype == POETX_F32 ? 4 : 2; }
// Do a and b, `na` and `nb` bytes from each, share any?  Nothing overlaps nothing.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const char *x = (const char*)a, *y = (const char*)b;
  return na > 0 && nb > 0 && x < y + nb && y < x + na;
}
// Bytes from the first element of a rows x cols matrix to its last one's end.
inline size_t span(i64 rows, i64 cols, i64 ld, size_t es) { return rows > 0 ? (size_t)((rows - 1) * ld + cols) * es : 0; }
constexpr i64 kMostElements = 1ll << 40;

inline int check_matrix(const void* p, int dtype, i64 rows, int cols, i64 ld) {
  if (!p || rows <= 0 || cols <= 0 || !dtype_ok(dtype)) return POETX_ERR_INVALID_ARG;
  if (ld < cols) return POETX_ERR_BAD_SHAPE;
  if (rows >= (1ll << 40) || ld >= kMostElements / rows) return POETX_ERR_UNSUPPORTED;
  return POETX_OK;
}

}  // namespace poetx
