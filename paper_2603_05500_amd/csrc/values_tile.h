// Which rows of a 4-bit weight a tile of a gated block loads (grouped_values.hip).  A group's weight has n rows of gate and n of up below them; the tile has `width` columns of H from
// n0 on, its first half of weight rows being gate's and its second half up's.  Rows are counted from row n0 of the group's gate.
#pragma once

#ifdef __HIP__
#define POETX_HOST_DEVICE __host__ __device__
#else
#define POETX_HOST_DEVICE
#endif

namespace poetx {
namespace values {

// row r of the tile's 2 width
POETX_HOST_DEVICE constexpr int gated_row(int r, int n, int width) { return r < width ? r : n - width + r; }
// How many rows the descriptors reach over: to the last of up that the tile has, so that no row of it reads behind the group's.  A tile behind column n, which only writes codes of
// zero past the columns, has none of up; with n below 32 it begins behind the group, and nothing is left to reach over.
POETX_HOST_DEVICE constexpr int gated_reach(int n, int n0, int width) {
  const int cols = n - n0 < width ? n - n0 : width;
  return n + cols > 0 ? n + cols : 0;
}

}  // namespace values
}  // namespace poetx
