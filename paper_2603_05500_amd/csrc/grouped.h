// Products of rows with their group's weight: what the kernels share.
#pragma once

#include "poetx_kernels.h"

namespace poetx {
namespace grouped {

// Which product.  FWD: Z = X W^T, INPUT: dX = dZ W, WEIGHT: dW = dZ^T X.
enum Dir { FWD = 0, INPUT = 1, WEIGHT = 2 };

// A call.  in: X (FWD, WEIGHT) or dZ (INPUT); in2: dZ (WEIGHT); w: the dense weight; out: Z, dX or dW.
struct Call {
  const void* in;
  const void* in2;
  const void* w;
  void* out;
  i64 ld_in, ld_in2, ld_out;
  const int32_t* offsets;
  i64 rows;
  int m, n, groups;
  int accumulate;
  int row_in = 0, row_in2 = 0;      // WEIGHT on the streams: elements that may be read of a row of in, in2, where that is more than m, n
};

// First row and end of a group.  Offsets are taken inside the tensor.  Where rows are computed none is taken below those before it: whatever they say, groups then share
// no row, so that every row has one result and the grids, which are made for that, hold every tile.  The weight gradient, whose groups have a result each, and what only has to know
// which weights may be needed go by a group's own two offsets (own_range), which are there sooner: in its place a check of the offsets before took up to 7 % of a weight
// gradient of short workgroups (100 groups of 513 x 1025, 9000 rows).
struct Range {
  int r0, r1;
};
__device__ __forceinline__ int offset_at(const int32_t* offsets, int g, i64 rows) {
  const int a = offsets[g], last = (int)rows;
  return a < 0 ? 0 : a > last ? last : a;
}
// Group g's by its own two offsets: no less than its rows.
__device__ __forceinline__ Range own_range(const int32_t* offsets, int g, i64 rows) {
  const int r0 = offset_at(offsets, g, rows), r1 = offset_at(offsets, g + 1, rows);
  return Range{r0, r1 < r0 ? r0 : r1};
}
// Group base + lane's two offsets, past the last group twice the last one; and its range from them.  end: the furthest end below base, 0 at first; moved on.
__device__ __forceinline__ Range lane_offsets(const int32_t* offsets, int groups, i64 rows, int base) {
  const int g = base + (int)(threadIdx.x & 63);
  return Range{offset_at(offsets, g < groups ? g : groups, rows), offset_at(offsets, g + 1 < groups ? g + 1 : groups, rows)};
}
__device__ __forceinline__ Range in_order(Range own, int& end) {
  if (__builtin_expect(__ballot(own.r1 < own.r0 || own.r0 < end) != 0, 0)) {
    const int lane = threadIdx.x & 63;
    int most = own.r0 > end ? own.r0 : end;
#pragma unroll 1
    for (int s = 1; s < 64; s *= 2) {
      const int o = __shfl_up(most, s);
      if (lane >= s && o > most) most = o;
    }
    own.r0 = most;
    own.r1 = own.r1 > most ? own.r1 : most;
  }
  end = __builtin_amdgcn_readlane(own.r1, 63);
  return own;
}
// The end of the last row that some group has, the same in every lane; the first one is the first offset.
__device__ inline int furthest_end(const int32_t* offsets, int groups, i64 rows) {
  const int last = offset_at(offsets, groups, rows);
  int most = last;
  for (int j = (int)(threadIdx.x & 63); j < groups; j += 64) {
    const int o = offset_at(offsets, j, rows);
    most = o > most ? o : most;
  }
  if (__builtin_expect(__ballot(most > last) == 0, 1)) return last;
#pragma unroll 1
  for (int s = 1; s < 64; s *= 2) {
    const int o = __shfl_xor(most, s);
    most = o > most ? o : most;
  }
  return __builtin_amdgcn_readfirstlane(most);
}
// Rows that weight gradients may sum over, from the first to the last, the same in every lane: those that some group's own two offsets name, which may lie below the first offset.
__device__ inline Range own_rows(const int32_t* offsets, int groups, i64 rows) {
  Range all{offset_at(offsets, 0, rows), offset_at(offsets, groups, rows)};
  int r0 = all.r0, r1 = all.r1;
  for (int g = (int)(threadIdx.x & 63); g < groups; g += 64) {
    const Range own = own_range(offsets, g, rows);
    if (own.r0 == own.r1) continue;
    r0 = own.r0 < r0 ? own.r0 : r0;
    r1 = own.r1 > r1 ? own.r1 : r1;
  }
  if (__builtin_expect(__ballot(r0 < all.r0 || r1 > all.r1) == 0, 1)) return all;
#pragma unroll 1
  for (int s = 1; s < 64; s *= 2) {
    const int a = __shfl_xor(r0, s), b = __shfl_xor(r1, s);
    r0 = a < r0 ? a : r0;
    r1 = b > r1 ? b : r1;
  }
  return Range{__builtin_amdgcn_readfirstlane(r0), __builtin_amdgcn_readfirstlane(r1)};
}

// Sum over a wave of the values of lower lanes and this one.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int o = __shfl_up(v, s);
    if (lane >= s) v += o;
  }
  return v;
}

// Tiles of `height` rows of all groups; a group's last tile may be short.
__device__ inline int count_row_tiles(const int32_t* offsets, int groups, i64 rows, int height) {
  int total = 0, end = 0;
  for (int base = 0; base < groups; base += 64) {
    const Range r = in_order(lane_offsets(offsets, groups, rows, base), end);
    total += __builtin_amdgcn_readlane(wave_scan((r.r1 - r.r0 + height - 1) / height), 63);
  }
  return total;
}
// Tile u of them (u below their number): its group, its first row and the group's end.
struct RowTile {
  int g, r0, r1;
};
__device__ inline RowTile find_row_tile(const int32_t* offsets, int groups, i64 rows, int height, int u) {
  int end = 0;
  for (int base = 0; base < groups; base += 64) {
    const Range r = in_order(lane_offsets(offsets, groups, rows, base), end);
    const int t = (r.r1 - r.r0 + height - 1) / height, sum = wave_scan(t), all = __builtin_amdgcn_readlane(sum, 63);
    if (u < all) {
      const int l = __builtin_ctzll(__ballot(sum > u));      // all > u: some lane has it
      const int before = __builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(t, l);
      return RowTile{base + l, __builtin_amdgcn_readlane(r.r0, l) + (u - before) * height, __builtin_amdgcn_readlane(r.r1, l)};
    }
    u -= all;
  }
  return RowTile{0, 0, 0};
}

// Row tiles that any offsets of so many groups and rows can have: groups share no row.
inline i64 most_row_tiles(i64 rows, int groups, int height) { return rows / height + (rows < groups ? rows : groups); }

// Workgroup bx of `total` that work: consecutive ones go to the 8 XCDs in turn, so that XCD's take contiguous runs of the work.
__device__ __forceinline__ int xcd_run(int bx, int total) {
  const int xcd = bx & 7, per = total >> 3, extra = total & 7;
  return xcd * per + (xcd < extra ? xcd : extra) + (bx >> 3);
}

// ---- which kernel ------------------------------------------------------------------------------------
enum Kernel { EDGE_32, EDGE_32_DEEP, EDGE_64, EDGE_128, STREAM_256, STREAM_256x128, STREAM_128, SINGLE_128, SINGLE_64, KERNELS };      // SINGLE: streams of fp32
// The one that a model of their times finds the fastest, from what one stage of its tile's contraction takes alone and how many tiles the chip works on at a time.
// scratch: bytes there are for the sums of a contraction split among workgroups; parts: what of them the plan takes.
struct Plan {
  Kernel kernel;
  int splits;
  size_t parts;
  double us;
};
Plan plan(int dtype, Dir dir, const Call& c, bool streams, size_t scratch);
// Output tiles of h x w that a call has, about.
double tiles_of(Dir dir, i64 rows, int m, int n, int groups, int h, int w);

// ---- launchers -----------------------------------------------------------------------------------
void edge_launch(int dtype, Dir dir, Kernel k, const Call& c, hipStream_t st);      // any shape (grouped_edge.hip)
// whole 16-byte vectors (grouped_stream.hip)
bool stream_supported(int dtype, Dir dir, const Call& c);
bool weight_stream_supported(int dtype, const Call& c);      // of operands in rows of whole vectors, whatever m and n, with scratch for what is not; c.out 16-byte aligned
void stream_launch(int dtype, Dir dir, const Plan& p, const Call& c, void* scratch, hipStream_t st);
// fp32 sums of a contraction's ranges, [split][rows][cols], added in order into c.out
void add_parts(int dtype, const void* parts, int splits, int cols, const Call& c, hipStream_t st);
// Z = X W^T as fp32 sums of the plan's ranges of the contraction, [split][rows][n]
void stream_sums(int dtype, const Plan& p, const Call& c, void* sums, hipStream_t st);
// Z = X W^T with X rounded to four bits on the way, W a 4-bit buffer
bool codes_supported(const poetx_grouped_desc* d, const void* Z, i64 ldz);
size_t codes_workspace_bytes(const poetx_grouped_desc* d);
void codes_launch(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, void* ws, hipStream_t st);

// Z = X W^T with W a 4-bit buffer, decoded on the way (grouped_values.hip): whole 16-byte vectors.  False where another way is the better one: the kernel for a handful of rows if `few`,
// otherwise the weight written out first if `whole`, the workspace holding it, with `scratch` bytes for its product.  ws: for sums of parts of the contraction.
bool values_supported(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Z, i64 ldz);
bool values_launch(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, bool few, bool whole, void* ws, size_t ws_bytes, size_t scratch,
                   hipStream_t st);

// the forward of a handful of rows per group (grouped_few.hip): any sizes, strides and alignments
enum Weight { DENSE_WEIGHT, VALUES_MX4, VALUES_STREAMED_MX4, CODES_MX4 };      // STREAMED: values_launch() takes the call; CODES: of X as well
bool few_supported(int dtype, Dir dir, i64 rows, int m, int n, int groups, Weight w);
double few_values_us(const poetx_grouped_desc* d);      // of few_values(), about
void few_dense(int dtype, const Call& c, hipStream_t st);
void few_values(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, hipStream_t st);      // 4-bit weight
void few_codes(const poetx_grouped_desc* d, const void* Xq, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, hipStream_t st);               // 4-bit rows too

}  // namespace grouped
}  // namespace poetx
