// Grouped products of any sizes, strides and alignments, bf16 and fp32: the edge-handling matrix-core product, one output tile of one
// group per workgroup.  A workgroup finds its group from the offsets on the device; the grid has room for the most tiles that any offsets could
// give, and the workgroups beyond the actual number leave.  Short groups of wide operands are bound by the latency of their few stages, the rest by the loads' bounds checks:
// the streams take what is aligned and large enough to fill the chip.
#include "edge_gemm.h"
#include "grouped.h"

namespace poetx {
namespace grouped {
namespace {

template <class O, bool ADD>
struct Store {
  O* p;
  i64 ld;
  int rows, cols;
  __device__ void operator()(int, int, int row, int col, const float (&v)[8]) const {
    if (row >= rows || col >= cols) return;
    O* at = p + (i64)row * ld + col;
    const int n = cols - col;
    if constexpr (ADD) {
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = e < n ? v[e] + at[e] : 0.f;
      edge::store8(at, s, n);
    } else {
      edge::store8(at, v, n);
    }
  }
};

template <class T, class O, int TILE, int BK, int WG, int WAVES, Dir DIR, bool ADD>
__global__ __launch_bounds__(64 * WAVES) void grouped_edge_kernel(Call c, int tiles_y, int tiles_x, int first) {
  const int bx = first + (int)blockIdx.x;
  edge::Args g = {};
  Store<O, ADD> epi;
  const i64 weight = (i64)c.n * c.m;
  if constexpr (DIR == WEIGHT) {
    const int total = c.groups * tiles_y * tiles_x;
    const int id = xcd_run(bx, total);
    const int gr = id / (tiles_y * tiles_x), t = id % (tiles_y * tiles_x), i0 = t % tiles_y * TILE, j0 = t / tiles_y * TILE;
    const Range r = own_range(c.offsets, gr, c.rows);
    g.A = edge::Op{(const T*)c.in2 + (i64)r.r0 * c.ld_in2 + i0, c.ld_in2, 0, nullptr, r.r1 - r.r0, c.n - i0, 0, 0, 1};
    g.B = edge::Op{(const T*)c.in + (i64)r.r0 * c.ld_in + j0, c.ld_in, 0, nullptr, r.r1 - r.r0, c.m - j0, 0, 0, 1};
    g.stages = (r.r1 - r.r0 + BK - 1) / BK;
    epi = Store<O, ADD>{(O*)c.out + gr * weight + (i64)i0 * c.m + j0, c.m, c.n - i0, c.m - j0};
  } else {
    const int total = count_row_tiles(c.offsets, c.groups, c.rows, TILE) * tiles_x;
    if (bx >= total) return;
    const int id = xcd_run(bx, total);
    const RowTile rt = find_row_tile(c.offsets, c.groups, c.rows, TILE, id / tiles_x);
    const int j0 = id % tiles_x * TILE, K = DIR == FWD ? c.m : c.n, N = DIR == FWD ? c.n : c.m;
    g.A = edge::Op{(const T*)c.in + (i64)rt.r0 * c.ld_in, c.ld_in, 0, nullptr, rt.r1 - rt.r0, K, 0, 0, 1};
    const T* W = (const T*)c.w + rt.g * weight;
    if constexpr (DIR == FWD) g.B = edge::Op{W + (i64)j0 * c.m, c.m, 0, nullptr, N - j0, K, 0, 0, 1};
    else g.B = edge::Op{W + j0, c.m, 0, nullptr, K, N - j0, 0, 0, 1};
    g.stages = (K + BK - 1) / BK;
    epi = Store<O, ADD>{(O*)c.out + (i64)rt.r0 * c.ld_out + j0, c.ld_out, rt.r1 - rt.r0, N - j0};
  }
  g.tiles_m = g.tiles_n = g.batches = 1;
  g.stages_per_split = g.stages;
  edge::edge_product<T, TILE, TILE, BK, WG, WG, WAVES, DIR != WEIGHT, DIR == FWD, Store<O, ADD>, edge::BRANCHED>(g, epi, 0, 1, 0);
}

template <class T, class O, int TILE, int BK, int WG, int WAVES, Dir DIR, bool ADD>
void launch_tile(const Call& c, hipStream_t st) {
  using S = edge::Shape<T, TILE, TILE, BK, WG, WG, WAVES>;
  auto kern = grouped_edge_kernel<T, O, TILE, BK, WG, WAVES, DIR, ADD>;
  static const bool configured = edge::lds_limit((const void*)kern, S::LDS);
  (void)configured;
  const int ty = DIR == WEIGHT ? ceil_div(c.n, TILE) : 0, tx = ceil_div(DIR == FWD ? c.n : c.m, TILE);
  const i64 total = DIR == WEIGHT ? (i64)c.groups * ty * tx : most_row_tiles(c.rows, c.groups, TILE) * tx;
  launch_in_rows(total, [&](int first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(64 * WAVES), S::LDS, st, c, ty, tx, first);
  });
}

template <class T, class O, Dir DIR, bool ADD>
void launch_dir(Kernel k, const Call& c, hipStream_t st) {
  constexpr int D = 128 / (int)sizeof(T);
  if (k == EDGE_128) launch_tile<T, O, 128, D, 2, 4, DIR, ADD>(c, st);
  else if (k == EDGE_64) launch_tile<T, O, 64, D, 2, 4, DIR, ADD>(c, st);
  else if (k == EDGE_32) launch_tile<T, O, 32, 2 * D, 1, 4, DIR, ADD>(c, st);
  else launch_tile<T, O, 32, 8 * D, 1, 16, DIR, ADD>(c, st);
}

}  // namespace

void edge_launch(int dtype, Dir dir, Kernel k, const Call& c, hipStream_t st) {
  const bool f = dtype == POETX_F32;
  if (dir == FWD) f ? launch_dir<float, float, FWD, false>(k, c, st) : launch_dir<uint16_t, uint16_t, FWD, false>(k, c, st);
  else if (dir == INPUT) f ? launch_dir<float, float, INPUT, false>(k, c, st) : launch_dir<uint16_t, uint16_t, INPUT, false>(k, c, st);
  else if (c.accumulate) f ? launch_dir<float, float, WEIGHT, true>(k, c, st) : launch_dir<uint16_t, float, WEIGHT, true>(k, c, st);
  else f ? launch_dir<float, float, WEIGHT, false>(k, c, st) : launch_dir<uint16_t, float, WEIGHT, false>(k, c, st);
}

}  // namespace grouped
}  // namespace poetx
