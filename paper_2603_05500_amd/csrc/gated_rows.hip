// The gated block's elementwise half: from G and U (as they were kept, or as sums of parts of the contraction) to H, what is kept, or the gradients dG, dU and H again.
//
// One pass: sixteen lanes take 128 columns of a row, eight each, of G, U and dH, so that 8-bit buffers come by whole units and every access of a wave is contiguous.
// Bound by bytes: 16384 x 14336 from eight bits, dG, dU and H in bf16, 403 to 420 us for 2.36 GB (5.7 TB/s; a large copy makes 5.1); 1001 x 1376 in fp32 9.2 us, of which 6.4 for the bytes.
#include "gated.h"

namespace poetx {
namespace gated {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int UPL = 2;      // units per sixteen lanes, their loads in flight together

struct RowsArgs {
  In in;
  Out out;
  const int32_t* offsets;
  int groups, n, upr;
  i64 rows;
};

template <class T, Source SRC, Mode MODE>
__global__ __launch_bounds__(256) void gated_rows_kernel(RowsArgs a, int block0) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + (int)blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  const i64 r0 = grouped::offset_at(a.offsets, 0, a.rows), r1 = grouped::furthest_end(a.offsets, a.groups, a.rows);
  const mx8::View qg = mx8::view(a.in.G, a.rows, a.n), qu = mx8::view(a.in.U, a.rows, a.n);      // MX8
  float g[UPL][8], u[UPL][8], dh[UPL][8];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 unit = first + 16 * p, at = unit / a.upr;
    const bool on = at >= r0 && at < r1;
    const i64 row = on ? at : 0;
    const int col = on ? (int)(unit - at * a.upr) * mx8::UNIT + 8 * lane : a.n;      // past the end: zeros, nothing is read
    if constexpr (SRC == MX8) {
      const i64 w = on ? unit : 0;      // buffers have whole units
      const u32x2 cg = *reinterpret_cast<const u32x2*>(qg.codes + w * mx8::UNIT + 8 * lane), cu = *reinterpret_cast<const u32x2*>(qu.codes + w * mx8::UNIT + 8 * lane);
      const int shift = 8 * (lane >> 2);
      mx8::values8(cg[0], cg[1], qg.scales[w] >> shift & 255, g[p]);
      mx8::values8(cu[0], cu[1], qu.scales[w] >> shift & 255, u[p]);
    } else if constexpr (SRC == SAME) {
      edge::load8((const T*)a.in.G + row * a.in.ld, col, a.n, g[p]);
      edge::load8((const T*)a.in.U + row * a.in.ld, col, a.n, u[p]);
    } else {
      const float* s = (const float*)a.in.G + row * 2 * a.n;
      edge::load8(s, col, a.n, g[p]);
      edge::load8(s + a.n, col, a.n, u[p]);
      for (int z = 1; z < a.in.splits; ++z) {      // in order
        s += a.rows * 2 * a.n;
        float x[8], y[8];
        edge::load8(s, col, a.n, x);
        edge::load8(s + a.n, col, a.n, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[p][e] += x[e], u[p][e] += y[e];
      }
    }
    if constexpr (MODE == BWD) edge::load8((const T*)a.out.dH + row * a.out.lddh, col, a.n, dh[p]);
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 unit = first + 16 * p, row = unit / a.upr;
    emit8<T, MODE>(a.out, a.rows, a.n, row, (int)(unit - row * a.upr) * mx8::UNIT + 8 * lane, row >= r0 && row < r1, g[p], u[p], dh[p]);
  }
}

}  // namespace

void rows_launch(int dtype, Source src, const In& in, const int32_t* offsets, int groups, i64 rows, int n, Mode mode, const Out& out, hipStream_t st) {
  const RowsArgs a{in, out, offsets, groups, n, mx8::units(n), rows};
  const i64 blocks = (rows * a.upr + 16 * UPL - 1) / (16 * UPL);
  auto go = [&](auto kern) { launch_in_rows(blocks, [&](int block0, unsigned count) { hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, a, block0); }); };
  auto typed = [&](auto zero) {
    typedef decltype(zero) T;
    if (src == SAME) go(gated_rows_kernel<T, SAME, BWD>);
    else if (src == MX8) go(gated_rows_kernel<T, MX8, BWD>);
    else if (mode == FWD) go(gated_rows_kernel<T, SUMS, FWD>);
    else if (mode == HOLD) go(gated_rows_kernel<T, SUMS, HOLD>);
    else if (mode == HOLD_MX8) go(gated_rows_kernel<T, SUMS, HOLD_MX8>);
    else go(gated_rows_kernel<T, SUMS, BWD>);
  };
  dtype == POETX_F32 ? typed(0.f) : typed((uint16_t)0);
}

}  // namespace gated
}  // namespace poetx
