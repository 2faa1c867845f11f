// The gated block for any sizes, strides and alignments, bf16 and fp32: the edge-handling product over rows of gate and up in turn, one tile of H of one group per
// workgroup, as the grouped edge products.  A lane gets eight neighbouring columns of a row, which are G and U of four elements.  Bound, as they are, by the latency of
// the stages of short or narrow products and by the loads' bounds checks of large ones (1967 rows over 11 groups of 2 x 1280 x 4142, whose weights would take as long to lay anew for a stream, 198 us, 0.21 PFLOP/s).
#include "gated.h"

namespace poetx {
namespace gated {
namespace {

typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// four neighbouring elements, of which n exist
__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4], int n) {
  const uint32_t a = mm::pack2_bf16(v[0], v[1]), b = mm::pack2_bf16(v[2], v[3]);
  if (n >= 4) {
    *reinterpret_cast<u32x2_a2*>(p) = u32x2_a2{a, b};
  } else {
    if (n > 0) p[0] = (uint16_t)a;
    if (n > 1) p[1] = (uint16_t)(a >> 16);
    if (n > 2) p[2] = (uint16_t)b;
  }
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4], int n) {
  if (n >= 4) *reinterpret_cast<f32x4_a4*>(p) = f32x4_a4{v[0], v[1], v[2], v[3]};
  else
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = v[e];
}
template <class T>
__device__ __forceinline__ void load4(const T* p, float (&v)[4], int n) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 4) v[e] = e < n ? p[e] : 0.f;
    else v[e] = e < n ? bf16_bits_to_float(p[e]) : 0.f;
  }
}

template <class T, Mode MODE>
struct Epilogue {
  Out o;
  i64 first;          // of the tile's rows
  i64 all_rows;
  int rows, h0, n;    // of the tile's rows; its first column; columns
  __device__ void operator()(int, int, int row, int col2, const float (&v)[8]) const {
    const int col = h0 + col2 / 2, left = row < rows ? n - col : 0;
    const i64 at = first + row;
    float g[4] = {v[0], v[2], v[4], v[6]}, u[4] = {v[1], v[3], v[5], v[7]}, h[4];
    if constexpr (MODE == HOLD_MX8) {      // eight lanes have a block of 32 columns
      auto keep = [&](const float (&z)[4], const void* Q) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t b = e < left ? __builtin_bit_cast(uint32_t, z[e]) & 0x7fffffffu : 0;
          m = b > m ? b : m;
        }
#pragma unroll
        for (int s = 1; s < 8; s *= 2) {
          const uint32_t other = __shfl_xor(m, s);
          m = other > m ? other : m;
        }
        if (row >= rows) return;
        const uint32_t sb = mx8::scale_byte(m);
        const mx8::View q = mx8::view(Q, all_rows, n);
        const i64 unit = at * mx8::units(n) + col / mx8::UNIT;
        *reinterpret_cast<uint32_t*>(q.codes + unit * mx8::UNIT + col % mx8::UNIT) =
            mx8::to_codes4(left > 0 ? z[0] : 0.f, left > 1 ? z[1] : 0.f, left > 2 ? z[2] : 0.f, left > 3 ? z[3] : 0.f, sb);
        if (col % 32 == 0) ((uint8_t*)q.scales)[unit * 4 + col % mx8::UNIT / 32] = (uint8_t)sb;
      };
      keep(g, o.G);
      keep(u, o.U);
    }
    if (left <= 0) return;
    if constexpr (MODE == HOLD) {
      store4((T*)o.G + at * o.ldgu + col, g, left);
      store4((T*)o.U + at * o.ldgu + col, u, left);
    }
    if constexpr (MODE == BWD) {
      float dh[4];
      load4((const T*)o.dH + at * o.lddh + col, dh, left);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float a, d;
        act_both(o.act, g[e], a, d);
        h[e] = a * u[e];
        g[e] = dh[e] * u[e] * d;
        u[e] = dh[e] * a;
      }
      store4((T*)o.G + at * o.ldgu + col, g, left);
      store4((T*)o.U + at * o.ldgu + col, u, left);
      if (!o.H) return;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = act_value(o.act, g[e]) * u[e];
    }
    store4((T*)o.H + at * o.ldh + col, h, left);
  }
};

template <class T, int BM, int BN, int BK, int WGM, int WGN, int WAVES, Mode MODE>
__global__ __launch_bounds__(64 * WAVES) void gated_edge_kernel(Call c, int tiles_x, int first) {
  const int bx = first + (int)blockIdx.x;
  const int total = grouped::count_row_tiles(c.offsets, c.groups, c.rows, BM) * tiles_x;
  if (bx >= total) return;
  const int id = grouped::xcd_run(bx, total), h0 = id % tiles_x * (BN / 2);
  const grouped::RowTile rt = grouped::find_row_tile(c.offsets, c.groups, c.rows, BM, id / tiles_x);
  const i64 half = (i64)c.n * c.m;
  edge::Args g = {};
  g.A = edge::Op{(const T*)c.X + (i64)rt.r0 * c.ldx, c.ldx, 0, nullptr, rt.r1 - rt.r0, c.m, 0, 0, 1};
  g.B = edge::Op{(const T*)c.W + 2 * rt.g * half + (i64)h0 * c.m, c.m, 0, nullptr, 2 * (c.n - h0), c.m, 0, 0, half};
  g.stages = g.stages_per_split = (c.m + BK - 1) / BK;
  g.tiles_m = g.tiles_n = g.batches = 1;
  const Epilogue<T, MODE> epi{c.out, rt.r0, c.rows, rt.r1 - rt.r0, h0, c.n};
  edge::edge_product<T, BM, BN, BK, WGM, WGN, WAVES, true, true, Epilogue<T, MODE>, edge::PAIRED>(g, epi, 0, 1, 0);
}

template <class T, int BM, int BN, int BK, int WGM, int WGN, int WAVES, Mode MODE>
void go(const Call& c, hipStream_t st) {
  using S = edge::Shape<T, BM, BN, BK, WGM, WGN, WAVES>;
  static_assert(MODE != HOLD_MX8 || S::TN == 2, "a wave's columns are whole blocks");
  auto kern = gated_edge_kernel<T, BM, BN, BK, WGM, WGN, WAVES, MODE>;
  static const bool configured = edge::lds_limit((const void*)kern, S::LDS);
  (void)configured;
  const int tx = ceil_div(MODE == HOLD_MX8 ? mx8::units(c.n) * mx8::UNIT : c.n, BN / 2);      // codes past the last column are zeros
  launch_in_rows(grouped::most_row_tiles(c.rows, c.groups, BM) * tx, [&](int first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(64 * WAVES), S::LDS, st, c, tx, first);
  });
}

template <class T, Mode MODE>
void pick(grouped::Kernel k, const Call& c, hipStream_t st) {
  constexpr int D = 128 / (int)sizeof(T);
  // What plan() gives forward products: 64 x 64, 32 x 32, and in bf16 32 x 32 with deep stages.  HOLD_MX8: a wave's columns are whole blocks.
  if constexpr (MODE == HOLD_MX8) {
    k == grouped::EDGE_64 ? go<T, 64, 64, D, 2, 1, 4, MODE>(c, st) : go<T, 32, 64, 2 * D, 1, 1, 4, MODE>(c, st);
  } else {
    if constexpr (sizeof(T) == 2) {
      if (k == grouped::EDGE_32_DEEP) return go<T, 32, 32, 8 * D, 1, 1, 16, MODE>(c, st);
    }
    k == grouped::EDGE_32 ? go<T, 32, 32, 2 * D, 1, 1, 4, MODE>(c, st) : go<T, 64, 64, D, 2, 2, 4, MODE>(c, st);
  }
}

}  // namespace

void edge_launch(int dtype, grouped::Kernel k, const Call& c, hipStream_t st) {
  auto typed = [&](auto zero) {
    typedef decltype(zero) T;
    if (c.mode == FWD) pick<T, FWD>(k, c, st);
    else if (c.mode == HOLD) pick<T, HOLD>(k, c, st);
    else if (c.mode == HOLD_MX8) pick<T, HOLD_MX8>(k, c, st);
    else pick<T, BWD>(k, c, st);
  };
  dtype == POETX_F32 ? typed(0.f) : typed((uint16_t)0);
}

}  // namespace gated
}  // namespace poetx
