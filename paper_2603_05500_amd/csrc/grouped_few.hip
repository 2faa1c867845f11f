// Forward products where groups have a handful of rows each (generation; a router's many experts): Z = X W_g^T as one read of the weights.
//
// What bounds it: the bytes of the weights, and their latency where a wave has a step or two.  A wave streams 16 RT rows of a weight straight into registers, as
// the first operand of 16 x 16 MFMAs whose second one is up to 16 NT rows of X; the waves of a workgroup split the contraction and meet in LDS.  The compiler decides how many of a step's
// loads go out before its first wait: 17 of 21 of (16 weight rows, 16 rows, 4 waves, 4 units) on 4-bit values, but 9 of 26 of (32,16,4,4), 16 of them of X, 9 to 12 of the dense ones.
// A lane's load is 16 bytes of one weight row, whatever they hold:
//   DENSE   8 bf16, one MFMA of depth 32
//   SINGLE  4 fp32, four MFMAs of depth 4, the groups of 16 lanes holding every fourth four
//   VALUES  32 codes with their scale, decoded in registers: four MFMAs of depth 32, in which the four groups of 16 lanes hold four different blocks of 32
//           (the order of a contraction is free as long as both operands keep it)
//   CODES   32 codes, and 32 of X: one scaled MFMA of depth 128
// A gated block's weight rows come in turn from gate and up, so that a tile has G and U of half as many columns of H.  One row by 2 x 14336 x 4096 in bf16 37 to 47 us (235 MB: 5.0 TB/s with
// weights from memory), eight rows, one each for eight of 64 groups of 2 x 1376 x 2048 in four bits 8.3.
#include "gated.h"

namespace poetx {
namespace grouped {
namespace {

using edge::load16;
using edge::u32x4;
using mm::bf16x8;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

enum Kind { DENSE, VALUES, CODES, SINGLE };

struct FewArgs {
  const void* X;            // rows; CODES: codes
  const uint8_t* xs;        // CODES: scales
  const void* W;            // rows of m, or codes
  const uint8_t* ws;
  void* Z;
  i64 ldx, ldz;             // elements; CODES: ldx is the bytes of a row of codes
  const int32_t* offsets;
  i64 rows;
  int m, n, groups, units, tiles_n;
};
// of a gated block (n: d_hidden)
struct GatedFewArgs : FewArgs {
  gated::Out block;
};

constexpr int NOT_GATED = gated::NONE;
template <int MODE>
using FewArgsOf = std::conditional_t<MODE == NOT_GATED, FewArgs, GatedFewArgs>;      // in one struct they cost every launch of a plain product 0.3 us of 7.1

// What a gated block makes of G and U of a tile, `part` being sums of NW waves [16 NT rows][8 RT pairs].  HOLD_MX8: RT = 4, the 32 columns of a block.
template <int RT, int NT, int NW, int MODE, class T>
__device__ __forceinline__ void gated_out(const GatedFewArgs& a, const RowTile& t, int rows, int h0, const float (&part)[NW][RT * NT * 256]) {
  const gated::Out& o = a.block;
  for (int i = threadIdx.x; i < RT * NT * 128; i += 64 * NW) {
    const int row = i / (8 * RT), col = h0 + i % (8 * RT);
    float g = 0.f, u = 0.f;
#pragma unroll
    for (int z = 0; z < NW; ++z) g += part[z][2 * i], u += part[z][2 * i + 1];
    const bool on = row < rows && col < a.n;
    const i64 at = t.r0 + row;
    if constexpr (MODE == gated::HOLD_MX8) {
      static_assert(MODE != gated::HOLD_MX8 || RT == 4, "a block of 32 columns to half a wave");
      auto keep = [&](float v, const void* Q) {
        uint32_t m = on ? __builtin_bit_cast(uint32_t, v) & 0x7fffffffu : 0;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
          const uint32_t other = __shfl_xor(m, s);
          m = other > m ? other : m;
        }
        const uint32_t sb = mx8::scale_byte(m);
        if (row >= rows) return;
        const mx8::View q = mx8::view(Q, a.rows, a.n);
        const i64 unit = at * mx8::units(a.n) + col / mx8::UNIT;
        q.codes[unit * mx8::UNIT + col % mx8::UNIT] = (uint8_t)(on && sb != 255 ? mx8::to_code(v, sb) & 255 : 0);
        if (i % 32 == 0) ((uint8_t*)q.scales)[unit * 4 + col % mx8::UNIT / 32] = (uint8_t)sb;
      };
      keep(g, o.G);
      keep(u, o.U);
    }
    if (!on) continue;
    auto put = [&](void* p, i64 ld, float v) {
      if constexpr (sizeof(T) == 4) ((float*)p)[at * ld + col] = v;
      else ((uint16_t*)p)[at * ld + col] = (uint16_t)mm::pack2_bf16(v, 0.f);
    };
    if constexpr (MODE == gated::HOLD) {
      put(o.G, o.ldgu, g);
      put(o.U, o.ldgu, u);
    }
    float v, d;
    gated::act_both(o.act, g, v, d);
    if constexpr (MODE == gated::BWD) {
      float dh;
      if constexpr (sizeof(T) == 4) dh = ((const float*)o.dH)[at * o.lddh + col];
      else dh = bf16_bits_to_float(((const uint16_t*)o.dH)[at * o.lddh + col]);
      put(o.G, o.ldgu, dh * u * d);
      put(o.U, o.ldgu, dh * v);
      if (!o.H) continue;
    }
    put(o.H, o.ldh, v * u);
  }
}

template <int RT, int NT, int NW, Kind KIND, int U, int MODE>
__global__ __launch_bounds__(64 * NW) void grouped_few_kernel(FewArgsOf<MODE> a, int first) {
  __shared__ float part[NW][RT * NT * 256];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = lane & 15, q = lane >> 4;
  const int bx = first + (int)blockIdx.x;
  const int rt_no = bx / a.tiles_n, n0 = bx % a.tiles_n * (MODE == NOT_GATED ? 16 * RT : 8 * RT);
  RowTile t;
  if (a.groups == 1) {
    const Range r = own_range(a.offsets, 0, a.rows);
    t = RowTile{0, r.r0 + rt_no * (16 * NT), r.r1};
  } else {
    t = find_row_tile(a.offsets, a.groups, a.rows, 16 * NT, rt_no);
  }
  const int rows = t.r1 - t.r0;      // 0 where there are fewer tiles
  if (rows <= 0) return;

  const int s0 = a.units * wave / NW, s1 = a.units * (wave + 1) / NW;
  // a row past the tile's end (of the weight) is some other one: what it gives goes nowhere
  i64 wrow[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    if constexpr (MODE == NOT_GATED) {
      const int row = n0 + 16 * r + x;
      wrow[r] = (i64)t.g * a.n + (row < a.n ? row : a.n - 1);
    } else {
      const int row = n0 + 8 * r + (x >> 1);
      wrow[r] = ((i64)t.g * 2 + (x & 1)) * a.n + (row < a.n ? row : a.n - 1);
    }
  }
  i64 xrow[NT];
#pragma unroll
  for (int c = 0; c < NT; ++c) xrow[c] = t.r0 + (16 * c + x < rows ? 16 * c + x : 0);

  floatx4 acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < NT; ++c) acc[r][c] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto steps = [&](int s, auto N_, auto WHOLE_) __attribute__((always_inline)) {      // that many units of 128; WHOLE: inside the rows
    constexpr int N = decltype(N_)::value;
    constexpr bool WHOLE = decltype(WHOLE_)::value;
    auto values = [&](const auto* row, int k) __attribute__((always_inline)) { return WHOLE ? load16(row + k) : edge::load_branched(row, k, a.m, true); };
    if constexpr (KIND == SINGLE) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {      // 64 of depth at a time
        u32x4 fw[N][4][RT], fx[N][4][NT];
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int k = (s + u) * 128 + 64 * h + 16 * p + 4 * q;
#pragma unroll
            for (int r = 0; r < RT; ++r) fw[u][p][r] = values((const float*)a.W + wrow[r] * a.m, k);
#pragma unroll
            for (int c = 0; c < NT; ++c) fx[u][p][c] = values((const float*)a.X + xrow[c] * a.ldx, k);
          }
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int c = 0; c < NT; ++c)
                  acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)fw[u][p][r][e]), __builtin_bit_cast(float, (uint32_t)fx[u][p][c][e]), acc[r][c], 0, 0, 0);
      }
    } else
    if constexpr (KIND == DENSE) {
      u32x4 fw[N][4][RT], fx[N][4][NT];
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int k = (s + u) * 128 + 32 * p + 8 * q;
#pragma unroll
          for (int r = 0; r < RT; ++r) fw[u][p][r] = values((const uint16_t*)a.W + wrow[r] * a.m, k);
#pragma unroll
          for (int c = 0; c < NT; ++c) fx[u][p][c] = values((const uint16_t*)a.X + xrow[c] * a.ldx, k);
        }
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < NT; ++c)
              acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[u][p][r]), __builtin_bit_cast(bf16x8, fx[u][p][c]), acc[r][c], 0, 0, 0);
    } else {
      u32x4 fw[N][RT];
      uint32_t sw[N][RT];
      // a row's scales of N units, of which a lane takes one byte each; four units' words are one load
      auto scales = [&](const uint8_t* p, auto put) __attribute__((always_inline)) {
        if constexpr (N == 4) {
          const u32x4 v = load16((const float*)p);
#pragma unroll
          for (int u = 0; u < 4; ++u) put(u, (v[u] >> (8 * q)) & 255);
        } else {
#pragma unroll
          for (int u = 0; u < N; ++u) put(u, p[4 * u + q]);
        }
      };
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          fw[u][r] = *reinterpret_cast<const u32x4*>((const uint8_t*)a.W + ((wrow[r] * a.units + s + u) * 4 + q) * 16);
        }
#pragma unroll
      for (int r = 0; r < RT; ++r) scales(a.ws + (wrow[r] * a.units + s) * 4, [&](int u, uint32_t b) { sw[u][r] = b; });
      if constexpr (KIND == VALUES) {
        u32x4 fx[N][4][NT];
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int c = 0; c < NT; ++c) fx[u][p][c] = values((const uint16_t*)a.X + xrow[c] * a.ldx, (s + u) * 128 + 32 * q + 8 * p);
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const float sc = mx4::scale_of(sw[u][r]);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              const bf16x8 w = __builtin_bit_cast(bf16x8, mx4::to_bf16(fw[u][r][p], sc));
#pragma unroll
              for (int c = 0; c < NT; ++c) acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, fx[u][p][c]), acc[r][c], 0, 0, 0);
            }
          }
      } else {
        u32x4 fx[N][NT];
        uint32_t sx[N][NT];
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int c = 0; c < NT; ++c) fx[u][c] = *reinterpret_cast<const u32x4*>((const uint8_t*)a.X + ((xrow[c] * a.units + s + u) * 4 + q) * 16);
#pragma unroll
        for (int c = 0; c < NT; ++c) scales(a.xs + (xrow[c] * a.units + s) * 4, [&](int u, uint32_t b) { sx[u][c] = b; });
        auto wide = [](const u32x4& v) { return intx8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < NT; ++c)
              acc[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(fw[u][r]), wide(fx[u][c]), acc[r][c], 4, 4, 0, (int)sw[u][r], 0, (int)sx[u][c]);
      }
    }
  };
  const int whole = KIND == CODES ? a.units : a.m / 128;
  int s = s0;
  for (; s + U <= s1 && s + U <= whole; s += U) steps(s, std::integral_constant<int, U>{}, std::true_type{});
  for (; s < s1 && s < whole; ++s) steps(s, std::integral_constant<int, 1>{}, std::true_type{});
  if constexpr (KIND != CODES) {
    if (s < s1) steps(s, std::integral_constant<int, 1>{}, std::false_type{});      // the last, short unit
  }

  // lane (row x of the tile, q), register e: weight row 4 q + e
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][((16 * c + x) * RT + r) * 16 + 4 * q + e] = acc[r][c][e];
  __syncthreads();
  if constexpr (MODE != NOT_GATED) return gated_out<RT, NT, NW, MODE, std::conditional_t<KIND == SINGLE, float, uint16_t>>(a, t, rows, n0, part);
  for (int i = tid; i < RT * NT * 256; i += 64 * NW) {
    const int row = i / (16 * RT), col = n0 + i % (16 * RT);
    float y = 0.f;
#pragma unroll
    for (int z = 0; z < NW; ++z) y += part[z][i];
    if (row < rows && col < a.n) {
      const i64 at = (t.r0 + row) * a.ldz + col;
      if constexpr (KIND == SINGLE) ((float*)a.Z)[at] = y;
      else ((uint16_t*)a.Z)[at] = (uint16_t)mm::pack2_bf16(y, 0.f);
    }
  }
}

template <int RT, int NT, int NW, Kind KIND, int U, int MODE = NOT_GATED>
void go(FewArgsOf<MODE> a, hipStream_t st) {
  a.tiles_n = MODE == NOT_GATED ? ceil_div(a.n, 16 * RT) : MODE == gated::HOLD_MX8 ? mx8::units(a.n) * 4 : ceil_div(a.n, 8 * RT);      // HOLD_MX8: codes past the last column are zeros
  const i64 total = (a.groups == 1 ? (a.rows + 16 * NT - 1) / (16 * NT) : most_row_tiles(a.rows, a.groups, 16 * NT)) * a.tiles_n;
  launch_in_rows(total, [&](int first, unsigned count) {
    hipLaunchKernelGGL((grouped_few_kernel<RT, NT, NW, KIND, U, MODE>), dim3(count), dim3(64 * NW), 0, st, a, first);
  });
}

// 16 x 16 tiles that groups of average size give
i64 small_tiles(i64 rows, int groups, int n) {
  const i64 live = rows < groups ? rows : groups, tiles = groups == 1 ? (rows + 15) / 16 : rows / 16 + live / 2;
  return (tiles > live ? tiles : live) * ((n + 15) / 16);
}

// Tiles of 16 x 16 where there are few in all, whatever the rows; otherwise as many rows of X as an average group has, and more weight rows per wave, as each wave reads its rows of X
// anew.  us, by (weight rows, rows of X, waves, units of a step), weights from memory:
//   4 bits:  4096 x 4096, 1 row (16,16,4,4) 4.1  (32,16,4,4) 6.0; 16 rows 6.8, 8.2; 14336 x 4096, 1 row (16,16,4,4) 11.2  (32,16,4,4) 9.9  (64,16,8,4) 11.0; 16 rows 21.6, 14.6, 12.5;
//            eight of 64 experts of 1376 x 2048 a row each 5.8, 6.1, 7.4; all of them with 8 each 45.6, 32.6, 35.8; 14336 x 4096, 32 rows (64,32,4,1) 18.6  (64,64,4,1) 22.7;
//            1024 x 4096, 64 rows (16,16,4,4) 6.8  (64,64,4,1) 25.8; 4096 x 4096, 128 rows (16,16,4,4) 39  (64,32,4,1) 17.9  (64,64,4,1) 26.7; eight experts, 512 rows 32.9, 19.4, 23.6
//   bf16:    14336 x 4096, 1 row (16,16,4,4) 23.2  (64,16,4,2) 24.9; 16 rows 35.3, 27.2; the experts 10.2, 11.4; with 8 rows each 81.0, 75.6
template <Kind KIND>
void pick(const FewArgs& a, hipStream_t st) {
  const i64 live = a.rows < a.groups ? a.rows : a.groups, mean = (a.rows + live - 1) / live, tiles = small_tiles(a.rows, a.groups, a.n);
  if (tiles <= (KIND == SINGLE ? 1024 : 768)) return go<1, 1, 4, KIND, KIND == SINGLE ? 1 : 4>(a, st);
  if constexpr (KIND == SINGLE) return go<2, 2, 4, KIND, 1>(a, st);
  else if constexpr (KIND == DENSE) tiles <= 1024 && mean <= 8 ? go<1, 1, 4, KIND, 4>(a, st) : go<4, 1, 4, KIND, 2>(a, st);
  else if (mean <= 8) go<2, 1, 4, KIND, 4>(a, st);
  else if (mean <= 16) go<4, 1, 8, KIND, 4>(a, st);
  else if (mean <= 32 || tiles < 512 * 16) go<4, 2, 4, KIND, 1>(a, st);
  else go<4, 4, 4, KIND, 1>(a, st);
}

// a gated block: of twice as many weight rows
template <Kind KIND, int MODE>
void pick_gated(const GatedFewArgs& a, hipStream_t st) {
  const i64 live = a.rows < a.groups ? a.rows : a.groups, mean = (a.rows + live - 1) / live, tiles = small_tiles(a.rows, a.groups, 2 * a.n);
  if constexpr (MODE != gated::HOLD_MX8) {
    if (tiles <= (KIND == SINGLE ? 1024 : 768)) return go<1, 1, 4, KIND, KIND == SINGLE ? 1 : 4, MODE>(a, st);
  }
  if constexpr (KIND == SINGLE) {
    if constexpr (MODE == gated::HOLD_MX8) return go<4, 1, 4, KIND, 1, MODE>(a, st);
    else return go<2, 2, 4, KIND, 1, MODE>(a, st);
  } else if constexpr (KIND == DENSE) {
    if constexpr (MODE != gated::HOLD_MX8) {
      if (tiles <= 1024 && mean <= 8) return go<1, 1, 4, KIND, 4, MODE>(a, st);
    }
    return go<4, 1, 4, KIND, 2, MODE>(a, st);
  } else {
    if constexpr (MODE != gated::HOLD_MX8) {
      if (mean <= 8) return go<2, 1, 4, KIND, 4, MODE>(a, st);
    }
    if (mean <= 16) return go<4, 1, 8, KIND, 4, MODE>(a, st);
    if (mean <= 32 || tiles < 512 * 16) return go<4, 2, 4, KIND, 1, MODE>(a, st);
    go<4, 4, 4, KIND, 1, MODE>(a, st);
  }
}

}  // namespace

// Where it pays: up to so many rows per group, or few tiles in all.  us, these / the streams and edge kernels: bf16 64 experts of 1376 x 2048 with 8 rows each 76 / 86, 32 each 101 / 91;
// both in four bits, 14336 x 4096, 16 rows 11 / 24, 64 experts with 32 rows each 51 / 37, 256 x 8192, four with 30 in all 9 / 33;
// a 4-bit weight against the stream that decodes it: 14336 x 4096, 32 rows 18.3 / 20.6, 64 rows 33 / 21, 4096 x 4096, 64 rows 17.0 / 20.0, 64 experts with 16 rows each 50 / 33;
// against its values in the workspace, for what that stream does not take: 14336 x 4096, 128 rows 49 / 66, 64 experts with 64 rows each 96 / 194.
// few tiles: bf16 1024 x 4096, 64 rows 9.5 / 13.8, 128 rows 16.5 / 14.6, 1024 x 1024, 128 rows 5.6 / 7.0; fp32 128 x 1749, 179 rows 7.4 / 32, 1024 x 2048, 256 rows 19 / 38.
bool few_supported(int dtype, Dir dir, i64 rows, int m, int n, int groups, Weight w) {
  if (dir != FWD) return false;
  const i64 most = dtype == POETX_F32 ? 4 : w == VALUES_MX4 ? 128 : 16;
  const i64 few = dtype == POETX_F32 ? 1024 : w == VALUES_STREAMED_MX4 ? 2048 : w != DENSE_WEIGHT ? 768 : m <= 2048 ? 640 : 320;
  return rows <= most * groups || small_tiles(rows, groups, n) <= few;
}
// The variants of pick() for VALUES: 4500 calls that few_supported() gives them, 12 % off on average.
double few_values_us(const poetx_grouped_desc* d) {
  const i64 live = d->rows < d->groups ? d->rows : d->groups, mean = (d->rows + live - 1) / live, tiles = small_tiles(d->rows, d->groups, d->d_out);
  const int units = mx4::units(d->d_in);
  if (tiles <= 768) return 2.74 + units * (0.0668 + 2.91e-4 * tiles);
  if (mean <= 8) return 3.15 + units * (0.0307 + 2.06e-4 * tiles);
  if (mean <= 16) return 3.49 + units * (0.0202 + 3.45e-4 * tiles);
  return 3.61 + units * (0.248 + 1.01e-4 * tiles);
}
void few_dense(int dtype, const Call& c, hipStream_t st) {
  const FewArgs a{c.in, nullptr, c.w, nullptr, c.out, c.ld_in, c.ld_out, c.offsets, c.rows, c.m, c.n, c.groups, (c.m + 127) / 128, 0};
  dtype == POETX_F32 ? pick<SINGLE>(a, st) : pick<DENSE>(a, st);
}
void few_values(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, hipStream_t st) {
  const mx4::View w = mx4::view(Wq, (i64)d->groups * d->d_out, d->d_in);
  pick<VALUES>(FewArgs{X, nullptr, w.codes, w.scales, Z, ldx, ldz, offsets, d->rows, d->d_in, d->d_out, d->groups, mx4::units(d->d_in), 0}, st);
}
void few_codes(const poetx_grouped_desc* d, const void* Xq, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, hipStream_t st) {
  const mx4::View w = mx4::view(Wq, (i64)d->groups * d->d_out, d->d_in), x = mx4::view(Xq, d->rows, d->d_in);
  pick<CODES>(FewArgs{x.codes, x.scales, w.codes, w.scales, Z, 0, ldz, offsets, d->rows, d->d_in, d->d_out, d->groups, mx4::units(d->d_in), 0}, st);
}

}  // namespace grouped

namespace gated {

// `four`: W is a 4-bit buffer
void few_launch(int dtype, bool four, const Call& c, hipStream_t st) {
  using namespace grouped;
  GatedFewArgs a{{c.X, nullptr, c.W, nullptr, nullptr, c.ldx, 0, c.offsets, c.rows, c.m, c.n, c.groups, (c.m + 127) / 128, 0}, c.out};
  auto typed = [&](auto MODE_) {
    constexpr int MODE = decltype(MODE_)::value;
    if (four) {
      const mx4::View w = mx4::view(c.W, 2 * (i64)c.groups * c.n, c.m);
      a.W = w.codes;
      a.ws = w.scales;
      pick_gated<VALUES, MODE>(a, st);
    } else {
      dtype == POETX_F32 ? pick_gated<SINGLE, MODE>(a, st) : pick_gated<DENSE, MODE>(a, st);
    }
  };
  if (c.mode == FWD) typed(std::integral_constant<int, FWD>{});
  else if (c.mode == HOLD) typed(std::integral_constant<int, HOLD>{});
  else if (c.mode == HOLD_MX8) typed(std::integral_constant<int, HOLD_MX8>{});
  else typed(std::integral_constant<int, BWD>{});
}

}  // namespace gated
}  // namespace poetx
