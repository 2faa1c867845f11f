// Forward products of bf16 rows with a 4-bit weight, some tens to some thousands of rows: Z = X W_g^T, the weight decoded between LDS and the multiplication.
//
// A stage is a unit of 128 columns: 256 bytes of a row of X, 64 bytes of codes and a word of scales of a row of W, by direct-to-LDS loads into a ring of NS stages, whose
// descriptors end where the operands do.  It is multiplied in four steps of 32.  As the order of a contraction is free, the group q of 16 lanes takes block q of the unit, step p of it
// elements 8 p .. 8 p + 7: a lane reads its 16 bytes of codes and its one scale of a row once per unit, and decodes a word of codes per step, a step ahead of its multiplication.
// One barrier per unit, before its last step: by then every wave holds what is left of the unit in registers, and the next one has landed.
//
// What bounds it: the instructions of one wave per SIMD, 4.2 beside every multiplication that takes 16 cycles (the conversions alone 8 %, the loads of X 10 %), so the descriptors move on
// a part per multiplication and the scales are converted when they are used (14336 x 4096, 128 rows, 128 x 128: 34 us with both in one place, 29 so; 40 with the accumulators left to the
// compiler).  4096 rows over 8 groups of 8192 x 4096 266 us (1.03 PFLOP/s; 426 by writing the weight out first).  The smallest tile leaves room for a second workgroup on a CU.
#include "grouped_stream.h"
#include "values_tile.h"

namespace poetx {
namespace grouped {
namespace {

struct ValuesArgs {
  const uint16_t* X;
  i64 ldx;
  const uint8_t* codes;
  const uint8_t* scales;
  uint16_t* Z;
  i64 ldz;
  const int32_t* offsets;
  i64 rows;
  int m, n, groups, units, tiles_n;
  int splits;      // PARTS: ranges of the contraction, whose fp32 sums go to parts, [split][rows][n]
  float* parts;
};
// MODE: of a gated block (n: d_hidden)
struct GatedValuesArgs : ValuesArgs {
  gated::Out block;
};
template <int MODE>
using ValuesArgsOf = std::conditional_t<MODE == NOT_GATED, ValuesArgs, GatedValuesArgs>;

// MODE: a gated block (14187 rows over 3 groups of 2 x 544 x 2336 107 us, 134 with the weight written out first), a tile's first half of columns being gate's and its second half up's of as many columns of H.
template <int BM, int BN, int NS, bool PARTS, int MODE>
__global__ __launch_bounds__(256) void grouped_values_kernel(ValuesArgsOf<MODE> g, int first) {
  constexpr int A_BYTES = BM * 256, B_BYTES = BN * 64, STAGE_BYTES = A_BYTES + B_BYTES + BN * 4;
  constexpr int IPWA = BM / 16, IPWB = BN / 64, LPU = IPWA + IPWB + 1, TM = BM / 32, TN = BN / 32, MF = TM * TN;
  constexpr bool GATED = MODE != NOT_GATED;
  constexpr int BW = GATED ? BN / 2 : BN;
  constexpr int OUT_LD = BN + 8;      // elements of a row of the tile on its way out: 16-byte chunks of 8 rows in different banks
  typedef typename std::conditional<PARTS || GATED, float, uint16_t>::type Out;
  static_assert(BN <= 256 && IPWA % 2 == 0 && (NS - 1) * LPU < 64 && NS >= 3 && BM * OUT_LD * (int)sizeof(Out) <= NS * STAGE_BYTES, "values tile");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tiles = count_row_tiles(g.offsets, g.groups, g.rows, BM) * g.tiles_n, total = PARTS ? tiles * g.splits : tiles;
  const int bx = first + (int)blockIdx.x;
  if (bx >= total) return;
  int id = xcd_run(bx, total);
  const int split = PARTS ? id / tiles : 0, u0 = PARTS ? g.units * split / g.splits : 0, u1 = PARTS ? g.units * (split + 1) / g.splits : g.units;
  id -= split * tiles;
  const RowTile t = find_row_tile(g.offsets, g.groups, g.rows, BM, id / g.tiles_n);
  const int n0 = id % g.tiles_n * BW;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1, q4 = lane >> 4, li = lane & 15;
  const int rows = t.r1 - t.r0 < BM ? t.r1 - t.r0 : BM, cols = g.n - n0 < BW ? g.n - n0 : BW;
  auto weight_row = [&](int r) __attribute__((always_inline)) { return GATED ? values::gated_row(r, g.n, BW) : r; };      // from the tile's first one
  const int wrows = GATED ? values::gated_reach(g.n, n0, BW) : cols;      // that the descriptors reach over

  // ---- loads: X a row's 16 chunks in the order chunk ^ row % 8, so that 8 rows' same chunk lies in different banks
  const int lda = 2 * (int)g.ldx, ldb = g.units * 64;
  uint32_t voffA[IPWA], voffB[IPWB];
  uint64_t past_end[2];      // lanes whose chunk lies behind the row in a short last unit (X only: codes are padded)
#pragma unroll
  for (int i = 0; i < IPWA; ++i) {
    const int r = (wave * IPWA + i) * 4 + q4;
    voffA[i] = (uint32_t)(r * lda + 16 * (li ^ (r & 7)));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) past_end[i] = __ballot(8 * (li ^ (4 * i + q4)) >= g.m % mx4::UNIT);
#pragma unroll
  for (int i = 0; i < IPWB; ++i) {
    const int slot = (wave * IPWB + i) * 64 + lane, r = slot >> 2;
    voffB[i] = (uint32_t)(weight_row(r) * ldb + 16 * dense::xk16_chunk(slot & 3, r));
  }
  const int srow = (wave * 64) % BN;      // BN < 256: some waves bring the same scales
  const uint32_t voffS = (uint32_t)(weight_row(srow + lane) * g.units * 4);
  const i64 wrow = (i64)t.g * (GATED ? 2 * g.n : g.n) + n0;
  // an operand's descriptor at the unit in issue, and the bytes from there on
  u32x4 ra{}, rb{}, rs{};
  int left_a = uniform((rows - 1) * lda + 2 * g.m - 256 * u0), left_b = uniform(wrows * ldb - 64 * u0), left_s = uniform((wrows * g.units - u0) * 4);
  auto start = [&](u32x4& r, const void* at, int left) __attribute__((always_inline)) {
    r = u32x4{(uint32_t)uniform((int)(uint64_t)at), (uint32_t)uniform((int)((uint64_t)at >> 32)) & 0xffffu, (uint32_t)left, 0x00020000u};
  };
  start(ra, g.X + (i64)t.r0 * g.ldx + u0 * mx4::UNIT, left_a);
  start(rb, g.codes + wrow * ldb + u0 * 64, left_b);
  start(rs, g.scales + (wrow * g.units + u0) * 4, left_s);
  const int short_unit = g.m % mx4::UNIT ? g.units - 1 : -1;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  uint32_t stage = lds_base;
  int iu = u0;
  uint64_t masked[2];
  auto mask = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) masked[i] = iu == short_unit ? past_end[i] : 0;
  };
  mask();
  auto issue = [&](int i) __attribute__((always_inline)) {      // load i of the unit
    if (i < IPWA) {
      dma16b_but(masked[i & 1], ra, voffA[i], stage + (wave * IPWA + i) * 1024);
    } else if (i < IPWA + IPWB) {
      dma16b(rb, voffB[i - IPWA], stage + A_BYTES + (wave * IPWB + i - IPWA) * 1024);
    } else {
      dma4b(rs, voffS, stage + A_BYTES + B_BYTES + srow * 4);
    }
  };
  // on to the next unit, a little at a time; behind the last one the descriptors are empty
  auto step = [&](u32x4& r, int& left, int bytes) __attribute__((always_inline)) {
    const uint64_t at = ((uint64_t)r[1] << 32 | r[0]) + bytes;
    left = iu < u1 ? left - bytes : 0;
    r[0] = (uint32_t)at;
    r[1] = (uint32_t)(at >> 32);
    r[2] = left > 0 ? left : 0;
  };
  auto advance = [&](int part) __attribute__((always_inline)) {
    if (part == 0) {
      ++iu;
      stage = stage == lds_base + (NS - 1) * STAGE_BYTES ? lds_base : stage + STAGE_BYTES;
    }
    if (part == 1) step(ra, left_a, 256);
    if (part == 2) step(rb, left_b, 64);
    if (part == 3) step(rs, left_s, 4);
    if (part == 4) mask();
  };

  // ---- fragments
  const int fragA = (wm * (BM / 2) + li) * 256, fragB = A_BYTES + (wn * (BN / 2) + li) * 64 + 16 * dense::xk16_chunk(q4, li), fragS = A_BYTES + B_BYTES + (wn * (BN / 2) + li) * 4 + q4;
  u32x4 x[2][TM], w[2][TN], code[TN];
  uint32_t byte[TN];
  float scale[TN];
  auto load_x = [&](const char* st, int p, int a) __attribute__((always_inline)) {
    x[p & 1][a] = *reinterpret_cast<const u32x4*>(st + fragA + a * 4096 + 16 * ((4 * q4 + p) ^ (li & 7)));
  };
  auto load_w = [&](const char* st, int b) __attribute__((always_inline)) {
    code[b] = *reinterpret_cast<const u32x4*>(st + fragB + b * 1024);
    byte[b] = *reinterpret_cast<const uint8_t*>(st + fragS + b * 64);
  };
  floatx4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};

  constexpr int Q = (LPU + 3) / 4;      // loads of a step; the first of a unit's go out in the last step of the one whose place it takes
#pragma unroll 1
  for (int u = 0; u < NS - 1; ++u) {
#pragma unroll
    for (int i = 0; i < LPU; ++i) issue(i);
#pragma unroll
    for (int i = 0; i < 5; ++i) advance(i);
  }
#pragma unroll
  for (int i = 0; i < Q; ++i) issue(i);
  mm::wait_vmcnt_and_barrier<(NS - 2) * LPU + Q>();
#pragma unroll
  for (int a = 0; a < TM; ++a) load_x(lds, 0, a);
#pragma unroll
  for (int b = 0; b < TN; ++b) {
    load_w(lds, b);
    scale[b] = mx4::scale_of(byte[b]);
    w[0][b] = mx4::to_bf16(code[b][0], scale[b]);
  }
  int slot = 0;
  for (int u = u0; u < u1; ++u) {
    in_turn(std::make_integer_sequence<int, 4>{}, [&](auto P) __attribute__((always_inline)) {
      constexpr int p = decltype(P)::value;
      if constexpr (p == 3) {
        mm::wait_all_reads_and_barrier<(NS - 2) * LPU>();
        slot = slot + 1 == NS ? 0 : slot + 1;
      }
      const char* st = lds + slot * STAGE_BYTES;
      in_turn(std::make_integer_sequence<int, MF>{}, [&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value, a = i % TM, b = i / TM;
        dense::mfma16(acc[a][b], __builtin_bit_cast(bf16x8, w[p & 1][b]), __builtin_bit_cast(bf16x8, x[p & 1][a]));
        // the next step's operands: its codes first where they are the next unit's, and decoded late
        constexpr int LW = p == 3 ? TN : 0, from = p == 3 ? MF / 2 : 0;
        if constexpr (i < LW) load_w(st, i);
        else if constexpr (i < LW + TM) load_x(st, (p + 1) & 3, i - LW);
        // the codes' words of two values, as evenly as they come
        constexpr int c0 = i < from ? 0 : (i - from) * 4 * TN / (MF - from), c1 = i < from ? 0 : (i + 1 - from) * 4 * TN / (MF - from);
        in_turn(std::make_integer_sequence<int, c1 - c0>{}, [&](auto J) __attribute__((always_inline)) {
          constexpr int c = c0 + decltype(J)::value;
          if constexpr (p == 3 && c % 4 == 0) scale[c / 4] = mx4::scale_of(byte[c / 4]);
          w[(p + 1) & 1][c / 4][c % 4] = mx4::to_bf16x2<c % 4>(code[c / 4][(p + 1) & 3], scale[c / 4]);
        });
        constexpr int at = (p == 3 ? 0 : p + 1) * Q, D = MF / Q;
        if constexpr (i % D == D / 2 && i / D < Q && at + i / D < LPU) issue(at + i / D);
        if constexpr (p == 2 && i >= MF - 5) advance(i - (MF - 5));      // the last load is out
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  }

  asm volatile("s_nop 15\n\ts_nop 3");      // the last products' results
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) asm volatile("" : "+a"(acc[a][b]));
  // ---- out through LDS, so that every instruction writes whole lines
  mm::wait_vmcnt_and_barrier<0>();      // no load is left, and every wave has read its last fragments
  Out* out = (Out*)lds;
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      Out* at = out + (wm * (BM / 2) + a * 16 + li) * OUT_LD + wn * (BN / 2) + b * 16 + 4 * q4;
      if constexpr (PARTS || GATED) *reinterpret_cast<floatx4*>(at) = acc[a][b];
      else *reinterpret_cast<u32x2*>(at) = u32x2{mm::pack2_bf16(acc[a][b][0], acc[a][b][1]), mm::pack2_bf16(acc[a][b][2], acc[a][b][3])};
    }
  __syncthreads();
  if constexpr (GATED) {
    for (int i = tid; i < BM * BW / 8; i += 256) {
      const int row = i / (BW / 8), col = i % (BW / 8) * 8;
      const bool on = row < rows;
      float G[8], U[8], dh[8] = {};
      const float* at = (const float*)out + row * OUT_LD + col;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const floatx4 x = *reinterpret_cast<const floatx4*>(at + 4 * h), y = *reinterpret_cast<const floatx4*>(at + BW + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) G[4 * h + e] = x[e], U[4 * h + e] = y[e];
      }
      if constexpr (MODE == gated::BWD) edge::load8((const uint16_t*)g.block.dH + (on ? t.r0 + row : t.r0) * g.block.lddh, on ? n0 + col : g.n, g.n, dh);
      gated::emit8<uint16_t, (gated::Mode)MODE>(g.block, g.rows, g.n, t.r0 + row, n0 + col, on, G, U, dh);
    }
    return;
  }
  constexpr int V = 16 / sizeof(Out);
  for (int i = tid; i < BM * BN / V; i += 256) {
    const int row = i / (BN / V), col = i % (BN / V) * V;
    Out* at = PARTS ? (Out*)g.parts + ((i64)split * g.rows + t.r0 + row) * g.n : (Out*)g.Z + (t.r0 + row) * g.ldz;
    if (row < rows && col < cols) *reinterpret_cast<u32x4*>(at + n0 + col) = *reinterpret_cast<const u32x4*>(out + row * OUT_LD + col);
  }
}

template <int BM, int BN, int NS, bool PARTS = false, int MODE = NOT_GATED>
void go(ValuesArgsOf<MODE> a, hipStream_t st) {
  constexpr int BYTES = NS * (BM * 256 + BN * 68);
  auto kern = grouped_values_kernel<BM, BN, NS, PARTS, MODE>;
  static const bool configured = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, BYTES) == hipSuccess;
  (void)configured;
  a.tiles_n = MODE == NOT_GATED ? ceil_div(a.n, BN) : ceil_div(MODE == gated::HOLD_MX8 ? mx8::units(a.n) * mx8::UNIT : a.n, BN / 2);      // HOLD_MX8: codes past the last column are zeros
  launch_in_rows((a.groups == 1 ? (a.rows + BM - 1) / BM : most_row_tiles(a.rows, a.groups, BM)) * a.tiles_n * (PARTS ? a.splits : 1),
                 [&](int first, unsigned count) { hipLaunchKernelGGL(kern, dim3(count), dim3(256), BYTES, st, a, first); });
}

}  // namespace

bool values_supported(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Z, i64 ldz) {
  return d->d_in % 8 == 0 && d->d_out % 8 == 0 && ldx % 8 == 0 && ldz % 8 == 0 && ((uintptr_t)X & 15) == 0 && ((uintptr_t)Z & 15) == 0 && ldx < (1 << 22) &&
         d->d_in < (1 << 22);
}
// The tile and number of ranges of the contraction that are the fastest by a model of their times, if they are faster than the other way: the kernel for a handful of rows (few; here only
// split contractions are weighed against it, few_supported() having chosen between it and whole ones), or the weight written out and a product of its values.
// Fitted to 9800 calls of random sizes (256 to 14336), groups (1 to 64) and rows (8 to 16384), each in every way that can take it, and for the ranges to 1800 with few tiles; the choices take
// 2 to 3 % more time than the best would.  us, 64 x 128 / 128 x 128 / 128 x 256 / values: 14336 x 4096, 128 rows 22.6 / 29 / 46 / 66, 512 rows 71 / 61 / 52 / 88; 2048 x 5632, 1999 rows
// 52 / 44 / 66 / 69 (three weights in turn; 128 x 128 41 to 43 with the one in the caches); 64 experts of 1376 x 2048 with 128 rows each 65 / 69 / 81 / 162.  64 x 128 four stages deep, one workgroup per CU: 23.7, 85, 60, 86.
// Whole / in ranges / few rows: 1152 x 12032, 219 rows 51 / 20 / 41, 832 x 7232, 223 rows 33 / 16 / 25.
namespace {

struct ValuesPlan {
  bool better;       // than the other way
  int tile, ranges;
};
ValuesPlan values_plan(const poetx_grouped_desc* d, const Call& c, bool few, bool whole, size_t ws_bytes, size_t scratch) {
  struct Tile {
    int h, w;
    double rest, unit;      // us: of a launch; of a unit of a round of 256 tiles
    double alone;           // share of it that a few tiles take as well
    double uneven;          // of a round, where groups end inside tiles
  };
  static const Tile tiles[] = {{64, 128, 4.4, 0.62, 0.73, 0.05}, {128, 128, 5.1, 1.04, 0.61, 0}, {128, 256, 6.7, 1.71, 0.67, 0}};
  const int units = mx4::units(d->d_in);
  int best = 0, ranges = 1;
  double least = 1e30;
  for (int i = 0; i < 3; ++i) {
    const Tile& t = tiles[i];
    const double whole = tiles_of(FWD, d->rows, d->d_in, d->d_out, d->groups, t.h, t.w) / 256;
    for (const int splits : {1, 2, 3, 4, 6, 8}) {
      const size_t parts = splits > 1 ? (size_t)splits * d->rows * d->d_out * sizeof(float) : 0;
      if (splits > 1 && (t.w > 128 || 2 * splits > units || parts > ws_bytes)) break;
      if (splits == 1 && few) continue;
      const double rounds = whole * splits, filled = t.alone + (1 - t.alone) * (rounds < 1 ? rounds : 1);
      const double last = d->groups == 1 ? (double)(i64)(rounds + 0.999) : rounds + t.uneven;
      double us = t.rest + (units + splits - 1) / splits * t.unit * (rounds > 1 ? last : filled);
      if (splits > 1) us += 4.5 + 2 * parts / 6e6;      // the launch that adds them, and their way through the caches
      if (us < least) least = us, best = i, ranges = splits;
    }
  }
  const double written = 2.5 + (double)(d->rows < d->groups ? d->rows : d->groups) * d->d_out * d->d_in * 2.53 / 5.5e6;
  const bool other = few ? least >= few_values_us(d) : whole && least >= written + plan(POETX_BF16, FWD, c, stream_supported(POETX_BF16, FWD, c), scratch).us;
  return ValuesPlan{!other, best, ranges};
}
void parts_launch(int tile, const ValuesArgs& a, hipStream_t st) { tile == 0 ? go<64, 128, 3, true>(a, st) : go<128, 128, 3, true>(a, st); }

}  // namespace

bool values_launch(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, bool few, bool whole, void* ws, size_t ws_bytes, size_t scratch,
                   hipStream_t st) {
  const Call c{X, nullptr, Wq, Z, ldx, 0, ldz, offsets, d->rows, d->d_in, d->d_out, d->groups, 0};
  const ValuesPlan p = values_plan(d, c, few, whole, ws_bytes, scratch);
  if (!p.better) return false;
  StageTimer tm(POETX_STAGE_DENSE, st);
  const mx4::View w = mx4::view(Wq, (i64)d->groups * d->d_out, d->d_in);
  const ValuesArgs a{(const uint16_t*)X, ldx, w.codes, w.scales, (uint16_t*)Z, ldz, offsets, d->rows, d->d_in, d->d_out, d->groups, mx4::units(d->d_in), 0, p.ranges, (float*)ws};
  if (p.ranges > 1) {
    parts_launch(p.tile, a, st);
    add_parts(POETX_BF16, ws, p.ranges, d->d_out, c, st);
  } else if (p.tile == 0) {
    go<64, 128, 3>(a, st);
  } else if (p.tile == 1) {
    go<128, 128, 3>(a, st);
  } else {
    go<128, 256, 3>(a, st);
  }
  return true;
}

}  // namespace grouped

namespace gated {
namespace {

poetx_grouped_desc twice(int m, int n, int groups, i64 rows) { return poetx_grouped_desc{m, 2 * n, groups, POETX_BF16, rows, POETX_GROUPED_W_MX4, 0}; }
grouped::Call product_of(const void* X, i64 ldx, const void* W, const int32_t* offsets, i64 rows, int m, int n, int groups) {
  return grouped::Call{X, nullptr, W, nullptr, ldx, 0, 2 * (i64)n, offsets, rows, m, 2 * n, groups, 0};
}

}  // namespace

bool values_supported(const Call& c) {
  return c.m % 8 == 0 && c.ldx % 8 == 0 && ((uintptr_t)c.X & 15) == 0 && c.ldx < (1 << 22) && c.m < (1 << 22) &&
         ((i64)c.n + 256) * mx4::units(c.m) * 64 < (1ll << 31);
}
size_t values_parts_bytes(int m, int n, int groups, i64 rows, bool few, size_t scratch) {
  const poetx_grouped_desc d = twice(m, n, groups, rows);
  const grouped::ValuesPlan p = grouped::values_plan(&d, product_of(nullptr, m, nullptr, nullptr, rows, m, n, groups), few, true, n % 2 == 0 ? ~(size_t)0 : 0, scratch);      // sums are stored in whole vectors
  return p.better && p.ranges > 1 ? (size_t)p.ranges * rows * 2 * n * sizeof(float) : 0;
}
// The choice is that of a product of 2n columns: the tiles, the contraction and the bytes of the weight are the same.
bool values_launch(const Call& c, bool few, void* sums, size_t sums_bytes, size_t scratch, hipStream_t st) {
  using grouped::go;
  const poetx_grouped_desc d = twice(c.m, c.n, c.groups, c.rows);
  const grouped::ValuesPlan p = grouped::values_plan(&d, product_of(c.X, c.ldx, c.W, c.offsets, c.rows, c.m, c.n, c.groups), few, true, c.n % 2 == 0 ? sums_bytes : 0, scratch);
  if (!p.better) return false;
  StageTimer tm(POETX_STAGE_DENSE, st);
  const mx4::View w = mx4::view(c.W, 2 * (i64)c.groups * c.n, c.m);
  grouped::GatedValuesArgs a{{(const uint16_t*)c.X, c.ldx, w.codes, w.scales, nullptr, 0, c.offsets, c.rows, c.m, c.n, c.groups, mx4::units(c.m), 0, p.ranges, (float*)sums}, c.out};
  if (p.ranges > 1) {
    a.n = 2 * c.n;
    grouped::parts_launch(p.tile, a, st);
    rows_launch(POETX_BF16, SUMS, In{sums, nullptr, 0, p.ranges}, c.offsets, c.groups, c.rows, c.n, c.mode, c.out, st);
    return true;
  }
  auto tiled = [&](auto MODE_) {
    constexpr int MODE = decltype(MODE_)::value;
    if (p.tile == 0) go<64, 128, 3, false, MODE>(a, st);
    else if (p.tile == 1) go<128, 128, 3, false, MODE>(a, st);
    else go<128, 256, 3, false, MODE>(a, st);
  };
  if (c.mode == FWD) tiled(std::integral_constant<int, FWD>{});
  else if (c.mode == HOLD) tiled(std::integral_constant<int, HOLD>{});
  else if (c.mode == HOLD_MX8) tiled(std::integral_constant<int, HOLD_MX8>{});
  else tiled(std::integral_constant<int, BWD>{});
  return true;
}

}  // namespace gated
}  // namespace poetx
