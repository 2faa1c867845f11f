// Grouped products on the streaming kernel: which of them it takes, on which tile.
#include "grouped_stream.h"

namespace poetx {
namespace grouped {
namespace {

typedef StreamTile<256, 256, 4, BF16> Tile256;
typedef StreamTile<256, 128, 6, BF16> Tile256x128;
typedef StreamTile<128, 128, 8, BF16> Tile128;
typedef StreamTile<128, 128, 8, BF16, 1, true> Parts128;
typedef StreamTile<256, 256, 4, CODES> Codes256;
typedef StreamTile<128, 128, 6, CODES> Codes128;
typedef StreamTile<128, 128, 4, F32, 2> Single128;
typedef StreamTile<64, 64, 8, F32, 2> Single64;

constexpr int kCUs = 256;

template <Dir DIR, class C>
void go(const StreamArgs& a0, hipStream_t st) {
  auto kern = grouped_stream_kernel<DIR, C>;
  static const bool configured = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES) == hipSuccess;
  (void)configured;
  StreamArgs a = a0;
  a.tiles_n = ceil_div(a.N, C::BN);
  hipLaunchKernelGGL(kern, dim3(kCUs * C::PER_CU), dim3(256), C::LDS_BYTES, st, a);
}

template <Dir DIR>
void pick(Kernel k, const StreamArgs& a, hipStream_t st) {
  if constexpr (DIR != WEIGHT) {
    if (k == STREAM_128 && a.splits > 1) return go<DIR, Parts128>(a, st);
  }
  if (k == SINGLE_128) go<DIR, Single128>(a, st);
  else if (k == SINGLE_64) go<DIR, Single64>(a, st);
  else if (k == STREAM_256) go<DIR, Tile256>(a, st);
  else if (k == STREAM_256x128) go<DIR, Tile256x128>(a, st);
  else go<DIR, Tile128>(a, st);
}

}  // namespace

// A group's last tile is half empty on average, and a group with rows has at least one.
double tiles_of(Dir dir, i64 rows, int m, int n, int groups, int h, int w) {
  const double across = ceil_div(dir == FWD ? n : m, w);
  if (dir == WEIGHT) return (double)groups * ceil_div(n, h) * across;
  if (groups == 1) return (double)((rows + h - 1) / h) * across;
  const double live = rows < groups ? (double)rows : groups, t = (double)rows / h + 0.5 * live;
  return (t > live ? t : live) * across;
}

namespace {

// The sums of a contraction's ranges, [split][rows][cols], added in order and rounded, for the rows that some group has.  A wave takes 256 columns of a row.
template <class T>
__global__ __launch_bounds__(256) void add_parts_kernel(const float* __restrict__ parts, int splits, i64 rows, int cols, T* __restrict__ out, i64 ld,
                                                        const int32_t* __restrict__ offsets, int groups, i64 waves, int block0) {
  const int lane = threadIdx.x & 63, across = (cols + 255) / 256;
  const i64 w = (block0 + (i64)blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= waves) return;
  const i64 row = w / across;
  const int col = (int)(w - row * across) * 256 + 4 * lane;
  if (row < offset_at(offsets, 0, rows) || row >= furthest_end(offsets, groups, rows) || col >= cols) return;
  const float* p = parts + row * cols + col;
  floatx4 sum = *reinterpret_cast<const floatx4*>(p);
  for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const floatx4*>(p + s * rows * cols);
  T* o = out + row * ld + col;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<floatx4*>(o) = sum;
  } else {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    *reinterpret_cast<u32x2*>(o) = u32x2{mm::pack2_bf16(sum[0], sum[1]), mm::pack2_bf16(sum[2], sum[3])};
  }
}
// The same of weight gradients, matrices of m columns one after the other; rows of the sums are whole vectors.
__global__ __launch_bounds__(256) void add_weights_kernel(const floatx4* __restrict__ parts, int splits, i64 vectors, int m, float* __restrict__ out, int accumulate, int block0) {
  const i64 i = (block0 + (i64)blockIdx.x) * 256 + threadIdx.x;
  if (i >= vectors) return;
  floatx4 sum = parts[i];
  for (int s = 1; s < splits; ++s) sum += parts[i + s * vectors];
  if (m % 4 == 0) {
    floatx4* o = reinterpret_cast<floatx4*>(out) + i;
    if (accumulate) sum += *o;
    *o = sum;
    return;
  }
  const int across = (m + 3) / 4;
  const i64 row = i / across;
  const int col = (int)(i - row * across) * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < m) out[row * m + col + e] = accumulate ? out[row * m + col + e] + sum[e] : sum[e];
}
template <class T>
void add(const float* parts, int splits, int cols, const Call& c, hipStream_t st) {
  const i64 waves = c.rows * ((cols + 255) / 256);
  launch_in_rows((waves + 3) / 4, [&](int block0, unsigned count) {
    hipLaunchKernelGGL(add_parts_kernel<T>, dim3(count), dim3(256), 0, st, parts, splits, c.rows, cols, (T*)c.out, c.ld_out, c.offsets, c.groups, waves, block0);
  });
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

void add_parts(int dtype, const void* parts, int splits, int cols, const Call& c, hipStream_t st) {
  dtype == POETX_F32 ? add<float>((const float*)parts, splits, cols, c, st) : add<uint16_t>((const float*)parts, splits, cols, c, st);
}

bool stream_supported(int dtype, Dir dir, const Call& c) {
  const int es = dtype == POETX_F32 ? 4 : 2, v = 16 / es;
  const i64 wide = (1ll << 31) / (es * 256);      // a tile's rows, or a stage's, span less than 2^31 bytes
  return c.groups <= Tile256::GROUPS && c.m % v == 0 && c.n % v == 0 && c.ld_in % v == 0 && c.ld_out % v == 0 && aligned16(c.in) && aligned16(c.out) &&
         c.ld_in < wide && c.ld_out < wide && c.m < wide / 2 &&
         (dir == WEIGHT ? c.ld_in2 % v == 0 && aligned16(c.in2) && c.ld_in2 < wide : aligned16(c.w));
}

bool weight_stream_supported(int dtype, const Call& c) {
  const int es = dtype == POETX_F32 ? 4 : 2, v = 16 / es;
  const i64 wide = (1ll << 31) / (es * 256);
  return c.groups <= Tile256::GROUPS && c.ld_in % v == 0 && c.ld_in2 % v == 0 && (c.m % v == 0 || c.row_in >= (c.m + v - 1) / v * v) && (c.n % v == 0 || c.row_in2 >= (c.n + v - 1) / v * v) &&
         c.ld_in < wide && c.ld_in2 < wide && c.ld_out < wide && c.m < wide / 2;
}

// The figures were fitted to 650 calls in bf16 and 700 in fp32 of random directions, sizes (64 to 14336; 64 to 4096), groups (1 to 128) and rows (1 to 32768; 8 to 8192), each
// with every kernel that could take it; the choices they lead to take 2 % more time than the best would (geometric mean).
Plan plan(int dtype, Dir dir, const Call& c, bool streams, size_t scratch) {
  struct Row {
    Kernel kernel;
    int h, w, depth;      // tile, depth of a stage
    double stage;         // us
    double at_once;       // tiles that the chip works on at a time
    double uneven;        // bf16 streams, which go round by round: part of a round that the last one takes more than its share, where groups end inside tiles
    double rest;          // us
  };
  static const Row bf16[] = {{EDGE_32, 32, 32, 128, 0.63, 465, 0, 3.6},   {EDGE_32_DEEP, 32, 32, 512, 0.88, 118, 0, 5.0},     {EDGE_64, 64, 64, 64, 0.73, 546, 0, 3.2},
                             {EDGE_128, 128, 128, 64, 1.51, 282, 0, 4.0}, {STREAM_256, 256, 256, 32, 0.645, kCUs, 0.39, 9.1}, {STREAM_256x128, 256, 128, 32, 0.52, kCUs, 0.28, 7.9},
                             {STREAM_128, 128, 128, 32, 0.32, kCUs, 0.58, 7.9}};
  static const Row fp32[] = {{EDGE_32, 32, 32, 64, 0.87, 356, 0, 3.9}, {EDGE_64, 64, 64, 32, 1.08, 260, 0, 3.6}, {SINGLE_128, 128, 128, 16, 1.42, 253, 0, 10.2},
                             {SINGLE_64, 64, 64, 16, 0.42, 295, 0, 7.0}};
  const bool f = dtype == POETX_F32;
  const Row* rows = f ? fp32 : bf16;
  const int count = f ? (int)(sizeof(fp32) / sizeof(Row)) : (int)(sizeof(bf16) / sizeof(Row));
  const double live = c.rows < c.groups ? (double)c.rows : c.groups;
  const double K = dir == FWD ? c.m : dir == INPUT ? c.n : live > 0 ? c.rows / live : 0;
  const int out_cols = dir == FWD ? c.n : c.m;
  const double out_us = dir == WEIGHT ? 4.0 * c.groups * c.n * c.m / 5.1e6 : 0;      // fp32 weights to memory
  Plan best{EDGE_32, 1, 0, 1e30};
  for (int i = 0; i < count; ++i) {
    const Row& r = rows[i];
    const bool stream = r.kernel >= STREAM_256;
    if (stream && !streams) break;
    const double tiles = tiles_of(dir, c.rows, c.m, c.n, c.groups, r.h, r.w), stages = (double)(i64)((K + r.depth - 1) / r.depth);
    const double stage = r.stage * (dir == FWD && stream && r.kernel != STREAM_256 ? 0.9 : 1.0);      // bf16: whole lines; fp32: the fewest instructions beside the multiplications
    // few tiles: their contraction in ranges, whose fp32 sums are added by another launch (7.5 us with the wait between the two, and their way through the caches)
    const bool splittable = dir == WEIGHT ? stream : r.kernel == STREAM_128 || r.kernel >= SINGLE_128;
    for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
      // a weight gradient whose rows are no whole vectors goes by way of the scratch in any case
      const bool through = splits > 1 || (stream && dir == WEIGHT && c.m % 4 != 0);
      const size_t parts = through ? (size_t)splits * (dir == WEIGHT ? (i64)c.groups * c.n : c.rows) * ((out_cols + 3) / 4 * 4) * sizeof(float) : 0;
      if (splits == 1 && parts > scratch) break;
      if (splits > 1 && (!splittable || parts > scratch || 4 * splits > stages || tiles * splits > 2 * r.at_once)) break;
      double us = tiles * splits / r.at_once;
      if (stream && !f) us = c.groups == 1 ? (double)(i64)(us + 0.999) : us + r.uneven;
      us = (us < 1 ? 1 : us) * (double)(i64)((stages + splits - 1) / splits) * stage;
      // a stream stores between multiplications; the others have several workgroups on a CU, but store less well
      const double stores = (f ? 1.5 : 1.35) * out_us;
      us = r.rest + (stream ? us + splits * out_us : us > stores ? us : stores);
      if (through) us += 7.5 + (dir == WEIGHT ? parts / 8e6 + out_us : 2 * parts / 8e6);
      if (us < best.us) best = Plan{r.kernel, splits, parts, us};
    }
  }
  return best;
}

void stream_launch(int dtype, Dir dir, const Plan& p, const Call& c, void* scratch, hipStream_t st) {
  const Kernel k = p.kernel;
  const int es = dtype == POETX_F32 ? 4 : 2;
  StreamArgs a = {};
  a.offsets = c.offsets;
  a.rows = (int)c.rows;
  a.groups = c.groups;
  a.C = c.out;
  a.ldc = (int)c.ld_out;
  a.accumulate = c.accumulate;
  a.splits = p.splits;
  if (dir == WEIGHT) {
    a.A = (const char*)c.in2;
    a.lda = (int)(es * c.ld_in2);
    a.B = (const char*)c.in;
    a.ldb = (int)(es * c.ld_in);
    a.M = c.n;
    a.N = c.m;
    a.row_a = c.row_in2 > c.n ? c.row_in2 : c.n;
    a.row_b = c.row_in > c.m ? c.row_in : c.m;
    if (!p.parts) return pick<WEIGHT>(k, a, st);
    const int ld = (c.m + 3) / 4 * 4;
    a.C = scratch;
    a.ldc = ld;
    a.N = ld <= a.row_b ? ld : c.m;
    a.accumulate = 0;
    pick<WEIGHT>(k, a, st);
    const i64 vectors = (i64)c.groups * c.n * (ld / 4);
    launch_in_rows((vectors + 255) / 256, [&](int block0, unsigned count) {
      hipLaunchKernelGGL(add_weights_kernel, dim3(count), dim3(256), 0, st, (const floatx4*)scratch, p.splits, vectors, c.m, (float*)c.out, c.accumulate, block0);
    });
    return;
  }
  a.A = (const char*)c.in;
  a.lda = (int)(es * c.ld_in);
  a.B = (const char*)c.w;
  a.ldb = es * c.m;
  a.K = dir == FWD ? c.m : c.n;
  a.N = dir == FWD ? c.n : c.m;
  if (p.splits > 1) {
    a.C = scratch;
    a.ldc = a.N;
  }
  dir == FWD ? pick<FWD>(k, a, st) : pick<INPUT>(k, a, st);
  if (p.splits > 1) add_parts(dtype, a.C, p.splits, a.N, c, st);
}

void stream_sums(int dtype, const Plan& p, const Call& c, void* sums, hipStream_t st) {
  const int es = dtype == POETX_F32 ? 4 : 2;
  StreamArgs a = {};
  a.offsets = c.offsets;
  a.rows = (int)c.rows;
  a.groups = c.groups;
  a.C = sums;
  a.A = (const char*)c.in;
  a.lda = (int)(es * c.ld_in);
  a.B = (const char*)c.w;
  a.ldb = es * c.m;
  a.K = c.m;
  a.N = a.ldc = c.n;
  a.splits = p.splits;
  if (dtype == POETX_BF16) return go<FWD, Parts128>(a, st);
  p.kernel == SINGLE_128 ? go<FWD, Single128>(a, st) : go<FWD, Single64>(a, st);
}

// ---- both operands in four bits ---------------------------------------------------------------------
bool codes_supported(const poetx_grouped_desc* d, const void* Z, i64 ldz) {
  return d->groups <= Codes256::GROUPS && d->d_out % 8 == 0 && ldz % 8 == 0 && ldz * 512 < (1ll << 31) && aligned16(Z) && (i64)mx4::units(d->d_in) * 64 * 256 < (1ll << 31) &&
         d->rows < (1 << 28) && (i64)d->groups * (d->d_out + 64) < (1 << 28);
}
size_t codes_workspace_bytes(const poetx_grouped_desc* d) {
  const size_t units = mx4::units(d->d_in);
  return align256(d->rows * units * 64) + align256(mx4::positions(d->rows, d->groups) * units * 4) + align256((size_t)d->groups * ((d->d_out + 63) / 64) * units * 256);
}
void codes_launch(const poetx_grouped_desc* d, const void* X, i64 ldx, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, void* ws, hipStream_t st) {
  const i64 wrows = (i64)d->groups * d->d_out;
  const int units = mx4::units(d->d_in);
  char* xs = (char*)ws + align256((size_t)d->rows * units * 64);
  char* wst = xs + align256(mx4::positions(d->rows, d->groups) * units * 4);
  {
    StageTimer tm(POETX_STAGE_DEQUANT, st);
    mx4_operands_launch(X, d->rows, d->d_in, ldx, offsets, d->groups, d->d_out, Wq, ws, xs, wst, st);
  }
  StageTimer tm(POETX_STAGE_DENSE, st);
  StreamArgs a = {};
  a.A = (const char*)ws;
  a.B = (const char*)mx4::view(Wq, wrows, d->d_in).codes;
  a.SA = (const uint32_t*)xs;
  a.SB = (const uint32_t*)wst;
  a.sa_step = (int)(4 * mx4::positions(d->rows, d->groups));
  a.sb_step = d->groups * ((d->d_out + 63) / 64) * 256;
  a.C = Z;
  a.lda = a.ldb = units * 64;
  a.ldc = (int)ldz;
  a.offsets = offsets;
  a.rows = (int)d->rows;
  a.groups = d->groups;
  a.K = units * mx4::UNIT;
  a.N = d->d_out;
  a.splits = 1;
  // A round of 256 x 256 tiles takes as long as 2.1 of 128 x 128 ones.
  auto rounds = [&](int side) {
    const double t = tiles_of(FWD, d->rows, d->d_in, d->d_out, d->groups, side, side) / kCUs;
    return t < 1 ? 1.0 : d->groups == 1 ? (double)(int)(t + 0.999) : t + 0.4;
  };
  const double c0 = 2.1 * rounds(256), c2 = rounds(128);
  if (c0 <= c2) go<FWD, Codes256>(a, st);
  else go<FWD, Codes128>(a, st);
}

}  // namespace grouped
}  // namespace poetx
