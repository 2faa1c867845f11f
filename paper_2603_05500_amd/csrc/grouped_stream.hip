// Grouped products on the streaming kernel: which of them it takes, on which tile.
#include "grouped_stream.h"

namespace poetx {
namespace grouped {
namespace {

typedef StreamTile<256, 256, 4, false> Tile256;
typedef StreamTile<256, 128, 6, false> Tile256x128;
typedef StreamTile<128, 128, 8, false> Tile128;
typedef StreamTile<256, 256, 4, true> Codes256;
typedef StreamTile<128, 128, 6, true> Codes128;

constexpr int kCUs = 256;

template <Dir DIR, class C>
void go(const StreamArgs& a0, hipStream_t st) {
  auto kern = grouped_stream_kernel<DIR, C>;
  static const bool configured = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES) == hipSuccess;
  (void)configured;
  StreamArgs a = a0;
  a.tiles_n = ceil_div(a.N, C::BN);
  hipLaunchKernelGGL(kern, dim3(kCUs), dim3(256), C::LDS_BYTES, st, a);
}

template <Dir DIR>
void pick(Kernel k, const StreamArgs& a, hipStream_t st) {
  if (k == STREAM_256) go<DIR, Tile256>(a, st);
  else if (k == STREAM_256x128) go<DIR, Tile256x128>(a, st);
  else go<DIR, Tile128>(a, st);
}

// Output tiles of h x w: a group's last tile is half empty on average, and a group with rows has at least one.
double tiles_of(Dir dir, i64 rows, int m, int n, int groups, int h, int w) {
  const double across = ceil_div(dir == FWD ? n : m, w);
  if (dir == WEIGHT) return (double)groups * ceil_div(n, h) * across;
  if (groups == 1) return (double)((rows + h - 1) / h) * across;
  const double live = rows < groups ? (double)rows : groups, t = (double)rows / h + 0.5 * live;
  return (t > live ? t : live) * across;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

bool stream_supported(Dir dir, const Call& c) {
  const i64 wide = 1ll << 31;
  return c.groups <= Tile256::GROUPS && c.m % 8 == 0 && c.n % 8 == 0 && c.ld_in % 8 == 0 && c.ld_out % 8 == 0 && aligned16(c.in) && aligned16(c.out) &&
         (dir == WEIGHT ? c.ld_in2 % 8 == 0 && aligned16(c.in2) && c.ld_in2 * 64 < wide && c.ld_in * 64 < wide && (i64)c.m * 1024 < wide
                        : aligned16(c.w) && c.ld_in * 512 < wide && (i64)c.m * 512 < wide && c.ld_out * 512 < wide);
}

// The figures were fitted to 600 calls of random directions, sizes (64 to 14336), groups (1 to 128) and rows (1 to 32768) with every kernel that could take them; the choices
// they lead to take 1.3 % more time than the best would (geometric mean), 10 % at worst in nine of ten.
Kernel plan(int dtype, Dir dir, const Call& c, bool streams) {
  struct Row {
    int h, w, depth;      // tile, depth of a stage
    double stage;         // us
    double at_once;       // edge kernels: tiles that the chip works on at a time
    double uneven;        // streams: part of a round that the last one takes more than its share, where groups end inside tiles
    double rest;          // us
  };
  static const Row bf16[KERNELS] = {{32, 32, 128, 0.64, 400, 0, 3.5}, {32, 32, 512, 1.1, 137, 0, 5.1}, {64, 64, 64, 0.80, 433, 0, 2.9}, {128, 128, 64, 1.58, 224, 0, 3.2},
                                    {256, 256, 32, 0.67, kCUs, 0.45, 11.8}, {256, 128, 32, 0.52, kCUs, 0.33, 7.5}, {128, 128, 32, 0.315, kCUs, 0.65, 7.7}};
  static const Row f32[EDGE_128] = {{32, 32, 64, 1.0, 430, 0, 3}, {32, 32, 256, 1e9, 1, 0, 3}, {64, 64, 32, 1.05, 360, 0, 3}};
  const double live = c.rows < c.groups ? (double)c.rows : c.groups;
  const double K = dir == FWD ? c.m : dir == INPUT ? c.n : live > 0 ? c.rows / live : 0;
  const double out_us = dir == WEIGHT ? 4.0 * c.groups * c.n * c.m / 5.1e6 : 0;      // fp32 weights to memory
  int best = EDGE_32;
  double least = 1e30;
  for (int k = 0; k < (dtype == POETX_F32 ? EDGE_128 : streams ? KERNELS : STREAM_256); ++k) {
    const Row& r = dtype == POETX_F32 ? f32[k] : bf16[k];
    const double tiles = tiles_of(dir, c.rows, c.m, c.n, c.groups, r.h, r.w), stages = (i64)((K + r.depth - 1) / r.depth);
    double us = tiles / r.at_once;
    if (k >= STREAM_256) us = c.groups == 1 ? (double)(i64)(us + 0.999) : us + r.uneven;
    us = (us < 1 ? 1 : us) * stages * r.stage;
    // a stream stores between multiplications; the others have several workgroups on a CU, but store less well
    us = r.rest + (k >= STREAM_256 ? us + out_us : us > 1.23 * out_us ? us : 1.23 * out_us);
    if (us < least) {
      least = us;
      best = k;
    }
  }
  return (Kernel)best;
}

void stream_launch(Dir dir, Kernel k, const Call& c, hipStream_t st) {
  StreamArgs a = {};
  a.offsets = c.offsets;
  a.rows = (int)c.rows;
  a.groups = c.groups;
  a.C = c.out;
  a.ldc = (int)c.ld_out;
  a.accumulate = c.accumulate;
  if (dir == WEIGHT) {
    a.A = (const char*)c.in2;
    a.lda = (int)(2 * c.ld_in2);
    a.B = (const char*)c.in;
    a.ldb = (int)(2 * c.ld_in);
    a.M = c.n;
    a.N = c.m;
    return pick<WEIGHT>(k, a, st);
  }
  a.A = (const char*)c.in;
  a.lda = (int)(2 * c.ld_in);
  a.B = (const char*)c.w;
  a.ldb = 2 * c.m;
  a.K = dir == FWD ? c.m : c.n;
  a.N = dir == FWD ? c.n : c.m;
  dir == FWD ? pick<FWD>(k, a, st) : pick<INPUT>(k, a, st);
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
