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

// Output tiles of height x width that groups of average size give, an average half a tile per group wasted.
double tiles_of(Dir dir, i64 rows, int m, int n, int groups, int h, int w) {
  if (dir == WEIGHT) return (double)groups * ((n + h - 1) / h) * ((m + w - 1) / w);
  const int cols = dir == FWD ? n : m;
  const double live = rows < groups ? (double)rows : groups;
  double t = (double)rows / h + (groups > 1 ? 0.5 * live : 0.0);
  if (t < live) t = live;
  if (groups == 1) t = (double)((rows + h - 1) / h);
  return t * ((cols + w - 1) / w);
}
// Rounds of the chip's workgroups over so many tiles; `work`: what a tile costs, of a 256 x 256 one.
double rounds(double tiles, double work) { return (tiles <= kCUs ? 1.0 : tiles / kCUs + 0.4) * work; }

template <Dir DIR>
void pick(const StreamArgs& a, i64 rows, int m, int n, hipStream_t st) {
  const double c0 = rounds(tiles_of(DIR, rows, m, n, a.groups, 256, 256), 1.0), c1 = rounds(tiles_of(DIR, rows, m, n, a.groups, 256, 128), 0.56),
               c2 = rounds(tiles_of(DIR, rows, m, n, a.groups, 128, 128), 0.32);
  if (c0 <= c1 && c0 <= c2) go<DIR, Tile256>(a, st);
  else if (c1 <= c2) go<DIR, Tile256x128>(a, st);
  else go<DIR, Tile128>(a, st);
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

bool stream_supported(Dir dir, const Call& c) {
  const i64 wide = 1ll << 31;
  return c.groups <= Tile256::GROUPS && c.m % 8 == 0 && c.n % 8 == 0 && c.ld_in % 8 == 0 && c.ld_out % 8 == 0 && aligned16(c.in) && aligned16(c.out) &&
         (dir == WEIGHT ? c.ld_in2 % 8 == 0 && aligned16(c.in2) && c.ld_in2 * 64 < wide && c.ld_in * 64 < wide && (i64)c.m * 1024 < wide
                        : aligned16(c.w) && c.ld_in * 512 < wide && (i64)c.m * 512 < wide && c.ld_out * 512 < wide);
}

void stream_launch(Dir dir, const Call& c, hipStream_t st) {
  StreamArgs a = {};
  a.offsets = c.offsets;
  a.rows = c.rows;
  a.groups = c.groups;
  a.C = c.out;
  a.ldc = c.ld_out;
  a.accumulate = c.accumulate;
  if (dir == WEIGHT) {
    a.A = (const char*)c.in2;
    a.lda = 2 * c.ld_in2;
    a.B = (const char*)c.in;
    a.ldb = 2 * c.ld_in;
    a.M = c.n;
    a.N = c.m;
    return pick<WEIGHT>(a, c.rows, c.m, c.n, st);
  }
  a.A = (const char*)c.in;
  a.lda = 2 * c.ld_in;
  a.B = (const char*)c.w;
  a.ldb = 2 * (i64)c.m;
  a.K = dir == FWD ? c.m : c.n;
  a.N = dir == FWD ? c.n : c.m;
  dir == FWD ? pick<FWD>(a, c.rows, c.m, c.n, st) : pick<INPUT>(a, c.rows, c.m, c.n, st);
}

// ---- both operands in four bits ---------------------------------------------------------------------
bool codes_supported(const poetx_grouped_desc* d, const void* Z, i64 ldz) {
  return d->groups <= Codes256::GROUPS && d->d_out % 8 == 0 && ldz % 8 == 0 && ldz * 512 < (1ll << 31) && aligned16(Z) && (i64)mx4::units(d->d_in) * 64 * 256 < (1ll << 31);
}
void codes_launch(const poetx_grouped_desc* d, const void* Xq, const void* Wq, const int32_t* offsets, void* Z, i64 ldz, hipStream_t st) {
  const mx4::View x = mx4::view(Xq, d->rows, d->d_in), w = mx4::view(Wq, (i64)d->groups * d->d_out, d->d_in);
  const int units = mx4::units(d->d_in);
  StreamArgs a = {};
  a.A = (const char*)x.codes;
  a.B = (const char*)w.codes;
  a.SA = x.scales;
  a.SB = w.scales;
  a.C = Z;
  a.lda = a.ldb = (i64)units * 64;
  a.ldc = ldz;
  a.offsets = offsets;
  a.rows = d->rows;
  a.groups = d->groups;
  a.K = units * mx4::UNIT;
  a.N = d->d_out;
  const double c0 = rounds(tiles_of(FWD, d->rows, d->d_in, d->d_out, d->groups, 256, 256), 1.0),
               c2 = rounds(tiles_of(FWD, d->rows, d->d_in, d->d_out, d->groups, 128, 128), 0.32);
  if (c0 <= c2) go<FWD, Codes256>(a, st);
  else go<FWD, Codes128>(a, st);
}

}  // namespace grouped
}  // namespace poetx
