// The gated block on the streaming kernel: both projections, the activation and the product in one launch, and the backward pass that makes G and U again.
//
// A tile of the weight has 16 rows of gate and 16 of up in turn, so that each lane ends with G and U of the same four elements: nothing is exchanged for the product, and a block of 32 columns
// of eight bits lies in one wave's registers.  G and U reach memory only where they are kept.
// What bounds it: the product, and what a tile writes while its CU multiplies nothing.  16384 x 4096 by 2 x 14336 x 4096, us and PFLOP/s: H alone 2855 (1.35; the grouped product of
// the same columns, which writes G and U, 2960), G and U kept 3170 (1.21), in eight bits 3140 (1.23), gradients from G and U made again 3280 (1.17).  The multiplications take 61 % of the
// cycles at 1.9 GHz, tiles' ends 9 to 20 us of each 110 (by what they write, at 5 TB/s, and 2300 to 4400 vector instructions of a wave), the rest waits for a stage's loads.  With operands in
// 64-byte pieces three stages ahead, instead of whole lines one unit ahead, 2 to 5 % more (8 groups of 2 x 8192 x 4096 1830 against 1724); loads of a unit in the first half of the
// stage 3 % more; two workgroups of 128 x 128 a CU, so that one ends tiles while the other multiplies, 5 to 15 % more but for contractions of 512 and less.
// Few rows per group: the bytes of the weights (57 groups, 8190 rows of 2 x 1376 x 2048 200 us for 743 MB, of which a copy would take 145).
#include "grouped_stream.h"

namespace poetx {
namespace gated {
namespace {

using grouped::BF16;
using grouped::F32;
using grouped::GatedStreamArgs;
using grouped::StreamTile;

constexpr int kCUs = 256;

template <class C>
void go(const GatedStreamArgs& a0, hipStream_t st) {
  auto kern = grouped::grouped_stream_kernel<grouped::FWD, C>;
  static const bool configured = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES) == hipSuccess;
  (void)configured;
  GatedStreamArgs a = a0;
  const int cols = C::GATED == HOLD_MX8 ? mx8::units(a.N) * mx8::UNIT : a.N;      // codes past the last column are zeros
  a.tiles_n = ceil_div(cols, C::BN / 2);
  hipLaunchKernelGGL(kern, dim3(kCUs * C::PER_CU), dim3(256), C::LDS_BYTES, st, a);
}

template <Mode MODE>
void pick(grouped::Kernel k, const GatedStreamArgs& a, hipStream_t st) {
  if (k == grouped::SINGLE_128) go<StreamTile<128, 128, 4, F32, 2, false, MODE>>(a, st);
  else if (k == grouped::SINGLE_64) {
    if constexpr (MODE == HOLD_MX8) go<StreamTile<128, 128, 4, F32, 2, false, MODE>>(a, st);      // a wave's columns have to be whole blocks
    else go<StreamTile<64, 64, 8, F32, 2, false, MODE>>(a, st);
  } else if (k == grouped::STREAM_256) go<StreamTile<256, 256, 4, BF16, 1, false, MODE>>(a, st);
  else if (k == grouped::STREAM_256x128) go<StreamTile<256, 128, 6, BF16, 1, false, MODE>>(a, st);
  else go<StreamTile<128, 128, 8, BF16, 1, false, MODE>>(a, st);
}
template <Mode MODE>
void pick_narrow(grouped::Kernel k, const GatedStreamArgs& a, hipStream_t st) {
  if (k == grouped::SINGLE_128 || k == grouped::SINGLE_64) go<StreamTile<128, 128, 4, F32, 2, false, MODE, true>>(a, st);
  else if (k == grouped::STREAM_256 || k == grouped::STREAM_256x128) go<StreamTile<256, 128, 6, BF16, 1, false, MODE, true>>(a, st);
  else go<StreamTile<128, 128, 8, BF16, 1, false, MODE, true>>(a, st);
}

}  // namespace

bool stream_supported(int dtype, const Call& c) {
  const int es = dtype == POETX_F32 ? 4 : 2, v = 16 / es;
  const i64 wide = (1ll << 31) / (es * 256);      // a tile's rows span less than 2^31 bytes, and so do a group's weights
  return c.groups <= 256 && c.m % v == 0 && c.ldx % v == 0 && (((uintptr_t)c.X | (uintptr_t)c.W) & 15) == 0 && c.ldx < wide && c.m < wide / 2 && 2 * (i64)c.n < wide &&
         (2 * (i64)c.n + 256) * c.m * es < (1ll << 31) && c.out.ldh < wide && c.out.ldgu < wide && c.out.lddh < wide;
}

void stream_launch(int dtype, grouped::Kernel k, const Call& c, hipStream_t st) {
  const int es = dtype == POETX_F32 ? 4 : 2;
  GatedStreamArgs a = {};
  a.A = (const char*)c.X;
  a.lda = (int)(es * c.ldx);
  a.B = (const char*)c.W;
  a.ldb = es * c.m;
  a.K = c.m;
  a.N = c.n;
  a.offsets = c.offsets;
  a.rows = (int)c.rows;
  a.groups = c.groups;
  a.splits = 1;
  a.block = c.out;
  const int v = 16 / es;
  auto whole = [&](const void* p, i64 ld) { return ((uintptr_t)p & 15) == 0 && ld % v == 0; };
  const bool pair = c.mode == HOLD || c.mode == BWD;
  const bool wide = c.n % v == 0 && whole(c.out.H, c.out.H ? c.out.ldh : 0) && (!pair || (whole(c.out.G, c.out.ldgu) && whole(c.out.U, c.out.ldgu))) &&
                    (c.mode != BWD || whole(c.out.dH, c.out.lddh));
  auto mode = [&](auto MODE_) {
    constexpr Mode MODE = decltype(MODE_)::value;
    wide ? pick<MODE>(k, a, st) : pick_narrow<MODE>(k, a, st);
  };
  if (c.mode == FWD) mode(std::integral_constant<Mode, FWD>{});
  else if (c.mode == HOLD) mode(std::integral_constant<Mode, HOLD>{});
  else if (c.mode == HOLD_MX8) mode(std::integral_constant<Mode, HOLD_MX8>{});
  else mode(std::integral_constant<Mode, BWD>{});
}

}  // namespace gated
}  // namespace poetx
