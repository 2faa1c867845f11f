// The 4-bit microscaled format on the device: where a buffer's parts lie, and its conversions.
#pragma once

#include "poetx_common.h"

namespace poetx {
namespace mx4 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int UNIT = 128;      // columns of 64 bytes of codes and one word of scales: what rows are rounded up to
__host__ __device__ inline int units(int cols) { return (int)(((i64)cols + UNIT - 1) / UNIT); }
inline size_t scale_offset(i64 rows, int cols) { return align256((size_t)rows * units(cols) * 64); }
inline size_t bytes(i64 rows, int cols) { return scale_offset(rows, cols) + (size_t)rows * units(cols) * 4; }
struct View {
  const uint8_t* codes;
  const uint8_t* scales;
};
inline View view(const void* Q, i64 rows, int cols) { return View{(const uint8_t*)Q, (const uint8_t*)Q + scale_offset(rows, cols)}; }

// ---- scales as the streaming product reads them -------------------------------------------------------
// Unit by unit, 256 bytes per 64 rows: byte (16 q + i) 4 + s is that of row 16 s + i and the unit's block q, so that a lane's word holds its fragments of four 16-row
// pieces.  A group starts a new 64: of the weight its rows are rounded up; the rows of X, whose groups start anywhere, have positions that leave room for it.
__host__ __device__ inline i64 position(i64 r0, int g) { return (r0 + 63) / 64 * 64 + 64 * (i64)g; }      // of a group's first row: past the last row of those before
inline __host__ __device__ i64 positions(i64 rows, int groups) { return position(rows, groups); }
__device__ __forceinline__ int scale_place(int row, int q) { return (16 * q + (row & 15)) * 4 + (row >> 4); }

// A scale byte as the fp32 power of two it stands for.  2^-127 has no exponent field of its own; 255 gives an infinity, whose field the conversions below take as NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u); }
// Scale byte of a block whose largest magnitude has these fp32 bits: the exponent field less 2 (e2m1 reaches 2^2), where infinities and NaN, whose bits are
// above all others', are NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  const uint32_t f = amax_bits >> 23;
  return f == 255 ? 255 : f > 2 ? f - 2 : 0;
}

// codes 2 I and 2 I + 1 of eight (elements in order, the first in the low four bits) -> two bf16 values
template <int I>
__device__ __forceinline__ uint32_t to_bf16x2(uint32_t c, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, I));
}
// eight codes (elements in order, the first in the low four bits) -> bf16 values
__device__ __forceinline__ u32x4 to_bf16(uint32_t c, float s) {
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return o;
}
__device__ __forceinline__ void to_f32(uint32_t c, float s, float (&v)[8]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
}
// eight fp32 values -> codes: nearest, ties to the even code, saturating, sign kept
__device__ __forceinline__ uint32_t to_codes(const float (&v)[8], float s) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return c;
}

}  // namespace mx4
}  // namespace poetx
