// The 8-bit microscaled format on the device: where a buffer's parts lie, and its conversions.
#pragma once

#include "mx4.h"

namespace poetx {
namespace mx8 {

using mx4::UNIT;
using mx4::units;
__host__ __device__ inline size_t scale_offset(i64 rows, int cols) { return align256((size_t)rows * units(cols) * UNIT); }
inline size_t bytes(i64 rows, int cols) { return scale_offset(rows, cols) + (size_t)rows * units(cols) * 4; }
struct View {
  uint8_t* codes;
  uint32_t* scales;      // a word per unit
};
__host__ __device__ inline View view(const void* Q, i64 rows, int cols) { return View{(uint8_t*)Q, (uint32_t*)((uint8_t*)Q + scale_offset(rows, cols))}; }

// Scale byte of a block whose largest magnitude has these fp32 bits: its exponent field, which is 0 for what is below 2^-126 and 255 for infinities and NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) { return amax_bits >> 23; }

// x 2^(133 - scale) to the nearest whole number, ties to even, at most 127, in the low byte (two's complement): the sum with 3 2^22 is rounded to a whole number by the addition itself.
// Values of 2^-133 have no reciprocal in fp32: the exponent is added, not multiplied.
__device__ __forceinline__ uint32_t to_code(float x, uint32_t scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(x, 133 - (int)scale), -127.f, 127.f) + 12582912.f);
}
// Four of them, the first in the low byte.  All are 0 in a block that is not finite.
__device__ __forceinline__ uint32_t to_codes4(float a, float b, float c, float d, uint32_t scale) {
  const uint32_t lo = __builtin_amdgcn_perm(to_code(b, scale), to_code(a, scale), 0x0c0c0400), hi = __builtin_amdgcn_perm(to_code(d, scale), to_code(c, scale), 0x0c0c0400);
  return scale == 255 ? 0 : lo | hi << 16;
}
// the largest magnitude of two: its bits are above all others' where one is infinite or NaN
__device__ __forceinline__ float largest(float a, float b) {
  float r;
  asm("v_maximum3_f32 %0, |%1|, |%2|, |%2|" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float largest(float a, float b, float c) {
  float r;
  asm("v_maximum3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// of four, as bits
__device__ __forceinline__ uint32_t largest4(float a, float b, float c, float d) { return __builtin_bit_cast(uint32_t, largest(largest(a, b, c), d)); }
// code E of four
template <int E>
__device__ __forceinline__ float value(uint32_t codes, uint32_t scale) {
  const float v = __builtin_amdgcn_ldexpf((float)((int)(codes << (24 - 8 * E)) >> 24), (int)scale - 133);
  return scale == 255 ? __builtin_nanf("") : v;
}
__device__ __forceinline__ void values8(uint32_t lo, uint32_t hi, uint32_t scale, float (&v)[8]) {
  v[0] = value<0>(lo, scale), v[1] = value<1>(lo, scale), v[2] = value<2>(lo, scale), v[3] = value<3>(lo, scale);
  v[4] = value<0>(hi, scale), v[5] = value<1>(hi, scale), v[6] = value<2>(hi, scale), v[7] = value<3>(hi, scale);
}

// Eight elements of a lane, four lanes a block -> the lane's codes and the block's scale byte.
__device__ __forceinline__ void quantise8(const float (&v)[8], uint32_t (&codes)[2], uint32_t& sb) {
  const uint32_t t0 = largest4(v[0], v[1], v[2], v[3]), t1 = largest4(v[4], v[5], v[6], v[7]);
  uint32_t top = t0 > t1 ? t0 : t1;
#pragma unroll
  for (int s = 1; s < 4; s *= 2) {
    const uint32_t o = __shfl_xor(top, s);
    top = o > top ? o : top;
  }
  sb = scale_byte(top);
  codes[0] = to_codes4(v[0], v[1], v[2], v[3], sb);
  codes[1] = to_codes4(v[4], v[5], v[6], v[7], sb);
}
// The same of sixteen lanes, a unit -> in every lane, the unit's four scale bytes.
__device__ __forceinline__ void quantise_unit(const float (&v)[8], int lane16, uint32_t (&codes)[2], uint32_t& word) {
  uint32_t sb;
  quantise8(v, codes, sb);
  word = sb << (8 * (lane16 >> 2));
  word |= __shfl_xor(word, 4);
  word |= __shfl_xor(word, 8);
}

}  // namespace mx8
}  // namespace poetx
