// Weights and activations in four bits: a matrix into codes and power-of-two scales, and back.
//
// Both kernels are plain streams: sixteen lanes take a unit of 128 columns, eight elements each, so that every access of a wave is
// contiguous (quantising bf16: 1 KB in, 256 bytes of codes and 16 of scales out).  Four lanes share a block of 32 and its largest magnitude.  The rounding is the hardware's
// (v_cvt_scalef32_pk_fp4_f32), which was compared with the definition on every bf16 value and around every tie.
#include "edge_gemm.h"
#include "mx4.h"

namespace poetx {
namespace {

using edge::u32x4;

constexpr int UPL = 2;      // units per sixteen lanes, their loads in flight together

__device__ __forceinline__ void load8(const uint16_t* row, int c, int cols, float (&v)[8]) {
  const u32x4 x = edge::load_branched(row, c, cols, true);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, x[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, x[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* row, int c, int cols, float (&v)[8]) {
  const u32x4 x = edge::load_branched(row, c, cols, true), y = edge::load_branched(row, c + 4, cols, true);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = __builtin_bit_cast(float, (uint32_t)x[i]);
    v[4 + i] = __builtin_bit_cast(float, (uint32_t)y[i]);
  }
}

template <class T>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const T* __restrict__ X, i64 ld, int cols, int upr, i64 total, uint32_t* __restrict__ codes,
                                                           uint32_t* __restrict__ scales, int block0) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  float v[UPL][8];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    const i64 row = u < total ? u / upr : 0;
    const int c = u < total ? (int)(u - row * upr) * mx4::UNIT + 8 * lane : cols;
    load8(X + row * ld, c, cols, v[p]);
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = __builtin_bit_cast(uint32_t, v[p][e]) & 0x7fffffffu;
      top = a > top ? a : top;
    }
#pragma unroll
    for (int s = 1; s < 4; s *= 2) {
      const uint32_t o = __shfl_xor(top, s);
      top = o > top ? o : top;
    }
    const uint32_t sb = mx4::scale_byte(top);
    const uint32_t c = sb == 255 ? 0 : mx4::to_codes(v[p], mx4::scale_of(sb));
    uint32_t word = sb << (8 * (lane >> 2));      // this block's byte of the unit's four
    word |= __shfl_xor(word, 4);
    word |= __shfl_xor(word, 8);
    if (u < total) {
      codes[u * 16 + lane] = c;
      if (lane == 0) scales[u] = word;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int cols, int upr, i64 total,
                                                             T* __restrict__ out, i64 ld, int block0) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  uint32_t c[UPL], sb[UPL];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p < total ? first + 16 * p : total - 1;
    c[p] = codes[u * 16 + lane];
    sb[p] = scales[u * 4 + (lane >> 2)];
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    if (u >= total) continue;
    const i64 row = u / upr;
    const int k = (int)(u - row * upr) * mx4::UNIT + 8 * lane;
    if (k >= cols) continue;
    float v[8];
    mx4::to_f32(c[p], mx4::scale_of(sb[p]), v);
    edge::store8(out + row * ld + k, v, cols - k);
  }
}

}  // namespace

void mx4_quantize_launch(int dtype, const void* X, i64 rows, int cols, i64 ld, void* Q, hipStream_t st) {
  const int upr = mx4::units(cols);
  const i64 total = rows * upr;
  uint32_t *codes = (uint32_t*)Q, *scales = (uint32_t*)((char*)Q + mx4::scale_offset(rows, cols));
  auto go = [&](auto kern, auto* x) {
    launch_in_rows((total + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, x, ld, cols, upr, total, codes, scales, block0);
    });
  };
  if (dtype == POETX_F32) go(mx4_quantize_kernel<float>, (const float*)X);
  else go(mx4_quantize_kernel<uint16_t>, (const uint16_t*)X);
}

void mx4_dequantize_launch(const void* Q, i64 rows, int cols, int dtype, void* out, i64 ld, hipStream_t st) {
  const int upr = mx4::units(cols);
  const i64 total = rows * upr;
  const mx4::View q = mx4::view(Q, rows, cols);
  auto go = [&](auto kern, auto* o) {
    launch_in_rows((total + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, (const uint32_t*)q.codes, q.scales, cols, upr, total, o, ld, block0);
    });
  };
  if (dtype == POETX_F32) go(mx4_dequantize_kernel<float>, (float*)out);
  else go(mx4_dequantize_kernel<uint16_t>, (uint16_t*)out);
}

}  // namespace poetx
