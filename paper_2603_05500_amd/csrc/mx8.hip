// Activations in eight bits: a matrix into codes and power-of-two scales, and back.
//
// Plain streams, as of the 4-bit buffers: sixteen lanes take a unit of 128 columns, eight elements each, four lanes share a block of 32 and its largest magnitude.  The
// scale is that magnitude's exponent, so that a code is the element with another exponent, rounded to a whole number: no division, and reading it back is exact.
// Bound by bytes: 16384 x 4096 bf16 to codes 40 to 46 us (4.5 to 5 TB/s), back 30 (its codes in the Infinity Cache); 16384 x 14336 back 108 to 125 (5.7 to 6.6 TB/s).
#include "edge_gemm.h"
#include "grouped.h"
#include "mx8.h"

namespace poetx {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int UPL = 2;      // units per sixteen lanes, their loads in flight together

template <class T>
__global__ __launch_bounds__(256) void mx8_quantize_kernel(const T* __restrict__ X, i64 ld, int cols, int upr, i64 total, mx8::View q, int block0) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  float v[UPL][8];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    const bool on = u < total;
    const i64 row = on ? u / upr : 0;
    edge::load8(X + row * ld, on ? (int)(u - row * upr) * mx8::UNIT + 8 * lane : cols, cols, v[p]);
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    uint32_t c[2], word;
    mx8::quantise_unit(v[p], lane, c, word);
    if (u < total) {
      *reinterpret_cast<u32x2*>(q.codes + u * mx8::UNIT + 8 * lane) = u32x2{c[0], c[1]};
      if (lane == 0) q.scales[u] = word;
    }
  }
}

// Every row, or (offsets) those that weight gradients sum over.
template <class T>
__global__ __launch_bounds__(256) void mx8_dequantize_kernel(mx8::View q, int cols, int upr, i64 rows, T* __restrict__ out, i64 ld, int block0, const int32_t* offsets, int groups) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  i64 u0 = 0, u1 = rows * upr;
  if (offsets) {
    const grouped::Range own = grouped::own_rows(offsets, groups, rows);
    u0 = (i64)own.r0 * upr;
    u1 = (i64)own.r1 * upr;
  }
  u32x2 c[UPL];
  uint32_t sb[UPL];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p < u1 ? first + 16 * p : 0;      // some unit
    c[p] = *reinterpret_cast<const u32x2*>(q.codes + u * mx8::UNIT + 8 * lane);
    sb[p] = q.scales[u] >> (8 * (lane >> 2)) & 255;
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    if (u < u0 || u >= u1) continue;
    const i64 row = u / upr;
    const int k = (int)(u - row * upr) * mx8::UNIT + 8 * lane;
    if (k >= cols) continue;
    float v[8];
    mx8::values8(c[p][0], c[p][1], sb[p], v);
    edge::store8(out + row * ld + k, v, cols - k);
  }
}

// Rows of whole vectors from rows of any length and alignment: a vector a lane, zeros past the columns.  Every row, or (offsets) those that some group has, or (OWN) that weight gradients sum over.
template <class T, bool OWN>
__global__ __launch_bounds__(256) void relay_rows_kernel(const T* __restrict__ X, i64 ld, int cols, i64 rows, T* __restrict__ out, i64 ldo, int block0, const int32_t* offsets, int groups) {
  constexpr int V = 16 / sizeof(T);
  const i64 across = ldo / V, i = (block0 + (i64)blockIdx.x) * 256 + threadIdx.x, row = i / across;
  const int col = (int)(i - row * across) * V;
  grouped::Range all{0, (int)rows};
  if (offsets) all = OWN ? grouped::own_rows(offsets, groups, rows) : grouped::Range{grouped::offset_at(offsets, 0, rows), grouped::furthest_end(offsets, groups, rows)};
  if (row < all.r0 || row >= all.r1) return;
  *reinterpret_cast<edge::u32x4*>(out + row * ldo + col) = edge::load_branched(X + row * ld, col, cols, true);
}

}  // namespace

void relay_rows_launch(int dtype, const void* X, i64 rows, int cols, i64 ld, void* out, i64 ldo, hipStream_t st, const int32_t* offsets, int groups, bool own) {
  auto go = [&](auto* x, auto* o) {
    typedef std::remove_pointer_t<decltype(o)> T;
    auto kern = own ? relay_rows_kernel<T, true> : relay_rows_kernel<T, false>;
    launch_in_rows((rows * (ldo * (i64)sizeof(*o) / 16) + 255) / 256, [&](int block0, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, x, ld, cols, rows, o, ldo, block0, offsets, groups);
    });
  };
  dtype == POETX_F32 ? go((const float*)X, (float*)out) : go((const uint16_t*)X, (uint16_t*)out);
}

void mx8_quantize_launch(int dtype, const void* X, i64 rows, int cols, i64 ld, void* Q, hipStream_t st) {
  const int upr = mx8::units(cols);
  const i64 total = rows * upr;
  auto go = [&](auto* x) {
    launch_in_rows((total + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(mx8_quantize_kernel, dim3(count), dim3(256), 0, st, x, ld, cols, upr, total, mx8::view(Q, rows, cols), block0);
    });
  };
  dtype == POETX_F32 ? go((const float*)X) : go((const uint16_t*)X);
}

void mx8_dequantize_launch(const void* Q, i64 rows, int cols, int dtype, void* out, i64 ld, hipStream_t st, const int32_t* offsets, int groups) {
  const int upr = mx8::units(cols);
  auto go = [&](auto* o) {
    launch_in_rows((rows * upr + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(mx8_dequantize_kernel, dim3(count), dim3(256), 0, st, mx8::view(Q, rows, cols), cols, upr, rows, o, ld, block0, offsets, groups);
    });
  };
  dtype == POETX_F32 ? go((float*)out) : go((uint16_t*)out);
}

}  // namespace poetx
