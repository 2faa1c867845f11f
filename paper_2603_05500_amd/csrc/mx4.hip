// Weights and activations in four bits: a matrix into codes and power-of-two scales, and back.
//
// Both kernels are plain streams: sixteen lanes take a unit of 128 columns, eight elements each, so that every access of a wave is
// contiguous (quantising bf16: 1 KB in, 256 bytes of codes and 16 of scales out).  Four lanes share a block of 32 and its largest magnitude.  The rounding is the hardware's
// (v_cvt_scalef32_pk_fp4_f32), which was compared with the definition on every bf16 value and around every tie.
// Bound by bytes: 14336 x 4096 bf16 to codes 31 us (4.8 TB/s), back 23 (its codes in the Infinity Cache).
#include "edge_gemm.h"
#include "grouped.h"
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

// Eight elements of a lane, sixteen lanes a unit -> the lane's codes and, in every lane, the unit's four scale bytes.
__device__ __forceinline__ uint32_t quantise_unit(const float (&v)[8], int lane, uint32_t& word) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
    top = a > top ? a : top;
  }
#pragma unroll
  for (int s = 1; s < 4; s *= 2) {
    const uint32_t o = __shfl_xor(top, s);
    top = o > top ? o : top;
  }
  const uint32_t sb = mx4::scale_byte(top);
  word = sb << (8 * (lane >> 2));      // this block's byte of the four
  word |= __shfl_xor(word, 4);
  word |= __shfl_xor(word, 8);
  return sb == 255 ? 0 : mx4::to_codes(v, mx4::scale_of(sb));
}

// Every row of X, `total` units, or (GROUPS) those that some group has: from the first offset to the furthest (0.2
// to 0.3 us of a product of a handful of rows, with the loads ahead of the second as well).
template <class T, bool GROUPS>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const T* __restrict__ X, i64 ld, int cols, int upr, i64 total, uint32_t* __restrict__ codes,
                                                           uint32_t* __restrict__ scales, int block0, const int32_t* offsets, int groups, i64 rows) {
  const int lane = threadIdx.x & 15;
  const i64 first = (i64)(block0 + blockIdx.x) * (16 * UPL) + (threadIdx.x >> 4);
  i64 u0 = 0, u1 = total;
  if constexpr (GROUPS) {
    u0 = (i64)grouped::offset_at(offsets, 0, rows) * upr;
    u1 = (i64)grouped::furthest_end(offsets, groups, rows) * upr;
  }
  float v[UPL][8];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    const bool on = u >= u0 && u < u1;
    const i64 row = on ? u / upr : 0;
    load8(X + row * ld, on ? (int)(u - row * upr) * mx4::UNIT + 8 * lane : cols, cols, v[p]);
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = first + 16 * p;
    uint32_t word;
    const uint32_t c = quantise_unit(v[p], lane, word);
    if (u >= u0 && u < u1) {
      codes[u * 16 + lane] = c;
      if (lane == 0) scales[u] = word;
    }
  }
}

// One matrix, or (GROUPS) the weights of the groups that have rows: `total` units each.
template <class T, bool GROUPS>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int cols, int upr, i64 total,
                                                             T* __restrict__ out, i64 ld, int block0, const int32_t* offsets, i64 rows, int per_group) {
  const int lane = threadIdx.x & 15;
  i64 block = block0 + (i64)blockIdx.x, base = 0;
  if constexpr (GROUPS) {
    const int g = (int)(block / per_group);
    const grouped::Range r = grouped::own_range(offsets, g, rows);
    if (r.r0 == r.r1) return;
    block -= (i64)g * per_group;
    base = g * total;
  }
  const i64 first = block * (16 * UPL) + (threadIdx.x >> 4);
  uint32_t c[UPL], sb[UPL];
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    const i64 u = base + (first + 16 * p < total ? first + 16 * p : total - 1);
    c[p] = codes[u * 16 + lane];
    sb[p] = scales[u * 4 + (lane >> 2)];
  }
#pragma unroll
  for (int p = 0; p < UPL; ++p) {
    if (first + 16 * p >= total) continue;
    const i64 u = base + first + 16 * p, row = u / upr;
    const int k = (int)(u - row * upr) * mx4::UNIT + 8 * lane;
    if (k >= cols) continue;
    float v[8];
    mx4::to_f32(c[p], mx4::scale_of(sb[p]), v);
    edge::store8(out + row * ld + k, v, cols - k);
  }
}

// What the streaming product of two 4-bit operands reads, in one launch: the rows of X as codes [rows][units] of 64 bytes, and both operands' scales in the order
// in which its fragments take them (mx4.h).  Read from a buffer's rows, 4 bytes of a line each, the scales were half of the product's requests to L2, and a byte per fragment from LDS
// a sixth of its time: 16384 x 4096 times 14336 x 4096 with scales in rows, in words by unit, so: 708, 594, 465 us for the product; this launch takes 50 to 55 there.
// Workgroups below `quantising` take 64 positions x UPL units of X, the others 64 rows x 64 units of the weight's scales.
struct OperandArgs {
  const uint16_t* X;
  i64 ld, rows;
  int cols, units;
  const int32_t* offsets;
  int groups, n;
  uint32_t* codes;
  uint32_t* xs;
  const uint32_t* ws;
  uint32_t* wst;
  int quantising;
};
__global__ __launch_bounds__(256) void mx4_operands_kernel(OperandArgs a, int block0) {
  __shared__ uint32_t t[64][65];
  const int tid = threadIdx.x, lane = tid & 63;
  int bx = block0 + (int)blockIdx.x;
  if (bx < a.quantising) {
    const int across = (a.units + UPL - 1) / UPL, u0 = bx % across * UPL;
    const i64 p0 = (i64)(bx / across) * 64;
    // the group that has these positions, if any
    int local = -1, r0 = 0, r1 = 0, end = 0;
    for (int base = 0; base < a.groups && local < 0; base += 64) {
      const grouped::Range r = grouped::in_order(grouped::lane_offsets(a.offsets, a.groups, a.rows, base), end);
      const i64 at = p0 - mx4::position(r.r0, base + lane);
      const uint64_t has = __ballot(at >= 0 && at < r.r1 - r.r0);
      if (has) {
        const int l = __builtin_ctzll(has);
        r0 = __builtin_amdgcn_readlane(r.r0, l);
        r1 = __builtin_amdgcn_readlane(r.r1, l);
        local = __builtin_amdgcn_readlane((int)at, l);
      }
    }
    if (local < 0) return;
    const int l16 = tid & 15;
    uint8_t* sc = (uint8_t*)&t[0][0];
    float v[4][UPL][8];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const i64 row = r0 + local + 16 * s + (tid >> 4);
#pragma unroll
      for (int p = 0; p < UPL; ++p)
        load8(a.X + (row < r1 ? row : 0) * a.ld, row < r1 && u0 + p < a.units ? (u0 + p) * mx4::UNIT + 8 * l16 : a.cols, a.cols, v[s][p]);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const i64 row = r0 + local + 16 * s + (tid >> 4);
#pragma unroll
      for (int p = 0; p < UPL; ++p) {
        uint32_t word;
        const uint32_t c = quantise_unit(v[s][p], l16, word);
        if (row < r1 && u0 + p < a.units) a.codes[(row * a.units + u0 + p) * 16 + l16] = c;
        if ((l16 & 3) == 0) sc[p * 256 + mx4::scale_place(16 * s + (tid >> 4), l16 >> 2)] = (uint8_t)(word >> (2 * l16));
      }
    }
    __syncthreads();
    const i64 positions = mx4::positions(a.rows, a.groups);
    if (tid < 64 * UPL && u0 + tid / 64 < a.units) a.xs[(u0 + tid / 64) * positions + p0 + lane] = ((uint32_t*)sc)[tid];
    return;
  }
  bx -= a.quantising;
  const int across = (a.units + 63) / 64, u0 = bx % across * 64, blocks = (a.n + 63) / 64, block = bx / across, gr = block / blocks, i0 = block % blocks * 64;
  const uint32_t* w = a.ws + ((i64)gr * a.n + i0) * a.units + u0;
  for (int i = tid >> 6; i < 64; i += 4) t[i][lane] = i0 + i < a.n && u0 + lane < a.units ? w[(i64)i * a.units + lane] : 0;
  __syncthreads();
  for (int i = tid >> 6; i < 64 && u0 + i < a.units; i += 4) {
    uint32_t word = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) word |= (t[16 * s + (lane & 15)][i] >> (8 * (lane >> 4)) & 255) << (8 * s);
    a.wst[((i64)(u0 + i) * a.groups * blocks + block) * 64 + lane] = word;
  }
}

}  // namespace

void mx4_operands_launch(const void* X, i64 rows, int cols, i64 ld, const int32_t* offsets, int groups, int n, const void* Wq, void* codes, void* xs, void* wst,
                         hipStream_t st) {
  const int units = mx4::units(cols);
  const i64 q = mx4::positions(rows, groups) / 64 * ((units + UPL - 1) / UPL), w = (i64)groups * ((n + 63) / 64) * ((units + 63) / 64);
  const OperandArgs a{(const uint16_t*)X, ld, rows, cols, units, offsets, groups, n, (uint32_t*)codes, (uint32_t*)xs,
                      (const uint32_t*)mx4::view(Wq, (i64)groups * n, cols).scales, (uint32_t*)wst, (int)q};
  launch_in_rows(q + w, [&](int block0, unsigned count) { hipLaunchKernelGGL(mx4_operands_kernel, dim3(count), dim3(256), 0, st, a, block0); });
}

void mx4_quantize_launch(int dtype, const void* X, i64 rows, int cols, i64 ld, void* Q, hipStream_t st, const int32_t* offsets, int groups) {
  const int upr = mx4::units(cols);
  const i64 total = rows * upr;
  uint32_t *codes = (uint32_t*)Q, *scales = (uint32_t*)((char*)Q + mx4::scale_offset(rows, cols));
  auto go = [&](auto kern, auto* x) {
    launch_in_rows((total + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, x, ld, cols, upr, total, codes, scales, block0, offsets, groups, rows);
    });
  };
  if (dtype == POETX_F32) go(mx4_quantize_kernel<float, false>, (const float*)X);
  else if (offsets) go(mx4_quantize_kernel<uint16_t, true>, (const uint16_t*)X);
  else go(mx4_quantize_kernel<uint16_t, false>, (const uint16_t*)X);
}

void mx4_dequantize_launch(const void* Q, i64 rows, int cols, int dtype, void* out, i64 ld, hipStream_t st) {
  const int upr = mx4::units(cols);
  const i64 total = rows * upr;
  const mx4::View q = mx4::view(Q, rows, cols);
  auto go = [&](auto kern, auto* o) {
    launch_in_rows((total + 16 * UPL - 1) / (16 * UPL), [&](int block0, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, (const uint32_t*)q.codes, q.scales, cols, upr, total, o, ld, block0, nullptr, 0, 0);
    });
  };
  if (dtype == POETX_F32) go(mx4_dequantize_kernel<float, false>, (float*)out);
  else go(mx4_dequantize_kernel<uint16_t, false>, (uint16_t*)out);
}

void mx4_dequantize_groups_launch(const void* Q, int groups, int n, int cols, const int32_t* offsets, i64 rows, void* out, hipStream_t st) {
  const int upr = mx4::units(cols);
  const i64 total = (i64)n * upr, per_group = (total + 16 * UPL - 1) / (16 * UPL);
  const mx4::View q = mx4::view(Q, (i64)groups * n, cols);
  launch_in_rows(per_group * groups, [&](int block0, unsigned count) {
    hipLaunchKernelGGL((mx4_dequantize_kernel<uint16_t, true>), dim3(count), dim3(256), 0, st, (const uint32_t*)q.codes, q.scales, cols, upr, total, (uint16_t*)out, (i64)cols,
                       block0, offsets, rows, (int)per_group);
  });
}

}  // namespace poetx
