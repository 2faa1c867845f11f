// The gated feed-forward block: what its kernels share.
//   G = X Wg^T, U = X Wu^T, H = act(G) U;   dG = dH U act'(G), dU = dH act(G)
// act(g) = g s(z), s the logistic function, z = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu in its tanh form, as (1 + tanh(z / 2)) / 2 = s(z)); so
// act'(g) = s (1 + g z'(g) (1 - s)).
#pragma once

#include "edge_gemm.h"
#include "grouped.h"
#include "mx8.h"

namespace poetx {
namespace gated {

// -z log2(e) = g (c1 + c3 g^2): both activations by the same instructions.  silu: c3 = -1e-38, nothing beside c1 wherever s is not 0 or 1, but no zero for an infinity to meet.
struct Act {
  float c1, c3;
};
inline Act act_of(int activation) { return activation == POETX_GATED_GELU ? Act{-2.3022081963f, -0.10294323954f} : Act{-1.4426950409f, -1e-38f}; }

// The larger of two, NaN if either is.
__device__ __forceinline__ float maximum(float a, float b) {
  float r;
  asm("v_maximum3_f32 %0, %1, %2, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// Its value and derivative.  Below -1e18 the value is that of -1e18, which is 0; beyond 1000 the derivative is 0 or 1 whatever g is, and 1 - s or s is zero.  NaN stays
// NaN.  exp and the reciprocal are the hardware's, a unit in the last place each; its rounded argument costs e^-z |z| 2^-24 of itself, times 4 for its roundings and constants.
__device__ __forceinline__ void act_both(Act k, float g, float& a, float& da) {
  const float lo = maximum(g, -1e18f);
  const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(lo * fmaf(k.c3, lo * lo, k.c1)));
  const float t = __builtin_amdgcn_fmed3f(g, -1000.f, 1000.f);
  a = lo * s;
  da = s * fmaf(t * fmaf(-3.f * 0.6931471806f * k.c3, t * t, -0.6931471806f * k.c1), 1.f - s, 1.f);
}
__device__ __forceinline__ float act_value(Act k, float g) {
  float a, da;
  act_both(k, g, a, da);
  return a;
}

// What a call makes of G and U
enum Mode { FWD, HOLD, HOLD_MX8, BWD };
constexpr int NONE = -1;      // kernels that also make plain products: no block
struct Out {
  void* H;            // BWD: may be null
  void* G;            // HOLD: G and U; BWD: dG and dU; HOLD_MX8: buffers
  void* U;
  const void* dH;     // BWD
  i64 ldh, ldgu, lddh;
  Act act;
};
struct Call {
  const void* X;
  const void* W;      // dense: groups x 2n x m, gate then up
  i64 ldx;
  const int32_t* offsets;
  i64 rows;
  int m, n, groups;
  Mode mode;
  Out out;
};

// Eight neighbouring columns of a row, from col on, in fp32 -> what the mode asks for.  g, u: G and U, changed; dh: dH (BWD).  HOLD_MX8: four lanes have the 32 columns of a block, all of
// which are here; columns past the last have codes of zero.
template <class T, Mode MODE>
__device__ __forceinline__ void emit8(const Out& o, i64 rows, int n, i64 row, int col, bool on, float (&g)[8], float (&u)[8], const float (&dh)[8]) {
  const int left = on ? n - col : 0;
  if constexpr (MODE == HOLD_MX8) {
    auto keep = [&](const float (&z)[8], const void* Q) __attribute__((always_inline)) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < left ? z[e] : 0.f;
      uint32_t codes[2], sb;
      mx8::quantise8(v, codes, sb);
      if (!on) return;
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      const mx8::View q = mx8::view(Q, rows, n);
      const i64 unit = row * mx8::units(n) + col / mx8::UNIT;
      *reinterpret_cast<u32x2*>(q.codes + unit * mx8::UNIT + col % mx8::UNIT) = u32x2{codes[0], codes[1]};
      if (col % 32 == 0) ((uint8_t*)q.scales)[unit * 4 + col % mx8::UNIT / 32] = (uint8_t)sb;
    };
    keep(g, o.G);
    keep(u, o.U);
  }
  if (left <= 0) return;
  if constexpr (MODE == HOLD) {
    edge::store8((T*)o.G + row * o.ldgu + col, g, left);
    edge::store8((T*)o.U + row * o.ldgu + col, u, left);
  }
  float h[8];
  if constexpr (MODE == BWD) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v, d;
      act_both(o.act, g[e], v, d);
      h[e] = v * u[e];
      g[e] = dh[e] * u[e] * d;
      u[e] = dh[e] * v;
    }
    edge::store8((T*)o.G + row * o.ldgu + col, g, left);
    edge::store8((T*)o.U + row * o.ldgu + col, u, left);
    if (!o.H) return;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = act_value(o.act, g[e]) * u[e];
  }
  edge::store8((T*)o.H + row * o.ldh + col, h, left);
}

// Where G and U come from: matrices of the type, 8-bit buffers, or fp32 sums of parts of the contraction, [split][rows][2n]
enum Source { SAME, MX8, SUMS };
struct In {
  const void* G;
  const void* U;
  i64 ld;
  int splits;         // SUMS
};
// a handful of rows per group, where grouped::few_supported() says so for 2n columns (grouped_few.hip): any sizes, strides and alignments; four: W is a 4-bit buffer
void few_launch(int dtype, bool four, const Call& c, hipStream_t st);
// W a 4-bit buffer, decoded on the way, and X of whole 16-byte vectors (grouped_values.hip).  False where another way is the better one: few_launch() if `few`, otherwise the weight written out
// first.  sums: the workspace for parts of the contraction, sums_bytes of it; scratch: what the other way has for its own
bool values_supported(const Call& c);
bool values_launch(const Call& c, bool few, void* sums, size_t sums_bytes, size_t scratch, hipStream_t st);
size_t values_parts_bytes(int m, int n, int groups, i64 rows, bool few, size_t scratch);
// X and W of whole 16-byte vectors (gated_stream.hip); k: of plan() for a forward of 2n columns
bool stream_supported(int dtype, const Call& c);
void stream_launch(int dtype, grouped::Kernel k, const Call& c, hipStream_t st);
void edge_launch(int dtype, grouped::Kernel k, const Call& c, hipStream_t st);      // any shape (gated_edge.hip)
// the rows that some group has, one pass over G and U (gated_rows.hip)
void rows_launch(int dtype, Source src, const In& in, const int32_t* offsets, int groups, i64 rows, int n, Mode mode, const Out& out, hipStream_t st);

}  // namespace gated
}  // namespace poetx
