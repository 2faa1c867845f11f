// Grouped products on the matrix cores, bf16, fp32 and of 4-bit operands: the kernel.
//   FWD     Z  (rows x n) = X  (rows x m) W_g^T      both operands contracted along their rows
//   INPUT   dX (rows x m) = dZ (rows x n) W_g        W_g over its strided index
//   WEIGHT  dW_g (n x m)  = dZ^T X over g's rows     both over their strided index; fp32 out
//
// The same persistent stream as the dense product's: one workgroup per CU, 4 waves (2 x 2), the operand stages of all the tiles a
// workgroup computes in one ring of LDS stages filled by direct-to-LDS loads well ahead of the multiplication and across tiles, fragments of the next stage read
// under the products of this one.  What differs:
//  - Which rows a tile has is only known on the device.  Each wave holds the groups' row ranges in registers (four groups per lane) and
//    finds a tile's group by ballots, once per tile on the loading side and once on the storing side.
//  - Groups end inside tiles, and contractions inside stages.  The loads go through buffer descriptors that end where the operand
//    does: what lies behind reads as zeros, on both operands, so that nothing of another group takes part.  Only the last stage of rows whose length is
//    no multiple of a stage needs a mask, the same 64 lanes for every load of it.  Past the last tile the descriptors are
//    empty: the number of loads in flight never changes and the last ones cost no traffic.
//  - A stage is 64 bytes of a row whatever they hold: 32 bf16, 16 fp32, or 128 codes with a word of four scales.  An MFMA of 16 x 16 x 128 codes takes as long
//    as one of 16 x 16 x 32 bf16: the same stream carries four times the products.  The fp32 ones take eight times as long for the bytes: smaller tiles and several
//    workgroups per CU.
// What bounds it: large bf16 products by power, as the dense one (16384 rows, 8 groups of 8192 x 4096: 960 to 1015 us, 1.08 to 1.15 PFLOP/s with the ragged tiles); products of codes by the
// loads of a stage, which take as long as its multiplications (16384 x 4096 by 14336 x 4096 465 us, 4.1 PFLOP/s; without loads 384); many small groups by the weights' bytes (8190 rows,
// 57 groups of 1376 x 2048, input gradient 92 to 103 us); weight gradients by their stores (8192 rows, 16 groups of 1376 x 2048 93 us for 180 MB).
#pragma once
#include <utility>

#include "grouped.h"
#include "mfma_dense_kernel.h"
#include "mx4.h"

namespace poetx {
namespace grouped {

using dense::floatx4;
using mm::bf16x8;
using mx4::u32x4;

enum Elem { BF16, F32, CODES };

// PARTS: fp32 sums of a range of the contraction go to `parts`, to be added up by another launch (bf16; fp32 needs no kernel of its own).
template <int BM_, int BN_, int NS_, Elem ELEM_, int PER_CU_ = 1, bool PARTS_ = false>
struct StreamTile {
  static constexpr int BM = BM_, BN = BN_, NS = NS_, NW = 4, PER_CU = PER_CU_;
  static constexpr Elem ELEM = ELEM_;
  static constexpr bool PARTS = PARTS_;
  static constexpr bool FP4 = ELEM == CODES;
  static constexpr int DEPTH = FP4 ? 128 : ELEM == F32 ? 16 : 32;      // elements of a stage
  static constexpr int SETS = 4, GROUPS = 64 * SETS;      // groups per lane, in all
  static constexpr int A_BYTES = BM * 64, B_BYTES = BN * 64, S_BYTES = FP4 ? (BM + BN) * 4 : 0, STAGE_BYTES = A_BYTES + B_BYTES + S_BYTES;
  static constexpr int TM = BM / 32, TN = BN / 32, MF = TM * TN * (ELEM == F32 ? 4 : 1);      // MFMAs of a stage; fp32: 4 of depth per MFMA
  static constexpr int RS = MF / (TM + TN) < 3 ? MF / (TM + TN) : 3;
  static constexpr int OUT_BYTES = ELEM == F32 || PARTS ? 0 : TN / 4 * 2048;
  static constexpr int LDS_BYTES = NS * STAGE_BYTES + NW * OUT_BYTES;
  static constexpr int IPWA = A_BYTES / 1024 / NW, IPWB = B_BYTES / 1024 / NW, IPWS = FP4 ? (BM + BN) / 256 : 0;
  static constexpr int LPT = IPWA + IPWB + IPWS;
  static constexpr int DS = MF / LPT;
  static_assert(!FP4 || (BM == BN && (BM + BN) % 256 == 0), "scale loads: as many for every wave, each of one operand");
  static_assert(NS * LPT < 64 && DS >= 1 && RS >= 1 && (TM + TN) * RS <= MF && (ELEM == F32 || TN % 4 == 0) && LDS_BYTES <= 160 * 1024, "stream tile");
};

struct StreamArgs {
  const char* A;          // FWD, INPUT: rows of X or dZ; WEIGHT: dZ.  FP4: codes
  const char* B;          // W, or X (WEIGHT).  FP4: codes
  const uint32_t* SA;     // FP4: scales, ordered as in mx4.h
  const uint32_t* SB;
  int sa_step, sb_step;   // bytes from unit to unit
  void* C;
  int lda, ldb, ldc;      // row strides: bytes of A and B, elements of C
  const int32_t* offsets;
  int rows, groups;
  int K;                  // FWD, INPUT: contraction, in elements (CODES: of whole units)
  int M, N;               // WEIGHT: rows of C (n); columns of C
  int tiles_n;            // column tiles
  int accumulate;
  int splits;             // FWD, INPUT: ranges of the contraction, whose sums go to [split][rows][N] at C; 1: the result does
};

// 16 (4) bytes per lane from base + voff straight into LDS at lds + 16 (4) * lane; zeros from the descriptor's end on.  Between M0's write and its use there has to be
// an instruction.
__device__ __forceinline__ void dma16b(const u32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void dma4b(const u32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds) : "memory");
}
// The same, the lanes in `off` behind the descriptor's end.
__device__ __forceinline__ void dma16b_but(uint64_t off, const u32x4& rsrc, uint32_t voff, uint32_t lds) {
  uint32_t v;
  asm volatile("v_cndmask_b32 %0, %1, %2, %3\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds" : "=&v"(v) : "v"(voff), "v"(0xfffffff0u), "s"(off), "s"(rsrc), "{m0}"(lds) : "memory");
}

// The same value in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ i64 uniform(i64 v) { return (i64)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v)); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) { return (uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v); }

// One operand of the tile in issue: where its next stage starts and how many bytes there are from there on (of rows along the contraction: of a tile's
// height of them, which is less than 2^31).
template <class Left>
struct Feed {
  uint64_t at;
  Left left;
  __device__ __forceinline__ uint32_t bytes(bool on) const {      // none if !on
    if constexpr (sizeof(Left) == 4) return (uint32_t)uniform(on && left > 0 ? (int)left : 0);
    const int high = (int)((i64)left >> 32);      // compared in halves: there is no scalar comparison of 64 bits
    const uint32_t low = (uint32_t)left, most = 0x7ffffff0u;      // a stage or a tile spans less
    return (uint32_t)uniform((int)(high < 0 || !on ? 0u : high > 0 || low > most ? most : low));
  }
  __device__ __forceinline__ void base(u32x4& r) const { r[0] = (uint32_t)uniform((int)at), r[1] = (uint32_t)uniform((int)(at >> 32)) & 0xffffu, r[3] = 0x00020000u; }
  __device__ __forceinline__ void step(Left bytes) {
    at += bytes;
    left -= bytes;
  }
};

constexpr int kNowhere = 0x7ffffff0;      // an offset behind every descriptor
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(void* p, i64 bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, (short)0, bytes <= 0 ? 0 : (int)(bytes < kNowhere ? bytes : kNowhere), 0x00020000);
}

// c += a b on 16 x 16 x 128 codes; SA, SB: which byte of a lane's words scales its 32 codes
template <int SA, int SB>
__device__ __forceinline__ void mfma_fp4(floatx4& c, const u32x4& a, const u32x4& b, uint32_t sa, uint32_t sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:4 blgp:4"
               : "+a"(c)
               : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(SA & 1), "n"(SB & 1), "n"(SA >> 1), "n"(SB >> 1));
}
// c += a b on 16 x 16 x 4 fp32
__device__ __forceinline__ void mfma_fp32(floatx4& c, uint32_t a, uint32_t b) { asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }

// f(0), f(1), .. as constants
template <int... I, class F>
__device__ __forceinline__ void in_turn(std::integer_sequence<int, I...>, const F& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <Dir DIR, class C>
__global__ __launch_bounds__(256) void grouped_stream_kernel(StreamArgs g) {
  constexpr bool FP4 = C::FP4, FP32 = C::ELEM == F32, A_K = DIR != WEIGHT, B_K = DIR == FWD;
  // WIDE: rows come 64 deep, whole 128-byte lines.  Two stages are a unit, which arrives in two halves of its rows, one per stage; as it is needed as a whole, and its
  // place is free, with its first stage, the last half is in flight a stage less, and the ring has to be deep.  As in the dense product, 64-byte pieces would ask for every line twice.
  constexpr bool WIDE = A_K && B_K && C::ELEM == BF16 && C::NS >= 6;
  constexpr int DEPTH = C::DEPTH, ES = FP32 ? 4 : 2;      // bytes of an element (not of a code)
  static_assert(!FP4 || DIR == FWD, "codes are contracted along their rows");
  constexpr int BM = C::BM, BN = C::BN, NS = C::NS, STAGE_BYTES = C::STAGE_BYTES, A_BYTES = C::A_BYTES;
  constexpr int IPWA = C::IPWA, IPWB = C::IPWB, IPWS = C::IPWS, LPT = C::LPT, TM = C::TM, TN = C::TN, MF = C::MF, RS = C::RS, DS = C::DS;
  constexpr int GROUP = dense::GROUP;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // ---- the groups: lane l of set q has group 64 q + l
  constexpr int kTableSets = C::SETS;
  int tr0[kTableSets], tr1[kTableSets], tsum[kTableSets];
  int row_tiles = 0, end = 0;
  Range own[kTableSets];
#pragma unroll
  for (int q = 0; q < kTableSets; ++q) {
    const int gr = 64 * q + lane;
    own[q] = Range{0, 0};
    if (DIR == WEIGHT && gr < g.groups) own[q] = own_range(g.offsets, gr, g.rows);
    if (DIR != WEIGHT && 64 * q < g.groups) own[q] = lane_offsets(g.offsets, g.groups, g.rows, 64 * q);
  }
#pragma unroll
  for (int q = 0; q < kTableSets; ++q) {
    const Range r = DIR != WEIGHT && 64 * q < g.groups ? in_order(own[q], end) : own[q];
    tr0[q] = r.r0;
    tr1[q] = r.r1;
    tsum[q] = 0;
    if (DIR != WEIGHT && 64 * q < g.groups) {
      tsum[q] = row_tiles + wave_scan((r.r1 - r.r0 + BM - 1) / BM);
      row_tiles = __builtin_amdgcn_readlane(tsum[q], 63);
    }
  }
  const int tiles_m = DIR == WEIGHT ? (g.M + BM - 1) / BM : row_tiles;      // WEIGHT: of one group
  const int per_weight = tiles_m * g.tiles_n;
  const int T = per_weight * (DIR == WEIGHT ? g.groups : g.splits);
  const int G = gridDim.x;
  // WEIGHT: a group's tiles take as long as it has rows.  Groups go by their size, the largest first, and workgroups through every other round backwards, so that their shares are
  // alike: 8192 rows, 15 of 16 groups of 1376 x 2048 that have 340 to 1200 of them each, 76 us as they come, 71 so.  Over many rounds shares are alike anyway (12 of 64 groups: 137, 139).
  // tsum: how many groups come before.
  const bool by_size = DIR == WEIGHT && g.groups <= 64 && T < 8 * G;
  if (by_size) {
    const int mine = tr1[0] - tr0[0];
    for (int j = 0; j < g.groups; ++j) {
      const int other = __builtin_amdgcn_readlane(mine, j);
      tsum[0] += other > mine || (other == mine && j < lane);
    }
  }
  int wq = blockIdx.x;
  if ((G & 7) == 0) wq = (wq & 7) * (G >> 3) + (wq >> 3);
  auto place = [&](int ti) { return DIR == WEIGHT && (ti & 1) ? G - 1 - wq : wq; };      // in a round
  const int n_my = T / G + (place(T / G) < T % G);
  if (n_my == 0) return;

  struct Where {
    int gr, first, r0, r1;      // group, its first row; FWD, INPUT: the tile's first row; WEIGHT: the group's; end of the group
    int i0, j0;          // WEIGHT: first row of C; first column
    int split, k0, k1;   // range of the contraction and its stages, in pairs from the first on
  };
  auto locate = [&](int ti) __attribute__((always_inline)) {
    Where w;
    int u = ti * G + place(ti);
    w.gr = w.split = 0;
    if (DIR == WEIGHT) {
      w.gr = u / per_weight;
      u -= w.gr * per_weight;
      if (by_size) w.gr = __builtin_ctzll(__ballot(tsum[0] == w.gr));
    } else if (g.splits > 1) {
      w.split = u / per_weight;
      u -= w.split * per_weight;
    }
    const int per_group = GROUP * g.tiles_n;
    const int first_m = (u / per_group) * GROUP;
    const int gsz = (tiles_m - first_m) < GROUP ? (tiles_m - first_m) : GROUP;
    const int rt = first_m + (u % per_group) % gsz;
    w.j0 = ((u % per_group) / gsz) * BN;
    w.i0 = rt * BM;
    w.first = w.r0 = w.r1 = 0;
    if (DIR == WEIGHT) {
#pragma unroll
      for (int q = 0; q < kTableSets; ++q)
        if (w.gr >> 6 == q) {
          w.r0 = __builtin_amdgcn_readlane(tr0[q], w.gr & 63);
          w.r1 = __builtin_amdgcn_readlane(tr1[q], w.gr & 63);
        }
      w.k0 = 0;
      w.k1 = (w.r1 - w.r0 + 2 * DEPTH - 1) / (2 * DEPTH) * 2;
    } else {
      bool found = false;
#pragma unroll
      for (int q = 0; q < kTableSets; ++q) {
        const uint64_t after = __ballot(tsum[q] > rt);      // the sums of lanes without a group repeat the last one's
        if (!found && 64 * q < g.groups && after) {
          found = true;
          const int l = __builtin_ctzll(after);
          w.gr = 64 * q + l;
          w.r0 = __builtin_amdgcn_readlane(tr0[q], l);
          w.r1 = __builtin_amdgcn_readlane(tr1[q], l);
          w.first = w.r0;
          const int end = __builtin_amdgcn_readlane(tsum[q], l), mine = (w.r1 - w.r0 + BM - 1) / BM;
          w.r0 += (rt - (end - mine)) * BM;
        }
      }
      const int pairs = (g.K + 2 * DEPTH - 1) / (2 * DEPTH);
      w.k0 = pairs * w.split / g.splits * 2;
      w.k1 = pairs * (w.split + 1) / g.splits * 2;
    }
    return w;
  };

  // ---- per-lane byte offsets of the loads, the same for every stage and tile
  uint32_t voffA[IPWA], voffB[FP4 ? 1 : IPWB], voffS[IPWS ? IPWS : 1];      // FP4: both operands' rows are as long, and the tile square
  // Rows along the output: where chunk c of row k lies.  bf16: as the transposing loads like it; fp32: a fragment's four rows 4 q + e, q = 0 .. 3, in four different 64 bytes.
  auto strided_chunk = [&](int c, int k) __attribute__((always_inline)) { return FP32 ? c ^ (4 * ((k >> 2) & 3)) : dense::kx16_chunk(c, k); };
  auto slot_offset = [&](int slot, bool kmajor, int width, int ld) __attribute__((always_inline)) {
    if (WIDE) {
      const int r = slot >> 3, c = (slot & 7) ^ ((r >> 1) & 7);
      return (uint32_t)(r * ld + c * 16);
    }
    if (kmajor) {
      const int r = slot >> 2, c = dense::xk16_chunk(slot & 3, r);
      return (uint32_t)(r * ld + c * 16);
    }
    const int k = slot / (width * ES / 16), c = strided_chunk(slot % (width * ES / 16), k);
    return (uint32_t)(k * ld + c * 16);
  };
#pragma unroll
  for (int s = 0; s < IPWA; ++s) voffA[s] = slot_offset((wave * IPWA + s) * 64 + lane, A_K, BM, g.lda);
#pragma unroll
  for (int s = 0; s < (FP4 ? 0 : IPWB); ++s) voffB[s] = slot_offset((wave * IPWB + s) * 64 + lane, B_K, BN, g.ldb);
  // scales: the first two waves bring A's, the others B's
  const bool scales_a = wave < 2;
#pragma unroll
  for (int s = 0; s < IPWS; ++s) {
    const int r = (wave * IPWS + s) * 64 + lane;
    voffS[s] = (uint32_t)((r < BM ? r : r - BM) * 4);
  }
  // Lanes whose 16 bytes lie past the end of a row in its last, short stage (WIDE: unit): the chunk a lane fetches is the same in each of its loads (WIDE: in every other).
  constexpr int PIECE = WIDE ? 2 * DEPTH : DEPTH;
  const int short_piece = !FP4 && DIR != WEIGHT && g.K % PIECE ? g.K / PIECE : -1;
  uint64_t past_end[2];
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int c = WIDE ? (lane & 7) ^ ((lane >> 4) + 4 * o) : dense::xk16_chunk(lane & 3, lane >> 2);
    past_end[o] = __ballot(16 / ES * c >= g.K % PIECE);
  }

  // ---- issue side
  typedef typename std::conditional<A_K, int, i64>::type LeftA;
  typedef typename std::conditional<B_K, int, i64>::type LeftB;
  Feed<LeftA> fa;
  Feed<LeftB> fb;
  Feed<int> fs{0, 0};      // FP4: scales of the tile's rows in this stage
  const int step_s = scales_a ? g.sa_step : g.sb_step;
  int iti = -1, ikt = 0, iKT = 0, islot = 0;
  const LeftA stepA = A_K ? 64 : DEPTH * (LeftA)g.lda;
  const LeftB stepB = B_K ? 64 : DEPTH * (LeftB)g.ldb;
  const int halfA = WIDE ? BM / 2 * g.lda : 0, halfB = WIDE ? BN / 2 * g.ldb : 0;
  auto next_tile = [&]() __attribute__((always_inline)) {
    Where w;
    do {
      ++iti;
      if (iti >= n_my) break;
      w = locate(iti);
    } while (DIR == WEIGHT && w.k1 == 0);
    Feed<LeftA> na{0, 0};      // nothing more: empty descriptors
    Feed<LeftB> nb{0, 0};
    int k0 = 0, k1 = 0x7fffffff, ha = 0, hb = 0;
    uint64_t nsa = 0, nsb = 0;
    if (iti < n_my) {
      k0 = w.k0;
      k1 = w.k1;
      if (DIR == FWD) hb = g.N - w.j0 < BN ? g.N - w.j0 : BN;      // rows of W in the tile
      if (DIR == WEIGHT) {
        const i64 len = w.r1 - w.r0;
        na.at = (uint64_t)(g.A + (i64)w.r0 * g.lda + ES * w.i0);
        na.left = (len - 1) * (i64)g.lda + ES * (i64)(g.M - w.i0);
        nb.at = (uint64_t)(g.B + (i64)w.r0 * g.ldb + ES * w.j0);
        nb.left = (len - 1) * (i64)g.ldb + ES * (i64)(g.N - w.j0);
      } else {
        ha = w.r1 - w.r0 < BM ? w.r1 - w.r0 : BM;
        const int row = FP4 ? g.K / 2 : ES * g.K;      // bytes of a row
        na.at = (uint64_t)(g.A + (i64)w.r0 * g.lda);
        na.left = (ha - 1) * (LeftA)g.lda + row;
        if (DIR == FWD) {
          const i64 first = (i64)w.gr * g.N + w.j0;
          nb.at = (uint64_t)(g.B + first * g.ldb);
          nb.left = (hb - 1) * (LeftB)g.ldb + row;
          nsa = (uint64_t)(g.SA + mx4::position(w.first, w.gr) + (w.r0 - w.first));      // a word per row
          nsb = (uint64_t)(g.SB + (i64)w.gr * ((g.N + 63) / 64 * 64) + w.j0);
        } else {
          nb.at = (uint64_t)(g.B + (i64)w.gr * g.K * g.ldb + ES * w.j0);
          nb.left = (i64)(g.K - 1) * g.ldb + ES * (i64)(g.N - w.j0);
        }
      }
    }
    if (DIR != WEIGHT) {
      na.step(k0 * stepA);
      nb.step(k0 * stepB);
      nsa += (i64)k0 * g.sa_step;
      nsb += (i64)k0 * g.sb_step;
    }
    ikt = uniform(k0);
    iKT = uniform(k1);
    fa = Feed<LeftA>{uniform(na.at), uniform(na.left)};
    fb = Feed<LeftB>{uniform(nb.at), uniform(nb.left)};
    fb.step(-(WIDE ? 2 * stepB - halfB : stepB));      // the step to the tile's first stage is yet to come
    if (FP4) {
      fs = Feed<int>{uniform(scales_a ? nsa : nsb) - step_s, uniform(((scales_a ? ha : hb) + 63) / 64 * 256)};
    }
  };
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  u32x4 ra{}, rb{}, rs{};
  uint64_t masked_a[2] = {0, 0}, masked_b[2] = {0, 0};
  uint32_t slot_a = lds_base, slot_b = lds_base + (WIDE ? 2 * A_BYTES : A_BYTES);      // where the operands' stage in issue goes
  // The descriptors of a stage come a few instructions at a time, between the multiplications of another: A's for the next stage once its loads of this one are out, B's and the
  // scales' for this one ahead of their first load.  All at once they held up the next multiplications (fp32 4096 rows, 4 groups of 2048 x 2048 384 us, 345 so;
  // codes 16384 x 4096 by 14336 x 4096 532, 521 with their quantising; bf16, bound by LDS on small tiles and by power on large ones, the same).  WIDE: the stages of a unit are the halves of its rows.
  auto bytes_on = [&](int kt) __attribute__((always_inline)) { return kt * DEPTH < g.K; };      // not a stage that only evens their number (WEIGHT: has no rows)
  auto mask = [&](uint64_t (&m)[2], int kt) __attribute__((always_inline)) {
    const bool is_short = (WIDE ? kt >> 1 : kt) == short_piece;
    m[0] = is_short ? past_end[0] : 0;
    if (WIDE) m[1] = is_short ? past_end[1] : 0;
  };
  auto set_a = [&](int part, int kt) __attribute__((always_inline)) {
    if (part == 0) fa.base(ra);
    if (part == 1) ra[2] = fa.bytes(WIDE || !A_K || bytes_on(kt));
    if (part == 2 && A_K && !FP4) mask(masked_a, kt);
  };
  auto next_a = [&](int part) __attribute__((always_inline)) {      // parts 0 .. 3
    if (part == 0) fa.step(WIDE ? (ikt & 1 ? 2 * stepA - halfA : (LeftA)halfA) : stepA);
    else set_a(part - 1, ikt + 1);
  };
  auto next_b = [&](int part) __attribute__((always_inline)) {      // parts 0 .. 5
    if (part == 0) fb.step(WIDE ? (ikt & 1 ? (LeftB)halfB : 2 * stepB - halfB) : stepB);
    if (part == 1) fb.base(rb);
    if (part == 2) rb[2] = fb.bytes(WIDE || !B_K || bytes_on(ikt));
    if (part == 3 && B_K && !FP4) mask(masked_b, ikt);
    if (FP4 && part == 4) {
      fs.at += step_s;
      fs.base(rs);
    }
    if (FP4 && part == 5) rs[2] = fs.bytes(bytes_on(ikt));
  };
  static_assert(IPWA * DS >= 6 && IPWA * DS + 4 <= MF, "B's descriptor ahead of its loads, A's behind its own");
  static_assert(!WIDE || (IPWA % 2 == 0 && IPWB % 2 == 0), "a wave's loads start with an even one");
  auto issue = [&](int i) __attribute__((always_inline)) {      // load i of the stage (a constant wherever this is called)
    if (i < IPWA) {
      const uint32_t at = slot_a + (wave * IPWA + i) * 1024;
      if (!FP4 && A_K) dma16b_but(masked_a[WIDE ? i & 1 : 0], ra, voffA[i], at);
      else dma16b(ra, voffA[i], at);
    } else if (i < IPWA + IPWB) {
      const int l = i - IPWA;
      const uint32_t at = slot_b + (wave * IPWB + l) * 1024;
      if (!FP4 && B_K) dma16b_but(masked_b[WIDE ? l & 1 : 0], rb, voffB[l], at);
      else dma16b(rb, FP4 ? voffA[l] : voffB[l], at);
    } else {
      const int s = i - IPWA - IPWB;
      dma4b(rs, voffS[s], slot_b + C::B_BYTES + (wave * IPWS + s) * 256);
    }
  };
  auto issue_advance = [&]() __attribute__((always_inline)) {
    islot = islot + 1 == NS ? 0 : islot + 1;
    ++ikt;
    slot_a = lds_base + (WIDE ? (islot >> 1) * 2 * STAGE_BYTES + (islot & 1) * A_BYTES : islot * STAGE_BYTES);
    slot_b = WIDE ? lds_base + (islot >> 1) * 2 * STAGE_BYTES + 2 * A_BYTES + (islot & 1) * C::B_BYTES : slot_a + A_BYTES;
  };
  auto start_tile = [&]() __attribute__((always_inline)) {
    next_tile();
#pragma unroll
    for (int i = 0; i < 3; ++i) set_a(i, ikt);
  };
  // after every second stage: tiles have even numbers of them, and so has the ring (WIDE, a stage behind: after the first of a pair of multiplications)
  static_assert(NS % 2 == 0, "a tile's first stage is issued first of a pair");
  auto tile_advance = [&]() __attribute__((always_inline)) {
    if (ikt == iKT) start_tile();
  };

  // ---- fragments
  // K major: the 16-row pieces lie 1024 (WIDE: 2048) bytes apart, as their swizzle is the same
  constexpr int PIECE_BYTES = WIDE ? 2048 : 1024, B_AT = WIDE ? 2 * A_BYTES : A_BYTES;
  int fragA[A_K ? 1 : TM], fragB[B_K ? 1 : TN];
  const int q4 = lane >> 4, li = lane & 15;
  {
    const int k = 8 * q4 + (li >> 2);
    auto frag = [&](int x0, bool kmajor, int width) {
      if (WIDE) return (x0 + li) * 128 + 16 * (q4 ^ (li >> 1));      // of a unit's first stage; the second's chunks are 4 further, bit 2 of the position
      if (kmajor) return (x0 + li) * 64 + 16 * dense::xk16_chunk(q4, li);
      if (FP32) return 4 * q4 * (width * 4) + 16 * strided_chunk((x0 + li) >> 2, 4 * q4) + 4 * (li & 3);
      return k * (width * 2) + 16 * dense::kx16_chunk((x0 >> 3) + ((li & 3) >> 1), k) + 8 * (li & 1);
    };
#pragma unroll
    for (int a = 0; a < (A_K ? 1 : TM); ++a) fragA[a] = frag(wm * (BM / 2) + a * 16, A_K, BM);
#pragma unroll
    for (int c = 0; c < (B_K ? 1 : TN); ++c) fragB[c] = B_AT + frag(wn * (BN / 2) + c * 16, B_K, BN);
  }
  const int scaleA = A_BYTES + C::B_BYTES + wm * (BM / 2) * 4 + lane * 4, scaleB = A_BYTES + C::B_BYTES + (BM + wn * (BN / 2)) * 4 + lane * 4;
  auto load_frag = [&](const char* p, bool kmajor, int row_bytes) -> u32x4 {
    if (kmajor) return *reinterpret_cast<const u32x4*>(p);
    if constexpr (FP32) {      // row_bytes: of a row of bf16
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint32_t*>(p + e * 2 * row_bytes);
      return v;
    }
    const mm::short4v lo = mm::lds_read_tr(p), hi = mm::lds_read_tr(p + 4 * row_bytes);
    const mm::short8v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(u32x4, v);
  };
  struct Frags {
    u32x4 a[TM], b[TN];
    uint32_t sa[(TM + 3) / 4], sb[(TN + 3) / 4];      // CODES: a byte per piece
  };
  // piece p, in the order the MFMAs first need them: A0 B0 A1 .. A(TM-1) B1 .. B(TN-1); odd: of the second stage of a unit
  auto load_piece = [&](Frags& f, int slot, int p, bool odd) __attribute__((always_inline)) {
    const char* st = lds + (WIDE ? slot & ~1 : slot) * STAGE_BYTES;
    const int flip = WIDE && odd ? 64 : 0;
    if (p != 1 && p <= TM) {
      const int a = p ? p - 1 : 0;
      f.a[a] = load_frag(st + (fragA[A_K ? 0 : a] ^ flip) + (A_K ? a * PIECE_BYTES : 0), A_K, BM * 2);
      if (FP4 && a % 4 == 0) f.sa[a / 4] = *reinterpret_cast<const uint32_t*>(st + scaleA + a * 64);
    } else {
      const int b = p == 1 ? 0 : p - TM;
      f.b[b] = load_frag(st + (fragB[B_K ? 0 : b] ^ flip) + (B_K ? b * PIECE_BYTES : 0), B_K, BN * 2);
      if (FP4 && b % 4 == 0) f.sb[b / 4] = *reinterpret_cast<const uint32_t*>(st + scaleB + b * 64);
    }
  };

  floatx4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int c = 0; c < TN; ++c) acc[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};

  start_tile();
#pragma unroll 1
  for (int t = 0; t < NS - (WIDE ? 1 : 0); ++t) {
#pragma unroll
    for (int i = 0; i < 6; ++i) next_b(i);
#pragma unroll
    for (int i = 0; i < LPT; ++i) issue(i);
#pragma unroll
    for (int i = 0; i < 4; ++i) next_a(i);
    issue_advance();
    tile_advance();
  }
  mm::wait_vmcnt_and_barrier<(WIDE ? NS - 3 : NS - 1) * LPT>();
  Frags F, Gf;
  int cslot = 0;
#pragma unroll
  for (int p = 0; p < TM + TN; ++p) load_piece(F, 0, p, false);

  // once per wave: wave W issues its loads W quarters of the way from one to the next
  auto run = [&](auto WC) __attribute__((always_inline)) {
    constexpr int W = decltype(WC)::value;
    auto multiply = [&](const Frags& X, Frags& Y, auto ODD) __attribute__((always_inline)) {      // ODD: the stage in X is the second of a unit
      constexpr bool odd = decltype(ODD)::value;
      // Every wave holds this stage in registers and the next one has landed (WIDE: with the other half of its unit).  Stages up to kt + NS - 1 are issued, WIDE one less.
      mm::wait_all_reads_and_barrier<(WIDE ? odd ? NS - 4 : NS - 3 : NS - 2) * LPT>();
      const int nslot = cslot + 1 == NS ? 0 : cslot + 1;
      in_turn(std::make_integer_sequence<int, MF>{}, [&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value, a = i % TM, b = i / TM % TN;
        if constexpr (FP4) mfma_fp4<b % 4, a % 4>(acc[a][b], X.b[b], X.a[a], X.sb[b / 4], X.sa[a / 4]);
        else if constexpr (FP32) mfma_fp32(acc[a][b], X.b[b][i / (TM * TN)], X.a[a][i / (TM * TN)]);
        else dense::mfma16(acc[a][b], __builtin_bit_cast(bf16x8, X.b[b]), __builtin_bit_cast(bf16x8, X.a[a]));
        if constexpr (i % RS == 0 && i / RS < TM + TN) load_piece(Y, nslot, i / RS, !odd);
        if constexpr (i % DS == W * DS / 4 && i / DS < LPT) issue(i / DS);
        if constexpr (i < 6) next_b(i);
        if constexpr (i >= IPWA * DS && i < IPWA * DS + 4) next_a(i - IPWA * DS);
        if constexpr (i == MF - 1) issue_advance();
        __builtin_amdgcn_sched_barrier(0);
      });
      cslot = nslot;
    };
    for (int ti = 0; ti < n_my; ++ti) {
      const Where range = locate(ti);
      for (int kt = range.k0; kt < range.k1; kt += 2) {
        multiply(F, Gf, std::false_type{});
        if (WIDE) tile_advance();
        multiply(Gf, F, std::true_type{});
        if (!WIDE) tile_advance();
      }
      if constexpr (FP32) {      // as settle() does
        asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
        for (int a = 0; a < TM; ++a) asm volatile("" : "+a"(acc[a][TN - 1]));
      } else {
        dense::settle(acc);
      }
      const Where w = locate(ti);
      // Stores go through a descriptor as well: rows past the group's end (of dW) lie behind it, and a lane whose columns do not exist gets an offset that does.
      if constexpr (DIR == WEIGHT || FP32 || C::PARTS) {
        // a lane's four columns of a row
        const int row = wm * (BM / 2) + li, col = wn * (BN / 2) + 4 * q4, rows = DIR == WEIGHT ? g.M - w.i0 : w.r1 - w.r0, cols = g.N - w.j0;
        const i64 first = DIR == WEIGHT ? ((i64)w.gr * g.M + w.i0) * g.ldc : ((i64)w.split * g.rows + w.r0) * g.ldc;
        const auto rc = make_rsrc((float*)g.C + first + w.j0, ((i64)(rows - 1) * g.ldc + cols) * 4);
        auto store = [&](auto ADD) __attribute__((always_inline)) {
#pragma unroll
          for (int a = 0; a < TM; ++a) {
            const int at = ((row + a * 16) * g.ldc + col) * 4;
#pragma unroll
            for (int c = 0; c < TN; ++c) {
              const int v = col + c * 16 < cols ? at + c * 64 : kNowhere;
              floatx4 x = acc[a][c];
              acc[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};
              if constexpr (decltype(ADD)::value) x += __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rc, v, 0, 0));
              __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), rc, v, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        if (DIR == WEIGHT && g.accumulate) store(std::true_type{});
        else store(std::false_type{});
      } else {
        // through LDS, 16 rows x 64 columns at a time, so that every instruction writes whole 128-byte lines
        char* stg = lds + NS * STAGE_BYTES + wave * C::OUT_BYTES;
        const int rows = w.r1 - w.r0, cols = g.N - w.j0;
        const auto rc = make_rsrc((uint16_t*)g.C + (i64)w.r0 * g.ldc + w.j0, ((i64)(rows - 1) * g.ldc + cols) * 2);
        const int row = wm * (BM / 2) + (lane >> 3), col = wn * (BN / 2) + (lane & 7) * 8, step = (int)g.ldc * 16;      // 8 rows further down
        int at[TN / 4];
#pragma unroll
        for (int cp = 0; cp < TN / 4; ++cp) at[cp] = (row * (int)g.ldc + col + cp * 64) * 2;
#pragma unroll
        for (int a = 0; a < TM; ++a) {
#pragma unroll
          for (int c = 0; c < TN; c += 2) {
            uint32_t o[4];
            dense::pack_pair(acc[a][c], acc[a][c + 1], o);
            acc[a][c] = floatx4{0.f, 0.f, 0.f, 0.f};
            acc[a][c + 1] = floatx4{0.f, 0.f, 0.f, 0.f};
            const int ch = ((c & 3) + (q4 & 1)) * 2 + (q4 >> 1);
            *reinterpret_cast<u32x4*>(stg + (c >> 2) * 2048 + li * 128 + 16 * (ch ^ ((li >> 1) & 7))) = u32x4{o[0], o[1], o[2], o[3]};
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // this wave's own writes; the area is private to it
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int cp = 0; cp < TN / 4; ++cp) {
              const int r = (lane >> 3) + 8 * i, ch = lane & 7;
              const u32x4 o = *reinterpret_cast<const u32x4*>(stg + cp * 2048 + r * 128 + 16 * (ch ^ ((r >> 1) & 7)));
              __builtin_amdgcn_raw_buffer_store_b128(o, rc, col + cp * 64 < cols ? at[cp] : kNowhere, 0, 0);
              at[cp] += step;
            }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read back before the area is rewritten
        }
      }
    }
  };
  switch (wave) {
    case 0: run(std::integral_constant<int, 0>{}); break;
    case 1: run(std::integral_constant<int, 1>{}); break;
    case 2: run(std::integral_constant<int, 2>{}); break;
    default: run(std::integral_constant<int, 3>{}); break;
  }
  mm::wait_vmcnt_and_barrier<0>();      // the last loads land before the LDS is released
}

}  // namespace grouped
}  // namespace poetx
