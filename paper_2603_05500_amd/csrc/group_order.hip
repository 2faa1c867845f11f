// The order that puts rows group by group: a stable counting sort by group number.
//
// A workgroup of 16 waves takes a range of the rows, a wave a sixteenth of it, 64 rows at a time in order.  Rows of the same group inside 64 are found
// by ballots, one per bit of the number; counts per wave and group lie in LDS, and become running positions once the counts before
// them -- lower groups, earlier ranges, earlier waves -- are added.  Rows that no group takes are a group of their own behind the others.
//
// What bounds it is latency: one launch up to 4096 rows (8192 rows of 128 groups 10.6 us in one, 16384 of 256 8.7 in two); beyond, a launch that counts every range first.  us: 2048 rows, 64 groups 4.5,
// 131072 rows, 128 groups 10.4 (ranges of 1024 rows 11.7, of 4096 11.3).
#include "poetx_kernels.h"

namespace poetx {
namespace {

constexpr int WAVES = 16, NTH = 64 * WAVES;
constexpr int SINGLE = 4096;       // rows of one workgroup alone
constexpr int RANGES = 128;        // workgroups at most

struct OrderArgs {
  const int32_t* ids;
  i64 n, per_wave;      // rows; rows of a wave, a multiple of 64
  int groups, bits;     // bits of the largest number, `groups` itself
  int ranges;
  int32_t* counts;      // [range][groups + 1]
  int32_t* offsets;
  int32_t* order;
};

__device__ __forceinline__ int bucket(const OrderArgs& a, i64 i) {
  const int g = a.ids[i];
  return g >= 0 && g < a.groups ? g : a.groups;
}
// lanes with this lane's bucket
__device__ __forceinline__ uint64_t same_bucket(int g, int bits, bool on) {
  uint64_t m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t v = __ballot((g >> b) & 1);
    m &= (g >> b) & 1 ? v : ~v;
  }
  return m;
}

// per-wave counts of this range into cnt [WAVES][B]
__device__ void count_range(const OrderArgs& a, int B, int32_t* cnt) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < WAVES * B; i += NTH) cnt[i] = 0;
  __syncthreads();
  const i64 w0 = ((i64)blockIdx.x * WAVES + wave) * a.per_wave;
  for (i64 i = w0 + lane; i < w0 + a.per_wave && i < a.n; i += 64) atomicAdd(cnt + wave * B + bucket(a, i), 1);      // whole numbers: any order
  __syncthreads();
}

__global__ __launch_bounds__(NTH) void order_count_kernel(OrderArgs a) {
  extern __shared__ int32_t cnt[];
  const int B = a.groups + 1;
  count_range(a, B, cnt);
  for (int g = threadIdx.x; g < B; g += NTH) {
    int s = 0;
    for (int w = 0; w < WAVES; ++w) s += cnt[w * B + g];
    a.counts[(i64)blockIdx.x * B + g] = s;
  }
}

__global__ __launch_bounds__(NTH) void order_place_kernel(OrderArgs a) {
  extern __shared__ int32_t cnt[];
  __shared__ int32_t all[POETX_GROUP_ORDER_MAX + 1], before[POETX_GROUP_ORDER_MAX + 1], wsum[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int B = a.groups + 1;
  static_assert(POETX_GROUP_ORDER_MAX + 1 <= NTH, "a thread per bucket");
  for (int g = tid; g < B; g += NTH) all[g] = before[g] = 0;
  count_range(a, B, cnt);
  // each bucket's rows in all, and in the ranges before this one
  if (a.ranges == 1) {
    if (tid < B) {
      int s = 0;
      for (int w = 0; w < WAVES; ++w) s += cnt[w * B + tid];
      all[tid] = s;
    }
  } else {
    const int parts = NTH / B, g = tid % B, part = tid / B;
    if (part < parts) {
      int s = 0, t = 0;
      for (int r = part; r < a.ranges; r += parts) {
        const int c = a.counts[(i64)r * B + g];
        s += c;
        if (r < (int)blockIdx.x) t += c;
      }
      atomicAdd(all + g, s);
      atomicAdd(before + g, t);
    }
  }
  __syncthreads();
  // where a bucket starts: the sum of those before it
  int mine = tid < B ? all[tid] : 0, sum = mine;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int o = __shfl_up(sum, s);
    if (lane >= s) sum += o;
  }
  if (lane == 63) wsum[wave] = sum;
  __syncthreads();
  int start = sum - mine;
  for (int w = 0; w < wave; ++w) start += wsum[w];
  if (tid < B) {
    if (blockIdx.x == 0) a.offsets[tid] = start;
    int at = start + before[tid];
    for (int w = 0; w < WAVES; ++w) {
      const int c = cnt[w * B + tid];
      cnt[w * B + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  const i64 w0 = ((i64)blockIdx.x * WAVES + wave) * a.per_wave;
  for (i64 i0 = w0; i0 < w0 + a.per_wave && i0 < a.n; i0 += 64) {
    const i64 i = i0 + lane;
    const bool on = i < a.n;
    const int g = on ? bucket(a, i) : a.groups;
    const uint64_t same = same_bucket(g, a.bits, on);
    const int rank = __popcll(same & ((1ull << lane) - 1));
    const int at = on ? cnt[wave * B + g] : 0;
    __builtin_amdgcn_wave_barrier();      // every lane has its position before the first of a bucket moves it on: LDS serves a wave in order
    if (on) {
      a.order[at + rank] = g < a.groups ? (int32_t)i : -1;
      if (rank == 0) cnt[wave * B + g] = at + __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

__global__ void order_empty_kernel(int32_t* offsets, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

inline int order_ranges(i64 n) {
  if (n <= SINGLE) return 1;
  const i64 r = (n + 2047) / 2048;
  return (int)(r < RANGES ? r : RANGES);
}

}  // namespace

size_t group_order_workspace_bytes(i64 n, int groups) {
  const int r = order_ranges(n);
  return r == 1 ? 0 : align256((size_t)r * (groups + 1) * sizeof(int32_t));
}

void group_order_launch(const int32_t* ids, i64 n, int groups, int32_t* offsets, int32_t* order, void* ws, hipStream_t st) {
  if (n == 0) {
    hipLaunchKernelGGL(order_empty_kernel, dim3(1), dim3(256), 0, st, offsets, groups + 1);
    return;
  }
  OrderArgs a{ids, n, 0, groups, 32 - __builtin_clz((unsigned)groups), order_ranges(n), (int32_t*)ws, offsets, order};
  a.per_wave = (n + (i64)a.ranges * WAVES * 64 - 1) / ((i64)a.ranges * WAVES * 64) * 64;
  const size_t lds = sizeof(int32_t) * WAVES * (groups + 1);
  if (a.ranges > 1) hipLaunchKernelGGL(order_count_kernel, dim3(a.ranges), dim3(NTH), lds, st, a);
  hipLaunchKernelGGL(order_place_kernel, dim3(a.ranges), dim3(NTH), lds, st, a);
}

}  // namespace poetx
