// Entries grouped by the group each one picked (a scene of Eq. 5, an expert):
// a stable counting sort of ids, with the groups' offsets, for the grouped
// products.
//
// One launch and no scratch: workgroup b owns a range of consecutive groups and
// reads all the ids (they stay in L2).  Its waves split the ids into runs of
// consecutive entries; each counts the ids below the range (their sum is where
// the range's rows begin) and, in LDS, those of each group of the range; a
// prefix sum over groups and waves gives every run its first slot in each
// group, and a second pass over the run writes the entries there in order.
// The result does not depend on timing: counts are sums, and a run's slots are
// handed out by its own wave alone.
#include "common.h"
#include "kernels.h"

namespace lookme {

constexpr int GR_WAVES = 16, GR_THREADS = GR_WAVES * 64;
constexpr int GR_BLOCKS = 256;              // ranges of groups: one workgroup a CU
constexpr int GR_RANGE = LOOKME_MAX_GROUPS / GR_BLOCKS;   // most groups of a range
constexpr int GR_LOADS = 4;                 // ids a lane has in flight

__global__ __launch_bounds__(GR_THREADS) void group_rows_kernel(
    const int32_t* __restrict__ pick, int64_t n, int groups, int range, int32_t* __restrict__ rows,
    int32_t* __restrict__ offsets) {
  __shared__ int32_t cnt[GR_WAVES][GR_RANGE];
  __shared__ int32_t below[GR_WAVES];
  __shared__ int32_t tot[GR_RANGE];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g0 = blockIdx.x * range;
  const int size = groups - g0 < range ? groups - g0 : range;
  for (int i = lane; i < range; i += 64) cnt[wv][i] = 0;
  // runs of whole 64 x GR_LOADS steps
  constexpr int STEP = 64 * GR_LOADS;
  const int64_t steps = (n + STEP - 1) / STEP;
  const int64_t per = (steps + GR_WAVES - 1) / GR_WAVES;
  const int64_t first = wv * per * STEP;
  int64_t end = first + per * STEP;
  end = end < n ? end : n;

  int less = 0;
  for (int64_t s = first; s < end; s += STEP) {
    int v[GR_LOADS];
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      const int64_t i = s + 64 * k + lane;
      v[k] = i < end ? pick[i] : -1;
    }
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      less += (v[k] >= 0) & (v[k] < g0);
      const unsigned j = (unsigned)v[k] - (unsigned)g0;
      if (v[k] >= g0 && j < (unsigned)size) atomicAdd(&cnt[wv][j], 1);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) less += __shfl_xor(less, d, 64);
  if (lane == 0) below[wv] = less;
  __syncthreads();
  // each group's total; the runs' counts become the runs' places in the group
  if ((int)threadIdx.x < size) {
    int sum = 0;
    for (int w = 0; w < GR_WAVES; ++w) {
      const int c = cnt[w][threadIdx.x];
      cnt[w][threadIdx.x] = sum;
      sum += c;
    }
    tot[threadIdx.x] = sum;
  }
  __syncthreads();
  if (wv == 0) {   // groups' first slots: a prefix sum, at most one group a lane
    static_assert(GR_RANGE <= 64, "one wave holds the range");
    int base = 0;
    for (int w = 0; w < GR_WAVES; ++w) base += below[w];
    const int c = lane < size ? tot[lane] : 0;
    const int incl = wave_scan_incl(c);
    if (lane < size) {
      tot[lane] = base + incl - c;
      offsets[g0 + lane] = base + incl - c;
      if (g0 + lane == groups - 1) offsets[groups] = base + incl;
    }
  }
  __syncthreads();
  if (lane < size) cnt[wv][lane] += tot[lane];
  __builtin_amdgcn_wave_barrier();

  for (int64_t s = first; s < end; s += STEP) {
    int v[GR_LOADS];
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      const int64_t i = s + 64 * k + lane;
      v[k] = i < end ? pick[i] : -1;
    }
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      const int j = v[k] - g0;
      bool mine = v[k] >= g0 && j < size;
      uint64_t left = __ballot(mine);
      while (left != 0) {   // one round per distinct group of the 64 entries
        const int lead = __builtin_ctzll(left);
        const int jl = __shfl(j, lead, 64);
        const uint64_t same = __ballot(mine && j == jl);
        const int at = cnt[wv][jl];
        if (mine && j == jl) {
          rows[at + __popcll(same & ((1ull << lane) - 1))] = (int32_t)(s + 64 * k + lane);
          if (lane == lead) cnt[wv][jl] = at + __popcll(same);
          mine = false;
        }
        left &= ~same;
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
}

hipError_t launch_group_rows(int groups, int64_t n, const int32_t* pick, int32_t* rows,
                             int32_t* offsets, hipStream_t st) {
  const int range = (groups + GR_BLOCKS - 1) / GR_BLOCKS;
  hipLaunchKernelGGL(group_rows_kernel, dim3((unsigned)((groups + range - 1) / range)),
                     dim3(GR_THREADS), 0, st, pick, n, groups, range, rows, offsets);
  return hipGetLastError();
}

}  // namespace lookme
