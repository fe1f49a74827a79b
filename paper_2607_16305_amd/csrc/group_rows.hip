// Entries grouped by the group each one picked (a scene of Eq. 5, an expert):
// a stable counting sort of ids, with the groups' offsets, for the grouped
// products.
//
// One launch and no scratch: workgroup b owns a range of consecutive groups and
// reads all the ids (they stay in L2).  Its waves split the ids into runs of
// consecutive entries; each counts the ids below the range (their sum is where
// the range's rows begin) and lists those of the range in order in LDS.  Over
// its list (or over the ids again, where the list ran full) a wave counts the
// entries of each group; a prefix sum over groups and waves gives every run its
// first slot in each group, and a last pass over the list hands them out.
// What bounds it is the instructions a CU issues for each id, so what a step
// does for the ids of other ranges (two comparisons, two scalar counts) counts
// most, and the busiest range's list after that.
// The result does not depend on timing: counts are sums, and a run's slots are
// handed out by its own wave alone.
#include "common.h"
#include "kernels.h"

namespace lookme {

constexpr int GR_WAVES = 16, GR_THREADS = GR_WAVES * 64;
constexpr int GR_BLOCKS = 256;              // ranges of groups: one workgroup a CU
constexpr int GR_RANGE = LOOKME_MAX_GROUPS / GR_BLOCKS;   // most groups of a range
constexpr int GR_LOADS = 16;                // ids a lane has in flight
constexpr int GR_LIST = 2400;               // entries of a wave's list (150 KiB of LDS)
constexpr int GR_STEP = 64 * GR_LOADS;
static_assert(GR_RANGE <= 64, "a group of the range in 6 bits, one a lane");

__global__ __launch_bounds__(GR_THREADS) void group_rows_kernel(
    const int32_t* __restrict__ pick, int64_t n, int groups, int range, int32_t* __restrict__ rows,
    int32_t* __restrict__ offsets) {
  __shared__ int32_t cnt[GR_WAVES][GR_RANGE];
  __shared__ uint32_t list[GR_WAVES][GR_LIST];   // entry in the run << 6 | group in the range
  __shared__ int32_t below[GR_WAVES];
  __shared__ int32_t tot[GR_RANGE];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t before = (1ull << lane) - 1;
  const int g0 = blockIdx.x * range;
  const int size = groups - g0 < range ? groups - g0 : range;
  // runs of whole steps: at most 2^26 entries
  const int64_t steps = (n + GR_STEP - 1) / GR_STEP;
  const int64_t per = (steps + GR_WAVES - 1) / GR_WAVES;
  const int64_t first = wv * per * GR_STEP;
  int64_t end = first + per * GR_STEP;
  end = end < n ? end : n;

  // id j of a step: entry s + 64 j + lane; -1 past the run
  auto load = [&](int64_t s, int (&v)[GR_LOADS]) {
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      const int64_t i = s + 64 * k + lane;
      v[k] = pick[i < end ? i : end - 1];
    }
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k)
      if (s + 64 * k + lane >= end) v[k] = -1;
  };
  int less = 0, listed = 0;   // the same in every lane
  for (int64_t s = first; s < end; s += GR_STEP) {
    int v[GR_LOADS];
    load(s, v);
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      const unsigned j = (unsigned)v[k] - (unsigned)g0;
      less += __popcll(__ballot((unsigned)v[k] < (unsigned)g0));
      const uint64_t mine = __ballot(j < (unsigned)size);
      if (mine != 0) {
        if (listed <= GR_LIST - 64 && j < (unsigned)size)
          list[wv][listed + __popcll(mine & before)] =
              (uint32_t)(s - first + 64 * k + lane) << 6 | j;
        listed += __popcll(mine);
      }
    }
  }
  // fn(mine, group in the range, entry) for the run's entries of the range in
  // order, up to 64 at a time (whole waves)
  auto each = [&](auto&& fn) {
    if (listed <= GR_LIST - 64) {
      for (int i = 0; i < listed; i += 64) {
        const bool mine = i + lane < listed;
        const uint32_t e = mine ? list[wv][i + lane] : 0;
        fn(mine, (int)(e & 63), first + (e >> 6));
      }
    } else {
      for (int64_t s = first; s < end; s += GR_STEP) {
        int v[GR_LOADS];
        load(s, v);
#pragma unroll
        for (int k = 0; k < GR_LOADS; ++k) {
          const unsigned j = (unsigned)v[k] - (unsigned)g0;
          fn(j < (unsigned)size, (int)j, s + 64 * k + lane);
        }
      }
    }
  };
  // fn(group, ballot of its entries) for every group of the range among them:
  // one after another in short ranges, in others those that occur
  auto groups_of = [&](bool mine, int j, auto&& fn) {
    if (size <= 8) {
      for (int q = 0; q < size; ++q) fn(q, __ballot(mine && j == q));
    } else {
      uint64_t left = __ballot(mine);
      while (left != 0) {
        const int q = __builtin_amdgcn_readlane(j, __builtin_ctzll(left));
        const uint64_t same = __ballot(mine && j == q);
        fn(q, same);
        left &= ~same;
      }
    }
  };
  int count = 0;   // lane j: the run's entries of group j
  each([&](bool mine, int j, int64_t) {
    groups_of(mine, j, [&](int q, uint64_t same) { count += lane == q ? __popcll(same) : 0; });
  });
  cnt[wv][lane] = count;
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
  if (wv == 0) {   // the groups' first slots
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
  // lane j holds the run's next slot of group j
  int next = lane < size ? cnt[wv][lane] + tot[lane] : 0;

  each([&](bool mine, int j, int64_t entry) {
    groups_of(mine, j, [&](int q, uint64_t same) {
      const int at = __builtin_amdgcn_readlane(next, q);
      if (mine && j == q) rows[at + __popcll(same & before)] = (int32_t)entry;
      next += lane == q ? __popcll(same) : 0;
    });
  });
}

hipError_t launch_group_rows(int groups, int64_t n, const int32_t* pick, int32_t* rows,
                             int32_t* offsets, hipStream_t st) {
  const int range = (groups + GR_BLOCKS - 1) / GR_BLOCKS;
  hipLaunchKernelGGL(group_rows_kernel, dim3((unsigned)((groups + range - 1) / range)),
                     dim3(GR_THREADS), 0, st, pick, n, groups, range, rows, offsets);
  return hipGetLastError();
}

}  // namespace lookme
