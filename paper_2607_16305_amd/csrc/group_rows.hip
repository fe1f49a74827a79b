// Entries grouped by the group each one picked (a scene of Eq. 5, an expert):
// a stable counting sort of ids, with the groups' offsets, for the grouped
// products.
//
// One launch and no scratch.  A workgroup owns a range of consecutive groups and
// (with fewer groups than CUs) one of several segments of the entries, and reads
// all the ids (2^18 of them are 1 MiB and stay in L2; see below): those below the range count towards where its
// rows begin, those of its group ahead of its segment towards where its own
// begin.  In its segment its waves own runs of consecutive entries, and each
// lists its run's entries of the range in order in LDS.  Over its list (or over
// the run again, where the list ran full) a wave counts the entries of each
// group; a prefix sum over groups and waves gives every run its first slot in
// each group, and a last pass over the list hands them out.
// What bounds it is the instructions a CU issues for each id: for 64 of another
// range a subtraction, whose borrow is the count of those below, an addition and
// a comparison (262144 ids in 1024 groups alike 21 us, 13 TB/s out of L2; with
// Zipf(1) groups 45, the largest being an eighth of the ids, and 130 where the
// largest ones are neighbours and so share a workgroup; 512 ids in 128 groups 4.1).
// The time grows with the ids, 2^20 in 1024 groups alike 71 us and 2^22 275, until
// the lists run full: 2^24 take 7.3 ms.
// The result does not depend on timing: counts are sums, and a run's slots are
// handed out by its own wave alone.
#include "common.h"
#include "kernels.h"

namespace lookme {

constexpr int GR_WAVES = 16, GR_THREADS = GR_WAVES * 64;
constexpr int GR_BLOCKS = 256;              // one workgroup a CU
constexpr int GR_RANGE = LOOKME_MAX_GROUPS / GR_BLOCKS;   // most groups of a range
constexpr int GR_LOADS = 16;                // ids a lane has in flight
constexpr int GR_LIST = 2400;               // entries of a wave's list (150 KiB of LDS)
constexpr int GR_STEP = 64 * GR_LOADS;
constexpr int GR_FEW = 4;                   // groups of a range whose counts stay in scalars
static_assert(GR_RANGE <= 64, "a group of the range in 6 bits, one a lane");

// base + the lanes of the mask below this one
__device__ __forceinline__ int gr_slot(uint64_t mask, int base) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)base));
}

__global__ __launch_bounds__(GR_THREADS) void group_rows_kernel(
    const int32_t* __restrict__ pick, int n, int groups, int range, int segments,
    int32_t* __restrict__ rows, int32_t* __restrict__ offsets) {
  __shared__ int32_t cnt[GR_WAVES][GR_RANGE];
  __shared__ uint32_t list[GR_WAVES][GR_LIST];   // entry in the run << 6 | group in the range
  __shared__ int32_t below[GR_WAVES], ahead[GR_WAVES];
  __shared__ int32_t tot[GR_RANGE];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g0 = (int)(blockIdx.x / segments) * range;
  const int seg = blockIdx.x % segments;
  const int size = groups - g0 < range ? groups - g0 : range;
  const unsigned lo = (unsigned)g0, span = (unsigned)size;

  // steps of GR_STEP entries: the segment's, dealt to the waves in runs (a run
  // is at most 2^26 entries), and the others, dealt one by one
  const int steps = (n + GR_STEP - 1) / GR_STEP;
  const int seg_steps = (steps + segments - 1) / segments;
  const int seg0 = seg * seg_steps < steps ? seg * seg_steps : steps;
  const int seg1 = seg0 + seg_steps < steps ? seg0 + seg_steps : steps;
  const int per = (seg1 - seg0 + GR_WAVES - 1) / GR_WAVES;
  const int run0 = seg0 + wv * per < seg1 ? seg0 + wv * per : seg1;
  const int run1 = run0 + per < seg1 ? run0 + per : seg1;

  // entry GR_STEP step + 64 k + lane; -1 past the last
  auto load = [&](int step, int (&v)[GR_LOADS]) {
    const int s = step * GR_STEP;
    const int32_t* p = pick + s + lane;
    if (s + GR_STEP <= n) {
#pragma unroll
      for (int k = 0; k < GR_LOADS; ++k) v[k] = p[64 * k];
    } else {
#pragma unroll
      for (int k = 0; k < GR_LOADS; ++k) v[k] = s + 64 * k + lane < n ? p[64 * k] : -1;
    }
  };
  // a lane's ids below the range, and of the range ahead of the segment; the run's
  // entries of the range (the same in every lane)
  int lane_less = 0, lane_early = 0, listed = 0;
  for (int step = wv; step < steps; step += GR_WAVES) {
    if (step >= seg0 && step < seg1) continue;
    int v[GR_LOADS];
    load(step, v);
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      lane_less += (unsigned)v[k] < lo ? 1 : 0;
      if (step < seg0) lane_early += (unsigned)v[k] - lo < span ? 1 : 0;
    }
  }
  for (int step = run0; step < run1; ++step) {
    int v[GR_LOADS];
    load(step, v);
#pragma unroll
    for (int k = 0; k < GR_LOADS; ++k) {
      lane_less += (unsigned)v[k] < lo ? 1 : 0;
      const unsigned j = (unsigned)v[k] - lo;   // group in the range
      const uint64_t mine = __ballot(j < span);
      if (mine != 0) {
        // (a full list is written over at its end, and not read)
        const int at = listed < GR_LIST - 64 ? listed : GR_LIST - 64;
        if (__builtin_amdgcn_inverse_ballot_w64(mine))
          list[wv][gr_slot(mine, at)] =
              j + (uint32_t)(lane << 6) + ((uint32_t)((step - run0) * GR_STEP + 64 * k) << 6);
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
        fn(mine, (int)(e & 63), run0 * GR_STEP + (int)(e >> 6));
      }
    } else {
      for (int step = run0; step < run1; ++step) {
        int v[GR_LOADS];
        load(step, v);
#pragma unroll
        for (int k = 0; k < GR_LOADS; ++k)
          fn((unsigned)v[k] - lo < span, v[k] - g0,
             step * GR_STEP + 64 * k + lane);
      }
    }
  };
  // fn(group, ballot of its entries) for every group that occurs among them
  auto groups_of = [&](bool mine, int j, auto&& fn) {
    uint64_t left = __ballot(mine);
    while (left != 0) {
      const int q = __builtin_amdgcn_readlane(j, __builtin_ctzll(left));
      const uint64_t same = __ballot(mine && j == q);
      fn(q, same);
      left &= ~same;
    }
  };
  int count = 0;   // lane j: the run's entries of group j
  if (range <= GR_FEW) {
    int few[GR_FEW] = {};
    each([&](bool mine, int j, int) {
#pragma unroll
      for (int q = 0; q < GR_FEW; ++q) few[q] += __popcll(__ballot(mine && j == q));
    });
#pragma unroll
    for (int q = 0; q < GR_FEW; ++q) count = lane == q ? few[q] : count;
  } else {
    each([&](bool mine, int j, int) {
      groups_of(mine, j, [&](int q, uint64_t same) { count += lane == q ? __popcll(same) : 0; });
    });
  }
  cnt[wv][lane] = count;
  const int less = wave_scan_incl(lane_less), early = wave_scan_incl(lane_early);
  if (lane == 63) {
    below[wv] = less;
    ahead[wv] = early;
  }
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
  if (wv == 0) {   // the groups' first slots (several segments: of the range's one group)
    int base = 0, first = 0;
    for (int w = 0; w < GR_WAVES; ++w) {
      base += below[w];
      first += ahead[w];
    }
    const int c = lane < size ? tot[lane] : 0;
    const int incl = wave_scan_incl(c);
    if (lane < size) {
      tot[lane] = base + first + incl - c;
      if (seg == 0) offsets[g0 + lane] = base + incl - c;
      if (seg == segments - 1 && g0 + lane == groups - 1) offsets[groups] = base + first + incl;
    }
  }
  __syncthreads();
  // lane j holds the run's next slot of group j
  int next = lane < size ? cnt[wv][lane] + tot[lane] : 0;
  if (range <= GR_FEW) {
    int few[GR_FEW];
#pragma unroll
    for (int q = 0; q < GR_FEW; ++q) few[q] = __builtin_amdgcn_readlane(next, q);
    each([&](bool mine, int j, int entry) {
      int at = 0;
#pragma unroll
      for (int q = 0; q < GR_FEW; ++q) {
        const uint64_t same = __ballot(mine && j == q);
        at = j == q ? gr_slot(same, few[q]) : at;
        few[q] += __popcll(same);
      }
      if (mine) rows[at] = entry;
    });
  } else {
    each([&](bool mine, int j, int entry) {
      groups_of(mine, j, [&](int q, uint64_t same) {
        const int at = __builtin_amdgcn_readlane(next, q);
        if (mine && j == q) rows[gr_slot(same, at)] = entry;
        next += lane == q ? __popcll(same) : 0;
      });
    });
  }
}

hipError_t launch_group_rows(int groups, int64_t n, const int32_t* pick, int32_t* rows,
                             int32_t* offsets, hipStream_t st) {
  const int range = (groups + GR_BLOCKS - 1) / GR_BLOCKS;
  const int ranges = (groups + range - 1) / range;
  // a CU a segment, and a step for each of them (25509 ids of one group in one
  // segment 21 us)
  const int64_t steps = (n + GR_STEP - 1) / GR_STEP;
  int64_t segments = range == 1 ? GR_BLOCKS / ranges : 1;
  if (segments > steps) segments = steps;
  if (segments < 1) segments = 1;
  return launch_kernel(group_rows_kernel, dim3((unsigned)(ranges * segments)), dim3(GR_THREADS), 0,
                       st, pick, (int)n, groups, range, (int)segments, rows, offsets);
}

}  // namespace lookme
