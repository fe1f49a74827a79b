// Products of rows that come grouped, every group with a matrix of its own (the
// rows of a scene of Eq. 5 with that scene's matrices, the rows of an expert):
//
//   out[i] = round(W[g] x[src(i)])                       for i in group g, or
//   out[i] = round(silu(W[g] x[src(i)]) * (W_up[g] x[src(i)]))
//
// The groups' sizes are on the device only.  A workgroup finds its tile by a
// prefix sum over the groups' tile counts, so no tile spans two groups, and
// empty groups cost nothing.  Three kernels:
//
//   grouped_rows_kernel   a few rows a group: bound by the stream of the weights
//       out of HBM.  A wave multiplies 16 weight rows by 16 tokens straight
//       from global memory (both operands are K-contiguous, a lane's 16 bytes
//       are its fragment), K split over the waves of a workgroup and summed
//       through LDS.
//   grouped_mid_kernel    some rows a group: 32 x 64 and 64 x 64 tiles, both
//       operands through a ring of stages in LDS.
//   grouped_tiles_kernel  many rows a group: 256 x 256 and 128 x 256 tiles on the
//       phased loop of phase_gemm.h, one workgroup a CU that takes tile after
//       tile: 64 groups of 1024 rows, 2048 x 2048 in bf16, 517 to 573 us by run and
//       card, 1063 to 959 TFLOP/s; 32 of 4096 x 4096 885 to 902, 1242 to 1219; 16 of
//       2048 rows, 4096 x 4096 in e4m3, 497 to 566, 2210 to 1940.
//       Bound by the stage stream out of L2 beside the fragment reads (the matrix
//       cores are busy 55% of the time, at the 2.0 GHz that such a load leaves)
//       and by the stores of a tile, 8 us in 63, which meet those of all others.
//
// e4m3 operands carry a float32 scale a row, applied once to the float32 sum:
// out = round((sum xs) ws).
#include "common.h"
#include "kernels.h"
#include "tile_gemm.h"

namespace lookme {

static_assert(GROUPED_E4M3 == DT_E4M3, "one numbering");

struct GpTile {
  int g;           // group, or -1
  int idx;         // tile inside the group
  int64_t a, b;    // rows of the group
};

// rows [a, b) of group g, kept inside [0, m) whatever the offsets hold (m is at
// most 2^30)
__device__ __forceinline__ void gp_rows(const GroupedParams& p, int g, int& a, int& b) {
  const int m = (int)p.m;
  a = p.offsets[g];
  b = p.offsets[g + 1];
  a = a < 0 ? 0 : (a > m ? m : a);
  b = b < a ? a : (b > m ? m : b);
}

// Tile number which(total) in the groups' order, count(rows) tiles a group; all
// threads of the block, which pass a barrier before the next call.  t.g is -1 past
// the last tile.  A wave counts a run of groups, 64 neighbours at a time; the one
// that has the tile goes through its run again.  (A thread's groups side by side
// are a load of 64 lines each: 4000 groups of one row, 256 x 512, 502 us, 368 so.)
template <int THREADS, class Count, class Which>
__device__ __forceinline__ void find_tile(const GroupedParams& p, int* lds, GpTile& t,
                                          Count&& count, Which&& which) {
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = (p.groups + THREADS - 1) / THREADS;
  const int first = wv * 64 * per + lane;
  int a = 0, b = 0;
  // tiles of group g; its rows in (a, b).  No branch, so that several groups'
  // loads are in flight.
  auto tiles = [&](int g) {
    gp_rows(p, g < p.groups ? g : p.groups - 1, a, b);
    return g < p.groups ? count(b - a) : 0;
  };
  int sum = 0;
  int k = 0;
  for (; k + 8 <= per; k += 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += tiles(first + 64 * (k + u));
  }
  for (; k < per; ++k) sum += tiles(first + 64 * k);
  if (threadIdx.x == 0) lds[0] = -1;
  const int incl = wave_scan_incl(sum);
  if (lane == 63) lds[4 + wv] = incl;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const int s = lds[4 + w];
    before += w < wv ? s : 0;
    total += s;
  }
  const int unit = which(__builtin_amdgcn_readfirstlane(total));
  int left = unit - __builtin_amdgcn_readfirstlane(before);   // in this wave's run
  if (left >= 0 && left < lds[4 + wv]) {
    int c = sum, end = incl, g = first;
    if (per != 1) {
      bool found = false;
      for (int q = 0; q < per && !found; q += 4) {
        int c4[4], a4[4], b4[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          c4[u] = tiles(first + 64 * (q + u));
          a4[u] = a;
          b4[u] = b;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (found) continue;
          c = c4[u];
          a = a4[u];
          b = b4[u];
          g = first + 64 * (q + u);
          end = wave_scan_incl(c);
          const int all = __builtin_amdgcn_readlane(end, 63);
          found = left < all;
          left -= found ? 0 : all;
        }
      }
      if (!found) c = end = 0;   // (never, while nobody changes the offsets)
    }
    if (end - c <= left && left < end) {
      lds[0] = g;
      lds[1] = left - (end - c);
      lds[2] = a;
      lds[3] = b;
    }
  }
  __syncthreads();
  t.g = __builtin_amdgcn_readfirstlane(lds[0]);
  t.idx = __builtin_amdgcn_readfirstlane(lds[1]);
  t.a = __builtin_amdgcn_readfirstlane(lds[2]);
  t.b = __builtin_amdgcn_readfirstlane(lds[3]);
}
constexpr int GP_FIND_LDS = 4 + 4;   // (of blocks of four waves)
// Most workgroups of a launch: the number of tiles is the device's, and a launch
// is for the most there can be, in passes of this many.
constexpr int64_t GP_GRID = 65536;

// Entry i: the row of x it reads (clamped) and the row of out it writes; false
// where either is out of range, which leaves the row as it was.
__device__ __forceinline__ bool gp_entry(const GroupedParams& p, int64_t i, int64_t& src,
                                         int64_t& dst) {
  src = dst = i;
  if (p.rows != nullptr) {
    const int r = p.rows[i];
    if (p.picks != 0) src = p.picks == 1 ? r : r / p.picks;
    if (p.scatter) dst = r;
    const bool ok = r >= 0 && src < p.x_rows && dst < p.m;
    src = src < 0 ? 0 : (src < p.x_rows ? src : p.x_rows - 1);
    return ok;
  }
  return true;
}

// float32 sums of one output and of its up half, made an output value.  The scales
// one after the other: their product may pass the range that the result keeps, and
// a sum of zero is zero.
template <int DT, bool UP>
__device__ __forceinline__ float gp_value(float c, float u, float xs, float ws, float us) {
  if constexpr (DT == DT_E4M3) {
    c = c * xs * ws;
    u = u * xs * us;
  }
  return UP ? silu_f(c) * u : c;
}

// ---------------------------------------------------------------------------
// few rows a group
// ---------------------------------------------------------------------------
constexpr int GS_THREADS = 256, GS_WAVES = 4;
constexpr int64_t GS_BLOCKS = 8192;   // of a launch, above which each takes more

// KS: waves that share the K of 16 weight rows; the workgroup's other waves take
// other rows.  Two steps (64 bytes of K) are in flight a wave: more registers
// for more of them cost as many waves (1 row in 128 groups of 2 x 1024 x 2048
// 187 us, 5.7 TB/s of weights, 195 with four).
template <int DT, int KS, bool UP>
__global__ __launch_bounds__(GS_THREADS) void grouped_rows_kernel(GroupedParams p) {
  constexpr int ODT = DT == DT_E4M3 ? DT_BF16 : DT;
  constexpr int OES = ODT == DT_BF16 ? 2 : 4;
  constexpr int MATS = UP ? 2 : 1;
  constexpr int COLS = 16 * (GS_WAVES / KS), D = 2;
  __shared__ int find_lds[GP_FIND_LDS];
  __shared__ f32x4_t part[GS_WAVES * MATS * 64];
  const int tiles_n = (p.cols + COLS - 1) / COLS;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int kp = wv % KS;
  const int chunks = (int)(p.k_bytes / 16);
  const int steps = (chunks + 3) / 4;
  const int per = (steps + KS - 1) / KS;
  const int s0 = kp * per;
  const int s1 = s0 + per < steps ? s0 + per : steps;

  const int cblocks = (tiles_n + p.span - 1) / p.span;

  for (int64_t unit = blockIdx.x;; unit += gridDim.x) {
    const int row_tile = (int)(unit / cblocks);
    GpTile t;
    find_tile<GS_THREADS>(
        p, find_lds, t, [](int r) { return (int)((unsigned)(r + 15) / 16); },
        [row_tile](int) { return row_tile; });
    if (t.g < 0) return;
    const int t0 = (int)(unit - (int64_t)row_tile * cblocks) * p.span;
    const int t1 = t0 + p.span < tiles_n ? t0 + p.span : tiles_n;

    int64_t i = t.a + (int64_t)t.idx * 16 + n16, src, dst;
    const bool in = i < t.b;
    i = in ? i : t.b - 1;
    const bool ok = gp_entry(p, i, src, dst) && in;
    const char* xp = p.x + src * p.k_bytes;
    const float xs = DT == DT_E4M3 ? p.x_scale[src] : 1.f;

    for (int ct = t0; ct < t1; ++ct) {
      const int c0 = ct * COLS + 16 * (wv / KS);
      const int wc = c0 + n16 < p.cols ? c0 + n16 : p.cols - 1;
      const int64_t wrow = ((int64_t)t.g * p.cols + wc) * p.k_bytes;
      const char* wp[MATS];
      wp[0] = p.w + wrow;
      if constexpr (UP) wp[1] = p.w_up + wrow;

      f32x4_t acc[MATS];
#pragma unroll
      for (int q = 0; q < MATS; ++q) acc[q] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      u32x4_t fw[D][MATS], fx[D];
      // unconditional loads from clamped addresses; chunks past K count as zero
      auto load = [&](int d, int s) {
        int c = 4 * s + g;
        c = c < chunks ? c : chunks - 1;
#pragma unroll
        for (int q = 0; q < MATS; ++q) fw[d][q] = ld16(wp[q] + (int64_t)c * 16);
        fx[d] = ld16(xp + (int64_t)c * 16);
      };
      if (s0 < s1) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
          load(d, s0 + d);
          asm volatile("" ::: "memory");
        }
        for (int s = s0; s < s1; s += D) {
#pragma unroll
          for (int d = 0; d < D; ++d) {
            const bool live = s + d < s1 && 4 * (s + d) + g < chunks;
            const u32x4_t none = {0, 0, 0, 0};
            u32x4_t w[MATS];
#pragma unroll
            for (int q = 0; q < MATS; ++q) w[q] = live ? fw[d][q] : none;
            const u32x4_t x = live ? fx[d] : none;
            load(d, s + d + D);
#pragma unroll
            for (int q = 0; q < MATS; ++q) acc[q] = mfma_chunk<DT>(w[q], x, acc[q]);
          }
        }
      }
      f32x4_t* mine = part + wv * (MATS * 64) + lane;
      if (kp != 0) {
#pragma unroll
        for (int q = 0; q < MATS; ++q) mine[q * 64] = acc[q];
      }
      __syncthreads();
      if (kp == 0) {
#pragma unroll
        for (int o = 1; o < KS; ++o)
#pragma unroll
          for (int q = 0; q < MATS; ++q) {
            const f32x4_t v = mine[(o * MATS + q) * 64];
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[q][r] += v[r];
          }
        // the lane holds columns c0 + 4 g + r of its token's row (cols is a multiple
        // of 4)
        const int col = c0 + 4 * g;
        if (col < p.cols && ok) {
          f32x4_t ws = {1.f, 1.f, 1.f, 1.f}, us = ws;
          if constexpr (DT == DT_E4M3) {
            const int64_t s = (int64_t)t.g * p.cols + col;
            ws = *reinterpret_cast<const f32x4_t*>(p.w_scale + s);
            if constexpr (UP) us = *reinterpret_cast<const f32x4_t*>(p.up_scale + s);
          }
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            v[r] = gp_value<DT, UP>(acc[0][r], UP ? acc[MATS - 1][r] : 0.f, xs, ws[r], us[r]);
          st_cols<ODT, 4>(p.out + (dst * p.cols + col) * OES, v);
        }
      }
      if (ct + 1 < t1) __syncthreads();   // (the next unit has find_tile's barriers)
    }
  }
}

// ---------------------------------------------------------------------------
// some rows a group
// ---------------------------------------------------------------------------
// 64 x 64 tiles (UP: 64 rows x 32 columns of both matrices), four waves in 2 x
// 2 of 32 rows x 32 weight rows, K in 128-byte stages loaded straight into a
// ring of NS in LDS (dtl.h), or 32 x 64 with two tiles a wave.  Bound by the
// stages' latency over the bytes in flight, so the ring is deeper where a CU has
// few tiles, and there are several workgroups a CU where it has more: 64 groups
// of 16 rows, 2048 x 2048 in bf16, 97 us, 5.5 TB/s of weights; 13 groups of 231
// rows, 840 x 1160 in float32, 71 us, 82 TFLOP/s with the matrix cores busy 71%
// (728 tiles on 256 CUs).
template <int TI>
using GmShape = DtlShape<2, 2, TI, 2, 128>;
constexpr int GM_THREADS = 256;

template <int DT, int NS, int TI, bool UP>
__global__ __launch_bounds__(GM_THREADS) void grouped_mid_kernel(GroupedParams p) {
  using S = GmShape<TI>;
  constexpr int RT = 32 * TI;
  constexpr int ODT = DT == DT_E4M3 ? DT_BF16 : DT;
  constexpr int OES = ODT == DT_BF16 ? 2 : 4;
  constexpr int COLS = UP ? 32 : 64;
  // one object, as in the large tiles' kernel below
  constexpr int STAGES = NS * S::STAGE;
  __shared__ __attribute__((aligned(1024))) char smem[STAGES + 4 * (GP_FIND_LDS + 3 * RT)];
  char (*lds)[S::STAGE] = reinterpret_cast<char (*)[S::STAGE]>(smem);
  int32_t* row_src = reinterpret_cast<int32_t*>(smem + STAGES);
  int32_t* row_dst = row_src + RT;
  float* row_xs = reinterpret_cast<float*>(row_dst + RT);
  int* find_lds = row_dst + 2 * RT;
  const int tn = (p.cols + COLS - 1) / COLS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int wm = (wv >> 1) * 16 * TI, wn = wv & 1;
  const int nst = (int)(p.k_bytes / 128);
  const int tail = (int)(p.k_bytes / 16) - 8 * nst;

  for (int64_t base = 0;; base += gridDim.x) {
    // the tiles of a group run down the row tiles of a column block first (they
    // share its weights), neighbours on one XCD
    GpTile t;
    find_tile<GM_THREADS>(
        p, find_lds, t, [tn](int r) { return (int)((unsigned)(r + RT - 1) / RT) * tn; },
        [&](int total) {
          const int64_t left = total - base;
          const int n = (int)(left < (int64_t)gridDim.x ? left : (int64_t)gridDim.x);
          const int u = n > 0 ? xcd_remap(blockIdx.x, n) : -1;
          return u < 0 ? -1 : (int)(base + u);
        });
    if (t.g < 0) return;
    const int row_tiles = (int)((t.b - t.a + RT - 1) / RT);
    const int ct = t.idx / row_tiles;
    const int64_t m0 = (int64_t)(t.idx - ct * row_tiles) * RT;
    const int n0 = ct * COLS;
    if (tid < RT) {
      int64_t i = t.a + m0 + tid, src, dst;
      const bool in = i < t.b;
      i = in ? i : t.b - 1;
      const bool ok = gp_entry(p, i, src, dst) && in;
      row_src[tid] = (int32_t)src;
      row_dst[tid] = ok ? (int32_t)dst : -1;
      if constexpr (DT == DT_E4M3) row_xs[tid] = p.x_scale[src];
    }
    __syncthreads();

    // load b of this wave covers stage row trow (RT rows of x, then 64 of the
    // weights: UP 32 of gate and the same 32 of up), the lane one chunk of it
    const char* src[S::PER_WAVE];
    int chunk[S::PER_WAVE];
#pragma unroll
    for (int b = 0; b < S::PER_WAVE; ++b) {
      const int trow = (wv * S::PER_WAVE + b) * S::RPI + lane / S::LPR;
      chunk[b] = (lane % S::LPR) ^ blk_swz<128>(trow & 15);
      if (trow < RT) {
        src[b] = p.x + row_src[trow] * p.k_bytes;
      } else {
        int c = trow - RT;
        const char* w = p.w;
        if (UP && c >= 32) {
          w = p.w_up;
          c -= 32;
        }
        c = n0 + c < p.cols ? n0 + c : p.cols - 1;
        src[b] = w + ((int64_t)t.g * p.cols + c) * p.k_bytes;
      }
      src[b] += chunk[b] * 16;
    }
    // the stages in a circle from one of the column block's own: see GtLoads
    const int rot = nst > 0 ? (int)((unsigned)(t.g * 8 + ct) % (unsigned)nst) : 0;
    auto issue = [&](int i) {
      int s = (i < nst ? i : nst - 1) + rot;   // past the end: a harmless reload
      s = s < nst ? s : s - nst;
      char* dst = lds[i % NS];
#pragma unroll
      for (int b = 0; b < S::PER_WAVE; ++b)
        load_lds16(src[b] + (int64_t)s * 128, dst + (wv * S::PER_WAVE + b) * 1024);
    };
    f32x4_t acc[TI][2];   // [row tile][weight tile]
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto read = [&](const char* buf, u32x4_t (&fa)[2][TI], u32x4_t (&fb)[2][2]) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
        for (int i = 0; i < TI; ++i) fa[ks][i] = read_frag<128>(buf, wm + 16 * i, ks, n16, g);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          fb[ks][j] =
              read_frag<128>(buf, RT + (UP ? 32 * j + 16 * wn : 32 * wn + 16 * j), ks, n16, g);
      }
    };
    // weights as operand A: a lane ends with four neighbouring columns of a row
    auto mma = [&](const u32x4_t (&fa)[2][TI], const u32x4_t (&fb)[2][2]) {
      if constexpr (DT == DT_E4M3) {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = mfma_stage_e4m3(fb[0][j], fb[1][j], fa[0][i], fa[1][i], acc[i][j]);
      } else {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mfma_chunk<DT>(fb[ks][j], fa[ks][i], acc[i][j]);
      }
    };
    // this wave's loads of all but the `younger` latest stages have landed; the
    // barrier makes every wave's visible and ends every read of the buffer
    // that the next loads fill
    auto sync = [&](auto younger) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(younger)::value * S::PER_WAVE) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    if (nst > 0) {
#pragma unroll
      for (int i = 0; i < NS - 1; ++i) issue(i);
      if constexpr (NS == 2) {
        for (int i = 0; i < nst; ++i) {
          sync(std::integral_constant<int, 0>{});
          issue(i + 1);
          u32x4_t fa[2][TI], fb[2][2];
          read(lds[i % NS], fa, fb);
          mma(fa, fb);
          // (the products, and with them the waits for the reads, ahead of the
          // next barrier)
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        // one or two waves a SIMD: stage i + 1 is read while i is multiplied
        auto step = [&](int i, const u32x4_t (&ca)[2][TI], const u32x4_t (&cb)[2][2],
                        u32x4_t (&na)[2][TI], u32x4_t (&nb)[2][2]) {
          sync(std::integral_constant<int, NS - 3>{});
          read(lds[(i + 1) % NS], na, nb);
          issue(i + NS - 1);
          __builtin_amdgcn_sched_barrier(0);
          mma(ca, cb);
          __builtin_amdgcn_sched_barrier(0);
        };
        u32x4_t fa0[2][TI], fb0[2][2], fa1[2][TI], fb1[2][2];
        sync(std::integral_constant<int, NS - 2>{});
        read(lds[0], fa0, fb0);
        int i = 0;
        for (; i + 1 < nst; i += 2) {
          step(i, fa0, fb0, fa1, fb1);
          step(i + 1, fa1, fb1, fa0, fb0);
        }
        if (i < nst) step(i, fa0, fb0, fa1, fb1);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS is left
    }
    if (tail != 0) {   // the chunks past the last whole stage, zeros behind them
      __syncthreads();
#pragma unroll
      for (int b = 0; b < S::PER_WAVE; ++b) {
        const bool in = chunk[b] < tail;
        const u32x4_t v = ld16(src[b] - (in ? 0 : chunk[b] * 16) + (int64_t)nst * 128);
        st16(lds[0] + (wv * S::PER_WAVE + b) * 1024 + lane * 16, in ? v : u32x4_t{0, 0, 0, 0});
      }
      __syncthreads();
      u32x4_t fa[2][TI], fb[2][2];
      read(lds[0], fa, fb);
      mma(fa, fb);
    }

    constexpr int NJ = UP ? 1 : 2;
    int col[NJ];
    f32x4_t ws[NJ], us = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      col[j] = n0 + (UP ? 16 * wn : 32 * wn + 16 * j) + 4 * g;
      ws[j] = us;
    }
    if constexpr (DT == DT_E4M3) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int c = col[j] < p.cols ? col[j] : p.cols - 4;
        const int64_t at = (int64_t)t.g * p.cols + c;
        ws[j] = *reinterpret_cast<const f32x4_t*>(p.w_scale + at);
        if constexpr (UP) us = *reinterpret_cast<const f32x4_t*>(p.up_scale + at);
      }
    }
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int row = wm + 16 * i + n16;
      const int dst = row_dst[row];
      const float xs = DT == DT_E4M3 ? row_xs[row] : 1.f;
      if (dst < 0) continue;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (col[j] >= p.cols) continue;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          v[r] = gp_value<DT, UP>(acc[i][j][r], acc[i][1][r], xs, ws[j][r], us[r]);
        st_cols<ODT, 4>(p.out + ((int64_t)dst * p.cols + col[j]) * OES, v);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// many rows a group
// ---------------------------------------------------------------------------
// One launch of GT_GRID workgroups, each a CU's.  The tiles of the launch are
// numbered, workgroup s takes tiles s, s + GT_GRID, ...; where they lie is
// found GT_WINDOW at a time, in one pass over the offsets (GtPlan).
constexpr int GT_THREADS = 512, GT_GRID = 256, GT_WINDOW = 64;
// Column tiles of a band: the 32 tiles that an XCD has at a time are then four
// blocks of weights by eight of tokens (16 groups of 2048 rows, 4096 x 4096 in
// e4m3, 658 us row by row, 627 in bands of 4, 636 of 8).
constexpr int GT_BAND = 4;
enum : int { GT_WHOLE = 0, GT_HALF = 1 };   // 256 x 256, 128 x 256

struct GtLds {
  int4 tile[GT_WINDOW];        // group (-1: none), first row in it, first column, kind
  int32_t src[256], dst[256];  // a tile's rows: row of x, row of out (-1: not stored)
  float xs[256];
  int scan[GT_THREADS / 64];
  int total[2];
  // whole and half row blocks before each thread's groups (in LDS: nothing but
  // scalars may live beside a tile's accumulators)
  int before[2][GT_THREADS];
};

// When the longest of GT_GRID workgroups is done, in hundredths of a whole tile's
// time, with the whole tiles dealt in turn and then the halves, in whose later
// turns the workgroups without a tile of the last round of whole ones are first.
template <int DT>
__host__ __device__ __forceinline__ int64_t gt_span(int64_t whole, int64_t halves) {
  constexpr int HALF = DT == DT_F32 ? 55 : 65;
  const int64_t full = whole / GT_GRID * 100, busy = whole % GT_GRID, free = GT_GRID - busy;
  if (halves <= free) return full + (busy != 0 ? 100 : halves != 0 ? HALF : 0);
  const int64_t turn = (halves - free - 1) / GT_GRID, in = (halves - free - 1) % GT_GRID;
  return full + (in < free ? HALF * (2 + turn) : 100 + HALF * (1 + turn));
}
// The whole tiles of the last round to be cut in two: all or none, whichever is
// done earlier.
template <int DT>
__host__ __device__ __forceinline__ int64_t gt_cut(int64_t whole, int64_t halves) {
  const int64_t rem = whole % GT_GRID;
  return gt_span<DT>(whole - rem, halves + 2 * rem) < gt_span<DT>(whole, halves) ? rem : 0;
}

// The launch's tiles: a group has a row block for every 256 rows, a last one of
// at most 128 rows as a half.
struct GtPlan {
  int64_t whole, halves, cut;   // whole tiles, the groups' own halves, whole tiles cut in two
  int64_t units;
};
template <int DT>
__device__ __forceinline__ GtPlan gt_plan(int blocks, int own_halves, int tn) {
  GtPlan pl;
  const int64_t all = (int64_t)blocks * tn;
  pl.halves = (int64_t)own_halves * tn;
  pl.cut = gt_cut<DT>(all, pl.halves);
  pl.whole = all - pl.cut;
  pl.units = pl.whole + pl.halves + 2 * pl.cut;
  return pl;
}

// PgLoads with the stages taken in another order: in aligned blocks of a power
// of two, stage s ^ turn.
template <class S>
struct GtLoads : PgLoads<S> {
  int turn, blocked;   // turn is below the power; stages in whole blocks
  __device__ __forceinline__ int at(int stage) const {
    const int s = stage < this->last ? stage : this->last;
    return (s < blocked ? s ^ turn : s) * 128;
  }
  __device__ __forceinline__ void a(int h, int stage, char* dst) const {
    const int k = at(stage);
#pragma unroll
    for (int q = 0; q < S::PA; ++q) load_lds16_at(this->a_base, this->oa[h][q], k, dst + q * 1024);
  }
  __device__ __forceinline__ void b(int h, int stage, char* dst) const {
    const int k = at(stage);
#pragma unroll
    for (int q = 0; q < S::PB; ++q)
      load_lds16_at(this->b_base[h], this->ob[h][q], k, dst + q * 1024);
  }
};

// One tile of kind (MI, NJ): the group's rows from m0, output columns from n0.
template <int DT, int MI, int NJ, bool UP>
__device__ __forceinline__ void grouped_tile(const GroupedParams& p, char* lds, GtLds& gl, int grp,
                                             int64_t m0, int n0) {
  using S = PgShape<MI, NJ>;
  constexpr int ODT = DT == DT_E4M3 ? DT_BF16 : DT;
  constexpr int OES = ODT == DT_BF16 ? 2 : 4;
  // opaque, so that nothing of a tile is computed ahead of the loop over the
  // tiles: kept in registers beside the accumulators it would be spilled, and
  // a reload inside the stage loop waits for every load in flight
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  int ra, rb;
  gp_rows(p, grp, ra, rb);
  const int64_t ga = ra, gb = rb;
  __syncthreads();   // the tile before this one is done with its rows and stages
  if (tid < S::BM) {
    int64_t i = ga + m0 + tid, src, dst;
    const bool in = i < gb;
    i = in ? i : gb - 1;
    const bool ok = gp_entry(p, i, src, dst) && in;
    gl.src[tid] = (int32_t)src;
    gl.dst[tid] = ok ? (int32_t)dst : -1;
    if constexpr (DT == DT_E4M3) gl.xs[tid] = p.x_scale[src];
  }
  __syncthreads();

  PgLoop<DT, MI, NJ> L(lds, tid);
  GtLoads<S> ld;
  const int nst = (int)(p.k_bytes / 128);
  ld.last = nst - 1;
  // gathered rows count from the operand's first row, others from the tile's
  const int64_t base = p.picks != 0 ? 0 : ga + m0;
  ld.a_base = p.x + base * p.k_bytes;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int q = 0; q < S::PA; ++q)
      ld.oa[h][q] = (uint32_t)((gl.src[h * S::HM + L.a_row(q)] - base) * p.k_bytes) +
                    L.a_chunk(q) * 16;
    const int nh = n0 + (UP ? 0 : h * S::HN);   // first weight row of the half
    const int first = nh < p.cols ? nh : p.cols - 1;
    ld.b_base[h] = (UP && h == 1 ? p.w_up : p.w) + ((int64_t)grp * p.cols + first) * p.k_bytes;
#pragma unroll
    for (int q = 0; q < S::PB; ++q) {
      int r = nh + L.b_row(q);
      r = r < p.cols ? r : p.cols - 1;
      ld.ob[h][q] = (uint32_t)((r - first) * p.k_bytes) + L.b_chunk(q) * 16;
    }
  }
  f32x4_t acc[2][2][MI][NJ];
  // Rows lie a multiple of some KiB apart, so tiles that are at the same stage
  // read the same few channels of L2 and of memory: each takes the stages in an
  // order of its own.  A group of one row block, whose weights are read once,
  // has all stages to choose from (64 groups of 64 rows, 2048 x 2048, 161 -> 139
  // us).  Else what an XCD's tiles read has to stay in its L2 meanwhile: eight
  // stages, the same order for tiles of the same rows, another one in every XCD
  // (16 groups of 2048 rows, 4096 x 4096 in e4m3, 627 -> 540 us; 16 stages 547; 32
  // groups of 1024 rows, 4096 x 4096 in bf16, 1120 -> 969; float32 the same).
  int power = 8;
  ld.turn = blockIdx.x / (8 * GT_BAND) + blockIdx.x;
  if (gb - ga <= 128) {
    for (power = 1; 2 * power <= nst;) power *= 2;
    ld.turn = grp * 8 + n0 / 64;
  }
  ld.turn &= power - 1;
  ld.blocked = nst & -power;
  L.run(nst, ld, acc, [](int, int) {});

  // the chunks past the last whole stage, zeros behind them
  const int tail = (int)(p.k_bytes / 16) - 8 * nst;
  if (tail != 0) {
    __syncthreads();
    auto fill = [&](const char* base, uint32_t off, int chunk, char* dst) {
      const bool in = chunk < tail;
      const u32x4_t v = ld16(base + (off - (in ? 0 : chunk * 16)) + (int64_t)nst * 128);
      st16(dst + L.lane * 16, in ? v : u32x4_t{0, 0, 0, 0});
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int q = 0; q < S::PA; ++q)
        fill(ld.a_base, ld.oa[h][q], L.a_chunk(q), L.a_dst(h, 0) + q * 1024);
#pragma unroll
      for (int q = 0; q < S::PB; ++q)
        fill(ld.b_base[h], ld.ob[h][q], L.b_chunk(q), L.b_dst(h, 0) + q * 1024);
    }
    __syncthreads();
    u32x4_t fa[2][MI], fb[2][NJ];
#pragma unroll
    for (int qi = 0; qi < 2; ++qi) {
      L.read_a(qi, 0, fa);
#pragma unroll
      for (int qj = 0; qj < 2; ++qj) {
        L.read_b(qj, 0, fb);
        L.mma(fa, fb, acc[qi][qj]);
      }
    }
  }

  // a lane holds W neighbouring columns of a row in every quadrant, stored in
  // pieces of at most 16 bytes (cols is a multiple of a 16-byte piece)
  constexpr int W = S::W, QJ = UP ? 1 : 2, PC = W * OES < 16 ? W : 16 / OES, NP = W / PC;
  int col[QJ][NP];
  float ws[QJ][W], us[W];
#pragma unroll
  for (int qj = 0; qj < QJ; ++qj)
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      col[qj][k] = n0 + qj * S::HN + L.wc * 16 * NJ + W * L.g + PC * k;
#pragma unroll
      for (int r = 0; r < PC; ++r) {
        ws[qj][PC * k + r] = us[PC * k + r] = 1.f;
        if constexpr (DT == DT_E4M3) {
          const int c = col[qj][k] < p.cols ? col[qj][k] : p.cols - PC;
          ws[qj][PC * k + r] = p.w_scale[(int64_t)grp * p.cols + c + r];
          if constexpr (UP) us[PC * k + r] = p.up_scale[(int64_t)grp * p.cols + c + r];
        }
      }
    }
#pragma unroll
  for (int qi = 0; qi < 2; ++qi)
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int row = qi * S::HM + L.wr * 16 * MI + 16 * i + L.n16;
      const int dst = gl.dst[row];
      const float xs = DT == DT_E4M3 ? gl.xs[row] : 1.f;
      if (dst < 0) continue;
#pragma unroll
      for (int qj = 0; qj < QJ; ++qj)
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          if (col[qj][k] >= p.cols) continue;
          float v[PC];
#pragma unroll
          for (int r = 0; r < PC; ++r) {
            const int x = PC * k + r;
            v[r] = gp_value<DT, UP>(acc[qi][qj][i][x >> 2][x & 3], acc[qi][1][i][x >> 2][x & 3],
                                    xs, ws[qj][x], us[x]);
          }
          st_cols<ODT, PC>(p.out + ((int64_t)dst * p.cols + col[qj][k]) * OES, v);
        }
    }
}

template <int DT, bool UP>
__global__ __launch_bounds__(GT_THREADS, 2) void grouped_tiles_kernel(GroupedParams p) {
  // One object: the compiler puts a wait for every load into LDS before a read of
  // one of several (16 groups of 2048 rows, 4096 x 4096 in e4m3, 532 -> 506 us, 64 of 1024,
  // 2048 x 2048 in bf16, 573 -> 522).
  constexpr int STAGES = 2 * PgShape<4, 2>::BUF;
  __shared__ __attribute__((aligned(1024))) char lds[STAGES + sizeof(GtLds)];
  GtLds& gl = *reinterpret_cast<GtLds*>(lds + STAGES);
  constexpr int TC = UP ? 128 : 256;   // output columns of a tile
  const int tn = (p.cols + TC - 1) / TC;
  // neighbouring tiles on one XCD
  const int slot = (blockIdx.x & 7) * (GT_GRID / 8) + (blockIdx.x >> 3);

  // this thread's groups and the numbers of row blocks before them
  const int per = (p.groups + GT_THREADS - 1) / GT_THREADS;
  auto blocks = [&](int g, int& whole, int& half) {
    int a, b;
    gp_rows(p, g, a, b);
    const int r = b - a, rem = r & 255;
    half = rem > 0 && rem <= 128 ? 1 : 0;
    whole = (r >> 8) + (rem > 128 ? 1 : 0);
  };
  {
    int n[2] = {0, 0};
    const int g0 = threadIdx.x * per;
    for (int g = g0; g < g0 + per && g < p.groups; ++g) {
      int b, h;
      blocks(g, b, h);
      n[0] += b;
      n[1] += h;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int incl = block_scan_incl<GT_THREADS / 64>(n[c], gl.scan);
      gl.before[c][threadIdx.x] = incl - n[c];
      if (threadIdx.x == GT_THREADS - 1) gl.total[c] = incl;
    }
  }
  __syncthreads();
  const GtPlan pl = gt_plan<DT>(__builtin_amdgcn_readfirstlane(gl.total[0]),
                                __builtin_amdgcn_readfirstlane(gl.total[1]), tn);

  // this workgroup's unit number k: from the halves' second turn on those without
  // a tile in the last round of whole ones are the first
  const int64_t last = pl.whole / GT_GRID;
  const int turned = (slot - (int)(pl.whole % GT_GRID)) & (GT_GRID - 1);
  auto unit = [&](int64_t k) { return k * GT_GRID + (k > last ? turned : slot); };

  for (int64_t k0 = 0; unit(k0) < pl.units; k0 += GT_WINDOW) {
    __syncthreads();
    if (threadIdx.x < GT_WINDOW) gl.tile[threadIdx.x] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    // this workgroup's tiles among [lo, hi) that lie in the window
    auto mark = [&](int64_t lo, int64_t hi, auto&& where) {
      for (int64_t k = lo / GT_GRID < k0 ? k0 : lo / GT_GRID; k < k0 + GT_WINDOW; ++k) {
        const int64_t u = unit(k);
        if (u >= hi) break;
        if (u >= lo) gl.tile[k - k0] = where(u - lo);
      }
    };
    int64_t at = gl.before[0][threadIdx.x], athalf = gl.before[1][threadIdx.x];
    const int g0 = threadIdx.x * per;
    for (int g = g0; g < g0 + per && g < p.groups; ++g) {
      int b, h;
      blocks(g, b, h);
      const int64_t lo = at * tn, hi = (at + b) * tn;
      auto whole = [&](int64_t u) {   // bands of GT_BAND column tiles, the group's rows in each
        const int v = (int)u, w0 = v / (GT_BAND * b) * GT_BAND, in = v - w0 * b;
        const int w = tn - w0 < GT_BAND ? tn - w0 : GT_BAND;
        return make_int4(g, in / w * 256, (w0 + in % w) * TC, GT_WHOLE);
      };
      mark(lo, hi < pl.whole ? hi : pl.whole, whole);
      if (h != 0)
        mark(pl.whole + athalf * tn, pl.whole + (athalf + 1) * tn,
             [&](int64_t u) { return make_int4(g, b * 256, (int)u * TC, GT_HALF); });
      const int64_t c0 = lo > pl.whole ? lo : pl.whole;   // its tiles that are cut
      if (c0 < hi)
        mark(pl.whole + pl.halves + 2 * (c0 - pl.whole), pl.whole + pl.halves + 2 * (hi - pl.whole),
             [&](int64_t u) {
               int4 t = whole(c0 - lo + (u >> 1));
               t.y += (int)(u & 1) * 128;
               t.w = GT_HALF;
               return t;
             });
      at += b;
      athalf += h;
    }
    __syncthreads();
    for (int k = 0; k < GT_WINDOW; ++k) {
      const int4 t = gl.tile[k];
      const int g = __builtin_amdgcn_readfirstlane(t.x);
      if (g < 0) break;
      const int m0 = __builtin_amdgcn_readfirstlane(t.y);
      const int n0 = __builtin_amdgcn_readfirstlane(t.z);
      const int kind = __builtin_amdgcn_readfirstlane(t.w);
      if (kind == GT_WHOLE) grouped_tile<DT, 4, 2, UP>(p, lds, gl, g, m0, n0);
      else grouped_tile<DT, 2, 2, UP>(p, lds, gl, g, m0, n0);
    }
  }
}

// K over two waves, or over four where that is long (16 rows of one in 16
// matrices of 4096 x 4096 114 -> 93 us) or the workgroups are few.  Where these
// would be many, each takes several column tiles for the row tile it has found
// (4000 groups of one row, 256 x 512, one column tile a workgroup and four: 368
// and 252 us; from 4096 workgroups on 2 rows in 64 groups of 2048 x 2048 take 102
// us instead of 90).
static void plan_rows(int64_t m, int groups, int cols, int64_t k_bytes, GroupedPlan* pl) {
  const int64_t most = m / 16 + groups;   // row tiles: one a group, one for each 16 rows
  const int64_t tiles = most < m ? most : m;
  pl->kernel = GROUPED_ROWS;
  pl->rows = 16;
  pl->depth = k_bytes >= 8192 || tiles * ((cols + 31) / 32) < 1024 ? 4 : 2;
  const int64_t per = 16 * (GS_WAVES / pl->depth);   // columns of a column tile
  const int64_t tn = (cols + per - 1) / per;
  int64_t blocks = GS_BLOCKS / tiles;
  blocks = blocks < 1 ? 1 : blocks < tn ? blocks : tn;
  pl->span = (int)((tn + blocks - 1) / blocks);
  const int64_t n = tiles * ((tn + pl->span - 1) / pl->span);
  pl->blocks = (int)(n < GP_GRID ? n : GP_GRID);
}

static void plan_ring(int64_t m, int groups, int64_t tn, int depth, int rows, GroupedPlan* pl) {
  const int64_t most = m / rows + groups;
  int64_t tiles = (most < m ? most : m) * tn;
  tiles = (tiles + 7) / 8 * 8;   // xcd_remap deals whole rounds over the XCDs
  pl->kernel = GROUPED_RING;
  pl->depth = depth;
  pl->rows = rows;
  pl->blocks = (int)(tiles < GP_GRID ? tiles : GP_GRID);
}

// The host knows the groups' number and their rows together, so the rules go
// by the mean; a group far from it is computed on tiles that fit it less well: 64
// groups of 512 rows among 960 empty ones, 1024 x 1024 in bf16, 305 us on tiles
// of 32 rows, without the empty ones 83 (float32, 128 rows each, 525 and 155).
//
// Up to 4 rows a group (float32, bound by the matrix cores, 8) the few-rows
// kernel: 64 groups of 2048 x 2048, it and 32-row tiles, 1 row 92 and 94 us, 4
// rows 101 and 95, 16 rows 147 and 97 (537 MB of weights: 5.5 TB/s); 8 groups of
// 1 row, 1024 x 2048, 11 and 17.  Also while its workgroups, whose waves share
// K, are no more than the CUs (float32 without an up half twice that): 4 groups of
// 11 rows, 2048 x 256, 7.9 and 9.0 us, float32 10.6 and 25.0; one of 128 rows, 2048
// x 1024, 12.6 and 9.3; but not with two matrices a wave in fewer bits (4 groups of
// 11 rows, 2048 x 256, 10.1 and 9.1, float32 17.1 and 25.4).
// And up to 32 rows a group where these are no more than the groups that a thread
// looks through for a tile, which this kernel does once for several column tiles
// (10 rows in 16000 groups of 512 x 64 1.1 and 4.5 ms, 30 in 8000 of 256 x 128 0.60
// and 0.86; 20 in 4000 of 512 x 512 1.23 and 0.75).
// Then tiles of 32 rows, of 64 above 32 rows a group where these are enough (64
// groups of 64 rows 148 and 114 us; one of 512 rows 12 and 14), with deep rings
// while all tiles are resident at once: four stages of 32 rows leave three
// workgroups a CU (768), of 64 rows two (512) (one group of 512 rows 12.4 us with 4
// stages, 13.7 with 3; of 2048 rows on 64-row tiles 30.6 us with 2, 35.7 with 4).
// float32, which the matrix cores bound, takes two stages only between 512 and 1024
// tiles of 64 rows, which are all resident with two and not with four (13 groups of
// 231 rows, 840 x 1160, 71 and 92), and four again beyond (16 of 256 rows 309 us with
// 2, 301 with 4).
// The large tiles where their rounds cost less: one of 256 whole ones takes as
// long as `round` 64 x 64 ones, one of halves 65% of that, float32 55% (2048 x
// 2048, 64-row tiles and large ones, bf16: 64 groups of 64 rows 114 and 117 us, of
// 96 169 and 120, of 256 293 and 170; 16 of 128 33 and 48, of 256 60 and 42; one of
// 2048 31 and 39; e4m3 16 of 256 38 and 30; 64 groups of 80 rows on average 168 and
// 120).  For float32, whose large tiles lose most by a round that is not full,
// the rule supposes groups of any size, and keeps even ones of 256, 512 or 80 rows,
// which would fill it, on rings (16 of 256 rows 309 us, on large tiles 268; of 512
// 576 and 492; 64 of 80 626 and 540; 13 groups of 231 rows, 840 x 1160, 72 and 154).
template <int DT, bool UP>
static GroupedPlan plan_dt(int64_t m, int groups, int cols, int64_t k_bytes, int picks,
                           int64_t x_rows) {
  const int64_t used = groups < m ? groups : m;
  const int64_t tn = (cols + (UP ? 127 : 255)) / (UP ? 128 : 256);
  const int64_t tn64 = (cols + (UP ? 31 : 63)) / (UP ? 32 : 64);
  // half a row tile of padding a group, half of the groups with a half tile
  const int64_t tiles64 = (m / 64 + used / 2 + 1) * tn64;
  constexpr int few = DT == DT_F32 ? (UP ? 256 : 512) : (UP ? 0 : 256);
  const int64_t tiles16 = used * ((m + 16 * used - 1) / (16 * used)) * (int64_t)((cols + 15) / 16);
  // large tiles as the mean has it: up to 128 rows a half a group, up to 224 a whole
  // one; above, where any place in a last block is as likely (float32, which loses
  // most by a second round, above 128), a whole one for every 256 rows and for
  // every second group a half
  const bool half = m <= 128 * used, one = !half && DT != DT_F32 && m <= 224 * used;
  const int64_t whole = half ? 0 : one ? used * tn : m * tn / 256;
  const int64_t halves = half ? used * tn : one ? 0 : (used + 1) / 2 * tn;
  const int64_t cut = gt_cut<DT>(whole, halves);
  const int64_t span = gt_span<DT>(whole - cut, halves + 2 * cut);
  const int64_t round = DT == DT_F32 ? 3340 : DT == DT_E4M3 ? 2400 : 2100;
  // (the phased kernel's lane offsets are 32-bit)
  const bool near = k_bytes < (4 << 20) &&
                    (picks == 0 || x_rows * k_bytes < ((int64_t)1 << 32));
  GroupedPlan pl{};
  if (span * round < 100 * tiles64 && k_bytes >= 128 && near) {
    pl.kernel = GROUPED_TILES;
    pl.blocks = GT_GRID;
  } else if (m <= (DT == DT_F32 ? 8 : 4) * used || tiles16 <= few ||
             (m <= 32 * used && m <= (groups / GS_THREADS) * used)) {
    plan_rows(m, groups, cols, k_bytes, &pl);
  } else if (m <= 32 * used || tiles64 <= 256) {
    plan_ring(m, groups, tn64, (m / 32 + used / 2 + 1) * tn64 <= 768 ? 4 : 3, 32, &pl);
  } else {
    plan_ring(m, groups, tn64, tiles64 <= 512 || (DT == DT_F32 && tiles64 > 1024) ? 4 : 2, 64,
              &pl);
  }
  return pl;
}

template <int DT, bool UP>
static hipError_t launch_plan(GroupedParams p, const GroupedPlan& pl, hipStream_t st) {
  const dim3 grid((unsigned)pl.blocks);
  p.span = pl.span;
  if (pl.kernel == GROUPED_TILES)
    return launch_kernel(grouped_tiles_kernel<DT, UP>, grid, dim3(GT_THREADS), 0, st, p);
  if (pl.kernel == GROUPED_ROWS && pl.depth == 4)
    return launch_kernel(grouped_rows_kernel<DT, 4, UP>, grid, dim3(GS_THREADS), 0, st, p);
  if (pl.kernel == GROUPED_ROWS)
    return launch_kernel(grouped_rows_kernel<DT, 2, UP>, grid, dim3(GS_THREADS), 0, st, p);
  if (pl.rows == 32 && pl.depth == 4)
    return launch_kernel(grouped_mid_kernel<DT, 4, 1, UP>, grid, dim3(GM_THREADS), 0, st, p);
  if (pl.rows == 32)
    return launch_kernel(grouped_mid_kernel<DT, 3, 1, UP>, grid, dim3(GM_THREADS), 0, st, p);
  if (pl.depth == 4)
    return launch_kernel(grouped_mid_kernel<DT, 4, 2, UP>, grid, dim3(GM_THREADS), 0, st, p);
  return launch_kernel(grouped_mid_kernel<DT, 2, 2, UP>, grid, dim3(GM_THREADS), 0, st, p);
}

GroupedPlan grouped_plan(int dt, bool up, int64_t m, int groups, int cols, int64_t k_bytes,
                         int picks, int64_t x_rows) {
  const auto plan = dt == DT_BF16 ? (up ? plan_dt<DT_BF16, true> : plan_dt<DT_BF16, false>)
                    : dt == DT_F32 ? (up ? plan_dt<DT_F32, true> : plan_dt<DT_F32, false>)
                                   : (up ? plan_dt<DT_E4M3, true> : plan_dt<DT_E4M3, false>);
  return plan(m, groups, cols, k_bytes, picks, x_rows);
}

hipError_t launch_grouped(int dt, const GroupedParams& p, hipStream_t st) {
  if (p.m == 0) return hipSuccess;
  const bool up = p.w_up != nullptr;
  const GroupedPlan pl = grouped_plan(dt, up, p.m, p.groups, p.cols, p.k_bytes, p.picks, p.x_rows);
  switch (dt) {
    case DT_BF16: return up ? launch_plan<DT_BF16, true>(p, pl, st)
                            : launch_plan<DT_BF16, false>(p, pl, st);
    case DT_F32: return up ? launch_plan<DT_F32, true>(p, pl, st)
                           : launch_plan<DT_F32, false>(p, pl, st);
    default: return up ? launch_plan<DT_E4M3, true>(p, pl, st)
                       : launch_plan<DT_E4M3, false>(p, pl, st);
  }
}

}  // namespace lookme
