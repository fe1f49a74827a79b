// Products of rows that come grouped, every group with a matrix of its own (the
// rows of a scene of Eq. 5 with that scene's matrices, the rows of an expert):
//
//   out[i] = round(W[g] x[src(i)])                       for i in group g, or
//   out[i] = round(silu(W[g] x[src(i)]) * (W_up[g] x[src(i)]))
//
// The groups' sizes are on the device only.  A workgroup finds its tile by a
// prefix sum over the groups' tile counts (find_tile), so no tile spans two
// groups, and empty groups cost nothing.  Two kernels:
//
//   grouped_rows_kernel   few rows a group: bound by the stream of the weights
//       out of HBM.  A wave multiplies 16 weight rows by 16 NT tokens straight
//       from global memory (both operands are K-contiguous, a lane's 16 bytes
//       are its fragment), D steps in flight in registers, K split over the
//       waves of a workgroup and summed through LDS.
//   grouped_tiles_kernel  many rows a group: 256 x 256, 128 x 256 and 128 x 128
//       tiles on the phased loop of phase_gemm.h, one workgroup a CU that takes
//       tile after tile.
//
// e4m3 operands carry a float32 scale a row, applied once to the float32 sum:
// out = round(xs ws sum).
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

// rows [a, b) of group g, kept inside [0, m) whatever the offsets hold
__device__ __forceinline__ void gp_rows(const GroupedParams& p, int g, int64_t& a, int64_t& b) {
  a = p.offsets[g];
  b = p.offsets[g + 1];
  a = a < 0 ? 0 : (a > p.m ? p.m : a);
  b = b < a ? a : (b > p.m ? p.m : b);
}

// Tile number `unit` in the groups' order, count(rows) tiles a group; all
// threads of the block.  Returns the number of tiles; t.g is -1 past the last.
template <int THREADS, class Count>
__device__ __forceinline__ int find_tile(const GroupedParams& p, int unit, int* lds, GpTile& t,
                                         Count&& count) {
  const int per = (p.groups + THREADS - 1) / THREADS;
  const int first = threadIdx.x * per;
  const int last = first + per < p.groups ? first + per : p.groups;
  int sum = 0;
  for (int g = first; g < last; ++g) {
    int64_t a, b;
    gp_rows(p, g, a, b);
    sum += count(b - a);
  }
  if (threadIdx.x == 0) lds[0] = -1;
  const int incl = block_scan_incl<THREADS / 64>(sum, lds + 3);
  int at = incl - sum;
  if (at <= unit && unit < incl) {
    for (int g = first; g < last; ++g) {
      int64_t a, b;
      gp_rows(p, g, a, b);
      const int c = count(b - a);
      if (unit < at + c) {
        lds[0] = g;
        lds[1] = unit - at;
        break;
      }
      at += c;
    }
  }
  if (threadIdx.x == THREADS - 1) lds[2] = incl;
  __syncthreads();
  t.g = __builtin_amdgcn_readfirstlane(lds[0]);
  t.idx = __builtin_amdgcn_readfirstlane(lds[1]);
  const int total = __builtin_amdgcn_readfirstlane(lds[2]);
  __syncthreads();
  if (t.g >= 0) gp_rows(p, t.g, t.a, t.b);
  return total;
}
constexpr int GP_FIND_LDS = 3 + 16;

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

// float32 sums of one output and of its up half, made an output value
template <int DT, bool UP>
__device__ __forceinline__ float gp_value(float c, float u, float xs, float ws, float us) {
  if constexpr (DT == DT_E4M3) {
    c *= xs * ws;
    u *= xs * us;
  }
  return UP ? silu_f(c) * u : c;
}

// ---------------------------------------------------------------------------
// few rows a group
// ---------------------------------------------------------------------------
constexpr int GS_THREADS = 256, GS_WAVES = 4;

// NT: token tiles of 16.  KS: waves that share the K of 16 weight rows; the
// workgroup's other waves take other rows.  D: steps (64 bytes of K) in flight.
template <int DT, int NT, int KS, int D, bool UP>
__global__ __launch_bounds__(GS_THREADS) void grouped_rows_kernel(GroupedParams p) {
  constexpr int ODT = DT == DT_E4M3 ? DT_BF16 : DT;
  constexpr int OES = ODT == DT_BF16 ? 2 : 4;
  constexpr int MATS = UP ? 2 : 1;
  constexpr int COLS = 16 * (GS_WAVES / KS);
  __shared__ int find_lds[GP_FIND_LDS];
  __shared__ f32x4_t part[KS > 1 ? GS_WAVES * MATS * NT * 64 : 1];
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

  for (int64_t unit = blockIdx.x;; unit += gridDim.x) {
    const int row_tile = (int)(unit / tiles_n);
    GpTile t;
    find_tile<GS_THREADS>(p, row_tile, find_lds, t,
                          [](int64_t r) { return (int)((r + 16 * NT - 1) / (16 * NT)); });
    if (t.g < 0) return;
    const int c0 = (int)(unit - (int64_t)row_tile * tiles_n) * COLS + 16 * (wv / KS);

    int64_t dst[NT];
    bool ok[NT];
    float xs[NT];
    const char* xp[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      int64_t i = t.a + (int64_t)t.idx * (16 * NT) + 16 * j + n16, src;
      const bool in = i < t.b;
      i = in ? i : t.b - 1;
      ok[j] = gp_entry(p, i, src, dst[j]) && in;
      xp[j] = p.x + src * p.k_bytes;
      xs[j] = 1.f;
      if constexpr (DT == DT_E4M3) xs[j] = p.x_scale[src];
    }
    const int wc = c0 + n16 < p.cols ? c0 + n16 : p.cols - 1;
    const int64_t wrow = ((int64_t)t.g * p.cols + wc) * p.k_bytes;
    const char* wp[MATS];
    wp[0] = p.w + wrow;
    if constexpr (UP) wp[1] = p.w_up + wrow;

    f32x4_t acc[MATS][NT];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    u32x4_t fw[D][MATS], fx[D][NT];
    // unconditional loads from clamped addresses; chunks past K count as zero
    auto load = [&](int d, int s) {
      int c = 4 * s + g;
      c = c < chunks ? c : chunks - 1;
#pragma unroll
      for (int q = 0; q < MATS; ++q) fw[d][q] = ld16_nt(wp[q] + (int64_t)c * 16);
#pragma unroll
      for (int j = 0; j < NT; ++j) fx[d][j] = ld16(xp[j] + (int64_t)c * 16);
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
          const bool in = s + d < s1 && 4 * (s + d) + g < chunks;
          u32x4_t w[MATS], x[NT];
#pragma unroll
          for (int q = 0; q < MATS; ++q) w[q] = in ? fw[d][q] : u32x4_t{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < NT; ++j) x[j] = in ? fx[d][j] : u32x4_t{0, 0, 0, 0};
          load(d, s + d + D);
#pragma unroll
          for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[q][j] = mfma_chunk<DT>(w[q], x[j], acc[q][j]);
        }
      }
    }
    if constexpr (KS > 1) {
      f32x4_t* mine = part + wv * (MATS * NT * 64) + lane;
      if (kp != 0) {
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
          for (int j = 0; j < NT; ++j) mine[(q * NT + j) * 64] = acc[q][j];
      }
      __syncthreads();   // (the next unit's find_tile keeps its writes behind these reads)
      if (kp != 0) continue;
#pragma unroll
      for (int o = 1; o < KS; ++o)
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const f32x4_t v = mine[(o * MATS * NT + q * NT + j) * 64];
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[q][j][r] += v[r];
          }
    }
    // the lane holds columns c0 + 4 g + r of its tokens' rows (cols is a
    // multiple of 4)
    const int col = c0 + 4 * g;
    if (col >= p.cols) continue;
    f32x4_t ws = {1.f, 1.f, 1.f, 1.f}, us = ws;
    if constexpr (DT == DT_E4M3) {
      const int64_t s = (int64_t)t.g * p.cols + col;
      ws = *reinterpret_cast<const f32x4_t*>(p.w_scale + s);
      if constexpr (UP) us = *reinterpret_cast<const f32x4_t*>(p.up_scale + s);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if (!ok[j]) continue;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = gp_value<DT, UP>(acc[0][j][r], UP ? acc[MATS - 1][j][r] : 0.f, xs[j], ws[r], us[r]);
      st_cols<ODT, 4>(p.out + (dst[j] * p.cols + col) * OES, v);
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
enum : int { GT_WHOLE = 0, GT_HALF = 1, GT_QUARTER = 2 };   // 256 x 256, 128 x 256, 128 x 128

struct GtLds {
  int4 tile[GT_WINDOW];        // group (-1: none), first row in it, first column, kind
  int32_t src[256], dst[256];  // a tile's rows: row of x, row of out (-1: not stored)
  float xs[256];
  int scan[GT_THREADS / 64];
  int total[3];
  // row blocks before each thread's groups (in LDS: nothing but scalars may
  // live beside a tile's accumulators)
  int before[3][GT_THREADS];
};

// The launch's tiles.  In 256 x 256 tiles a group has a row block for every 256
// rows, a last one of at most 128 rows as a half; when the last round of whole
// tiles would be at most half full its tiles are cut in halves too.  Where
// that leaves most CUs idle the launch is all quarters.  A half round takes
// about 0.55 of a whole one's time, a round of quarters a third.
struct GtPlan {
  int64_t whole, halves, cut;   // whole tiles, a group's own halves, whole tiles cut in two
  int64_t units;
  bool quarters;
};
__device__ __forceinline__ GtPlan gt_plan(int blocks256, int blocks128, int own_halves, int tn,
                                          int tn_quarter) {
  GtPlan pl;
  const int64_t all = (int64_t)blocks256 * tn;
  const int64_t rem = all % GT_GRID;
  pl.cut = rem <= GT_GRID / 2 ? rem : 0;
  pl.whole = all - pl.cut;
  pl.halves = (int64_t)own_halves * tn;
  const int64_t quarters = (int64_t)blocks128 * tn_quarter;
  auto rounds = [](int64_t n) { return (float)((n + GT_GRID - 1) / GT_GRID); };
  pl.quarters = 0.33f * rounds(quarters) <
                rounds(pl.whole) + 0.55f * rounds(pl.halves + 2 * pl.cut);
  pl.units = pl.quarters ? quarters : pl.whole + pl.halves + 2 * pl.cut;
  return pl;
}

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
  int64_t ga, gb;
  gp_rows(p, grp, ga, gb);
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
  PgLoads<S> ld;
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
  __shared__ __attribute__((aligned(1024))) char lds[2 * PgShape<4, 2>::BUF];
  __shared__ GtLds gl;
  constexpr int TC = UP ? 128 : 256, QC = UP ? 64 : 128;   // output columns of a tile
  const int tn = (p.cols + TC - 1) / TC, tq = (p.cols + QC - 1) / QC;
  // neighbouring tiles on one XCD
  const int slot = (blockIdx.x & 7) * (GT_GRID / 8) + (blockIdx.x >> 3);

  // this thread's groups and the numbers of row blocks before them
  const int per = (p.groups + GT_THREADS - 1) / GT_THREADS;
  auto blocks = [&](int g, int& b256, int& b128, int& half) {
    int64_t a, b;
    gp_rows(p, g, a, b);
    const int r = (int)(b - a), rem = r & 255;
    half = rem > 0 && rem <= 128 ? 1 : 0;
    b256 = (r >> 8) + (rem > 128 ? 1 : 0);
    b128 = (r + 127) >> 7;
  };
  {
    int n[3] = {0, 0, 0};
    const int g0 = threadIdx.x * per;
    for (int g = g0; g < g0 + per && g < p.groups; ++g) {
      int b, q, h;
      blocks(g, b, q, h);
      n[0] += b;
      n[1] += q;
      n[2] += h;
    }
#pragma unroll
    for (int c = 0; c < 3; ++c) {
      const int incl = block_scan_incl<GT_THREADS / 64>(n[c], gl.scan);
      gl.before[c][threadIdx.x] = incl - n[c];
      if (threadIdx.x == GT_THREADS - 1) gl.total[c] = incl;
    }
  }
  __syncthreads();
  const GtPlan pl = gt_plan(__builtin_amdgcn_readfirstlane(gl.total[0]),
                            __builtin_amdgcn_readfirstlane(gl.total[1]),
                            __builtin_amdgcn_readfirstlane(gl.total[2]), tn, tq);

  for (int64_t k0 = 0; slot + k0 * GT_GRID < pl.units; k0 += GT_WINDOW) {
    __syncthreads();
    if (threadIdx.x < GT_WINDOW) gl.tile[threadIdx.x] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    // this workgroup's tiles among [lo, hi) that lie in the window
    auto mark = [&](int64_t lo, int64_t hi, auto&& where) {
      int64_t k = lo <= slot ? 0 : (lo - slot + GT_GRID - 1) / GT_GRID;
      for (k = k < k0 ? k0 : k; k < k0 + GT_WINDOW; ++k) {
        const int64_t u = slot + k * GT_GRID;
        if (u >= hi) break;
        gl.tile[k - k0] = where(u - lo);
      }
    };
    int64_t at256 = gl.before[0][threadIdx.x], at128 = gl.before[1][threadIdx.x];
    int64_t athalf = gl.before[2][threadIdx.x];
    const int g0 = threadIdx.x * per;
    for (int g = g0; g < g0 + per && g < p.groups; ++g) {
      int b, q, h;
      blocks(g, b, q, h);
      if (pl.quarters) {
        mark(at128 * tq, (at128 + q) * tq, [&](int64_t u) {
          return make_int4(g, (int)(u / tq) * 128, (int)(u % tq) * QC, GT_QUARTER);
        });
      } else {
        const int64_t lo = at256 * tn, hi = (at256 + b) * tn;
        auto whole = [&](int64_t u) {
          return make_int4(g, (int)(u / tn) * 256, (int)(u % tn) * TC, GT_WHOLE);
        };
        mark(lo, hi < pl.whole ? hi : pl.whole, whole);
        if (h != 0)
          mark(pl.whole + athalf * tn, pl.whole + (athalf + 1) * tn, [&](int64_t u) {
            return make_int4(g, b * 256, (int)u * TC, GT_HALF);
          });
        const int64_t c0 = lo > pl.whole ? lo : pl.whole;   // its tiles that are cut
        if (c0 < hi)
          mark(pl.whole + pl.halves + 2 * (c0 - pl.whole),
               pl.whole + pl.halves + 2 * (hi - pl.whole), [&](int64_t u) {
                 int4 t = whole(c0 - lo + (u >> 1));
                 t.y += (int)(u & 1) * 128;
                 t.w = GT_HALF;
                 return t;
               });
      }
      at256 += b;
      at128 += q;
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
      else if (kind == GT_HALF) grouped_tile<DT, 2, 2, UP>(p, lds, gl, g, m0, n0);
      else grouped_tile<DT, 2, 1, UP>(p, lds, gl, g, m0, n0);
    }
  }
}

// ---------------------------------------------------------------------------

template <int DT, int NT, int KS, int D, bool UP>
static hipError_t launch_rows(const GroupedParams& p, hipStream_t st) {
  constexpr int COLS = 16 * (GS_WAVES / KS);
  // row tiles: at most one a group and one more for each 16 NT rows
  const int64_t most = p.m / (16 * NT) + p.groups;
  int64_t tiles = (most < p.m ? most : p.m) * ((p.cols + COLS - 1) / COLS);
  tiles = tiles < 65536 ? tiles : 65536;
  hipLaunchKernelGGL((grouped_rows_kernel<DT, NT, KS, D, UP>), dim3((unsigned)tiles),
                     dim3(GS_THREADS), 0, st, p);
  return hipGetLastError();
}

template <int DT, bool UP>
static hipError_t launch_grouped_dt(const GroupedParams& p, hipStream_t st) {
  // the phased kernel's lane offsets are 32-bit
  const bool near = p.k_bytes < (4 << 20) &&
                    (p.picks == 0 || p.x_rows * p.k_bytes < ((int64_t)1 << 32));
  if (p.m > 32 * (int64_t)p.groups && p.k_bytes >= 128 && near) {
    hipLaunchKernelGGL((grouped_tiles_kernel<DT, UP>), dim3(GT_GRID),
                       dim3(GT_THREADS), 0, st, p);
    return hipGetLastError();
  }
  if (p.m > 8 * (int64_t)p.groups) return launch_rows<DT, 2, 4, 4, UP>(p, st);
  return launch_rows<DT, 1, 4, 4, UP>(p, st);
}

hipError_t launch_grouped(int dt, const GroupedParams& p, hipStream_t st) {
  if (p.m == 0) return hipSuccess;
  const bool up = p.w_up != nullptr;
  switch (dt) {
    case DT_BF16: return up ? launch_grouped_dt<DT_BF16, true>(p, st)
                            : launch_grouped_dt<DT_BF16, false>(p, st);
    case DT_F32: return up ? launch_grouped_dt<DT_F32, true>(p, st)
                           : launch_grouped_dt<DT_F32, false>(p, st);
    default: return up ? launch_grouped_dt<DT_E4M3, true>(p, st)
                       : launch_grouped_dt<DT_E4M3, false>(p, st);
  }
}

}  // namespace lookme
