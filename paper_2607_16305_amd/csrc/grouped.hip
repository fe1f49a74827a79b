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
//   grouped_tiles_kernel  many rows a group: 256 x 256 tiles (a group's last
//       rows, where at most 128: 128 x 256) on the phased loop of
//       phase_gemm.h, one workgroup a CU that takes tile after tile.
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
constexpr int GT_THREADS = 512;

// One tile: the group's rows from m0, output columns from n0.
template <int DT, int MI, int NJ, bool UP>
__device__ __forceinline__ void grouped_tile(const GroupedParams& p, char* lds, const GpTile& t,
                                             int64_t m0, int n0) {
  using S = PgShape<MI, NJ>;
  constexpr int ODT = DT == DT_E4M3 ? DT_BF16 : DT;
  constexpr int OES = ODT == DT_BF16 ? 2 : 4;
  PgLoop<DT, MI, NJ> L(lds, threadIdx.x);
  PgLoads<S> ld;
  const int nst = (int)(p.k_bytes / 128);
  ld.last = nst - 1;
  // gathered rows count from the operand's first row, others from the tile's
  const bool gather = p.picks != 0;
  ld.a_base = p.x + (gather ? 0 : (t.a + m0) * p.k_bytes);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int q = 0; q < S::PA; ++q) {
      int64_t i = t.a + m0 + h * S::HM + L.a_row(q), src, dst;
      i = i < t.b ? i : t.b - 1;
      gp_entry(p, i, src, dst);
      if (!gather) src = i - (t.a + m0);
      ld.oa[h][q] = (uint32_t)(src * p.k_bytes) + L.a_chunk(q) * 16;
    }
    const int nh = n0 + (UP ? 0 : h * S::HN);   // first weight row of the half
    const int first = nh < p.cols ? nh : p.cols - 1;
    ld.b_base[h] = (UP && h == 1 ? p.w_up : p.w) + ((int64_t)t.g * p.cols + first) * p.k_bytes;
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

  constexpr int W = S::W, QJ = UP ? 1 : 2, PC = 16 / OES, NP = W * OES / 16;   // 16-byte pieces
  static_assert(W * OES % 16 == 0, "whole pieces");
#pragma unroll
  for (int qi = 0; qi < 2; ++qi)
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t e = t.a + m0 + qi * S::HM + L.wr * 16 * MI + 16 * i + L.n16;
      int64_t src, dst;
      if (e >= t.b || !gp_entry(p, e, src, dst)) continue;
      const float xs = DT == DT_E4M3 ? p.x_scale[src] : 1.f;
#pragma unroll
      for (int qj = 0; qj < QJ; ++qj)
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          const int col = n0 + qj * S::HN + L.wc * 16 * NJ + W * L.g + PC * k;
          if (col >= p.cols) continue;   // cols is a multiple of a piece
          float v[PC];
#pragma unroll
          for (int r = 0; r < PC; ++r) {
            const int x = PC * k + r;
            float ws = 1.f, us = 1.f;
            if constexpr (DT == DT_E4M3) {
              ws = p.w_scale[(int64_t)t.g * p.cols + col + r];
              if constexpr (UP) us = p.up_scale[(int64_t)t.g * p.cols + col + r];
            }
            v[r] = gp_value<DT, UP>(acc[qi][qj][i][x >> 2][x & 3], acc[qi][1][i][x >> 2][x & 3],
                                    xs, ws, us);
          }
          st_cols<ODT, PC>(p.out + (dst * p.cols + col) * OES, v);
        }
    }
}

template <int DT, bool UP>
__global__ __launch_bounds__(GT_THREADS, 2) void grouped_tiles_kernel(GroupedParams p) {
  using S = PgShape<4, 2>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * S::BUF];
  __shared__ int find_lds[GP_FIND_LDS];
  constexpr int TCOLS = UP ? S::HN : S::BN;
  const int tn = (p.cols + TCOLS - 1) / TCOLS;
  // whole row blocks of a group (a last one of more than 128 rows counts), and
  // its half row block
  auto whole = [](int64_t r) { return (int)((r + 127) / 256); };
  auto half = [](int64_t r) {
    const int rem = (int)(r % 256);
    return rem > 0 && rem <= 128 ? 1 : 0;
  };
  GpTile t;
  int64_t wholes = INT64_MAX;
  // a workgroup of the launch's rounds: neighbouring tiles on one XCD
  const int slot = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  for (int64_t unit = slot;; unit += gridDim.x) {
    if (unit < wholes) {
      const int rb = (int)(unit / tn);
      wholes = (int64_t)find_tile<GT_THREADS>(p, rb, find_lds, t, whole) * tn;
      if (t.g >= 0) {
        grouped_tile<DT, 4, 2, UP>(p, lds, t, (int64_t)t.idx * S::BM,
                                   (int)(unit - (int64_t)rb * tn) * TCOLS);
        continue;
      }
    }
    const int rb = (int)((unit - wholes) / tn);
    find_tile<GT_THREADS>(p, rb, find_lds, t, half);
    if (t.g < 0) return;
    grouped_tile<DT, 2, 2, UP>(p, lds, t, (t.b - t.a) / 256 * 256,
                               (int)(unit - wholes - (int64_t)rb * tn) * TCOLS);
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
    hipLaunchKernelGGL((grouped_tiles_kernel<DT, UP>), dim3(256), dim3(GT_THREADS), 0, st, p);
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
