// Products of few rows with weights of 4 bits and scales (and zero points) by
// groups along K, the form in which the fusion of Eq. 10 serves single tokens:
//
//   out = round(add + sum_G s_G sum_{k in G} (q_k - z_G) x_k), or
//   out = round(silu(gate) * up) of two such sums.
//
// Bound by the weights' stream out of HBM.  A wave takes 16 weight rows and
// 16 NT tokens on the matrix cores.  A lane's 16 bytes are 32 weights of a row;
// two nibbles at a time become two bf16 values 16 + q in two instructions
// (0x4180 + 8 q: exact), so that
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x,
// with sum x from a product with ones.  Every product is exact in float32 and
// the group's scale multiplies its float32 sum: no weight is rounded.  float32
// tokens are three bf16 values (8 + 8 + 8 bits of the significand), three
// products a step.
// The scales and zero points of a workgroup's rows wait in LDS as float32.
#include "common.h"
#include "kernels.h"
#include "tile_gemm.h"

namespace lookme {

constexpr int QP_WAVES = 4, QP_THREADS = 64 * QP_WAVES;
constexpr int QP_GROUPS = 256;   // groups whose scales are in LDS at a time

// 8 nibbles as the bf16 values 16 + q of nibbles (0, 4), (1, 5), (2, 6), (3, 7)
__device__ __forceinline__ u32x4_t qp_expand(uint32_t u) {
  constexpr uint32_t M = 0x00780078u, B = 0x41804180u;
  return u32x4_t{((u << 3) & M) | B, ((u >> 1) & M) | B, ((u >> 5) & M) | B, ((u >> 9) & M) | B};
}

// eight bf16 values in the order of qp_expand
__device__ __forceinline__ u32x4_t qp_order(u32x4_t x) {
  return u32x4_t{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u),
                 __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                 __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                 __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

// regs r of lane group g hold words 4 g + r of a row's 64 bytes; afterwards
// words 4 r + g
__device__ __forceinline__ void qp_transpose(u32x4_t& v) {
  typedef unsigned u32x2_v __attribute__((ext_vector_type(2)));
  const auto a = __builtin_amdgcn_permlane16_swap(v[0], v[1], false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(v[2], v[3], false, false);
  const auto c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
  const auto d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
  v = u32x4_t{c[0], d[0], c[1], d[1]};
}

// Eight tokens' values of a lane as bf16 parts whose sum they are: one part,
// or for float32 three (truncated, so that none overflows; the later parts of
// a value that is not finite are zero).
template <int DT>
struct QpFrag {
  static constexpr int PARTS = DT == DT_BF16 ? 1 : 3;
  u32x4_t raw[DT == DT_BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* row, int c) {   // chunk of 8 values
    if constexpr (DT == DT_BF16) {
      raw[0] = ld16(row + (int64_t)c * 16);
    } else {
      raw[0] = ld16(row + (int64_t)c * 32);
      raw[1] = ld16(row + (int64_t)c * 32 + 16);
    }
  }
  __device__ __forceinline__ void split(bool in, u32x4_t (&f)[PARTS]) const {
    const u32x4_t none = {0, 0, 0, 0};
    if constexpr (DT == DT_BF16) {
      f[0] = in ? qp_order(raw[0]) : none;
    } else {
      uint32_t h[3][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = in ? raw[e >> 2][e & 3] : 0u;
        const uint32_t hi = u & 0xFFFF0000u;
        const bool finite = (u & 0x7F800000u) != 0x7F800000u;
        const float r1 = finite ? as_f32(u) - as_f32(hi) : 0.f;
        const uint32_t mid = as_u32(r1) & 0xFFFF0000u;
        const float r2 = r1 - as_f32(mid);
        // a NaN whose payload is in the low half keeps a high one
        h[0][e] = finite || (u & 0x007FFFFFu) == 0 ? hi : hi | 0x00400000u;
        h[1][e] = mid;
        h[2][e] = as_u32(r2);
      }
      // pairs (0, 4), (1, 5), (2, 6), (3, 7): upper halves
#pragma unroll
      for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          f[q][e] = __builtin_amdgcn_perm(h[q][e + 4], h[q][e], 0x07060302u);
    }
  }
};

// NT: token tiles of 16.  D: blocks of 128 weights a row in flight.  SHORT:
// groups of 32 or 64 (the words of a block are transposed so that a product
// step stays inside one), else of whole blocks.  K is split over the
// workgroup's waves.
template <int DT, int NT, int D, bool UP, bool SHORT>
__global__ __launch_bounds__(QP_THREADS) void quant_rows_kernel(QuantParams p) {
  constexpr int ES = DT == DT_BF16 ? 2 : 4;
  constexpr int MATS = UP ? 2 : 1;
  constexpr int PARTS = QpFrag<DT>::PARTS;
  __shared__ __attribute__((aligned(16))) float sz[MATS][QP_GROUPS][2][16];
  __shared__ f32x4_t part[QP_WAVES * MATS * NT * 64];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int c0 = blockIdx.x * 16;
  const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);
  const int64_t k_bytes = (int64_t)p.k * ES;
  const int groups = p.k / p.group;

  const char* xp[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t t = t0 + 16 * j + n16;
    xp[j] = p.x + (t < p.n ? t : p.n - 1) * k_bytes;
  }
  const int wc = c0 + n16 < p.cols ? c0 + n16 : p.cols - 1;
  const char* wp[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) wp[q] = p.m[q].w + (int64_t)wc * (p.k / 2);

  f32x4_t acc[MATS][NT];
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const int wchunks = p.k / 32, xchunks = p.k / 8;
  u32x4_t fw[D][MATS];
  QpFrag<DT> fx[D][NT][4];
  auto load = [&](int d, int b) {
    int c = 4 * b + g;
    c = c < wchunks ? c : wchunks - 1;
#pragma unroll
    for (int q = 0; q < MATS; ++q) fw[d][q] = ld16_nt(wp[q] + (int64_t)c * 16);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        int x = SHORT ? 16 * b + 4 * s + g : 16 * b + 4 * g + s;
        x = x < xchunks ? x : xchunks - 1;
        fx[d][j][s].load(xp[j], x);
      }
  };

  // blocks whose groups' scales fit LDS; one pass for all but long K of short groups
  const int seg_blocks = p.group >= 128 ? QP_GROUPS * (p.group / 128) : QP_GROUPS * p.group / 128;
  const int blocks = (p.k + 127) / 128;
  for (int seg = 0; seg < blocks; seg += seg_blocks) {
    const int left = blocks - seg < seg_blocks ? blocks - seg : seg_blocks;
    const int per = (left + QP_WAVES - 1) / QP_WAVES;
    const int b0 = seg + wv * per;
    const int b1 = b0 + per < seg + left ? b0 + per : seg + left;
    if (b0 < b1) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        load(d, b0 + d);
        asm volatile("" ::: "memory");
      }
    }
    const int first = (int)((int64_t)seg * 128 / p.group);
    const int count = groups - first < QP_GROUPS ? groups - first : QP_GROUPS;
    if (seg != 0) __syncthreads();
    for (int i = threadIdx.x; i < 16 * count; i += QP_THREADS) {
      const int r = i / count, k = i - r * count;
      const int row = c0 + r < p.cols ? c0 + r : p.cols - 1;
      const int64_t at = (int64_t)row * groups + first + k;
#pragma unroll
      for (int q = 0; q < MATS; ++q) {
        if constexpr (DT == DT_BF16)
          sz[q][k][0][r] = bf16lo(reinterpret_cast<const uint16_t*>(p.m[q].scale)[at]);
        else
          sz[q][k][0][r] = reinterpret_cast<const float*>(p.m[q].scale)[at];
        sz[q][k][1][r] = 16.f + (p.m[q].zero != nullptr ? (float)p.m[q].zero[at] : 8.f);
      }
    }
    __syncthreads();
    for (int b = b0; b < b1; b += D) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        if (b + d < b1) {   // the same for the whole wave
          u32x4_t w[MATS];
#pragma unroll
          for (int q = 0; q < MATS; ++q) {
            w[q] = fw[d][q];
            if constexpr (SHORT) qp_transpose(w[q]);
          }
          f32x4_t sp[MATS][NT], sx[NT];
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            sx[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < MATS; ++q) sp[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          }
          auto flush = [&](int grp) {   // the group's sums, scaled, into acc
#pragma unroll
            for (int q = 0; q < MATS; ++q) {
              const f32x4_t s = *reinterpret_cast<const f32x4_t*>(&sz[q][grp - first][0][4 * g]);
              const f32x4_t z = *reinterpret_cast<const f32x4_t*>(&sz[q][grp - first][1][4 * g]);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  acc[q][j][r] = fmaf(s[r], fmaf(-z[r], sx[j][r], sp[q][j][r]), acc[q][j][r]);
                sp[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
              }
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) sx[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          };
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int x = SHORT ? 16 * (b + d) + 4 * s + g : 16 * (b + d) + 4 * g + s;
            const u32x4_t ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
            u32x4_t a[MATS];
#pragma unroll
            for (int q = 0; q < MATS; ++q) a[q] = qp_expand(w[q][s]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              u32x4_t f[PARTS];
              fx[d][j][s].split(x < xchunks, f);
#pragma unroll
              for (int e = 0; e < PARTS; ++e) {
                sx[j] = mfma_chunk<DT_BF16>(ones, f[e], sx[j]);
#pragma unroll
                for (int q = 0; q < MATS; ++q) sp[q][j] = mfma_chunk<DT_BF16>(a[q], f[e], sp[q][j]);
              }
            }
            if constexpr (SHORT) {
              // (K may end inside the last block)
              const int k = 128 * (b + d) + 32 * s;
              if (k < p.k && (p.group == 32 || (s & 1) != 0)) flush(k / p.group);
            }
          }
          if constexpr (!SHORT) flush(128 * (b + d) / p.group);
        }
        load(d, b + d + D);
      }
    }
  }

  f32x4_t* mine = part + wv * (MATS * NT * 64) + lane;
  if (wv != 0) {
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
      for (int j = 0; j < NT; ++j) mine[(q * NT + j) * 64] = acc[q][j];
  }
  __syncthreads();
  if (wv != 0) return;
#pragma unroll
  for (int o = 1; o < QP_WAVES; ++o)
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const f32x4_t v = mine[(o * MATS * NT + q * NT + j) * 64];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[q][j][r] += v[r];
      }
  const int col = c0 + 4 * g;
  if (col >= p.cols) return;   // cols is a multiple of 4
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t t = t0 + 16 * j + n16;
    if (t >= p.n) continue;
    const int64_t at = (t * p.cols + col) * ES;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = UP ? silu_f(acc[0][j][r]) * acc[MATS - 1][j][r] : acc[0][j][r];
    if (p.add != nullptr) {
      float a[4];
      ld_cols<DT, 4>(p.add + at, a);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] += a[r];
    }
    st_cols<DT, 4>(p.out + at, v);
  }
}

template <int DT, int NT, int D, bool UP>
static void launch_quant_nt(const QuantParams& p, hipStream_t st) {
  const dim3 grid((unsigned)((p.cols + 15) / 16), (unsigned)((p.n + 16 * NT - 1) / (16 * NT)));
  if (p.group < 128)
    hipLaunchKernelGGL((quant_rows_kernel<DT, NT, D, UP, true>), grid, dim3(QP_THREADS), 0, st, p);
  else
    hipLaunchKernelGGL((quant_rows_kernel<DT, NT, D, UP, false>), grid, dim3(QP_THREADS), 0, st, p);
}

template <int DT, bool UP>
static void launch_quant_dt(const QuantParams& p, hipStream_t st) {
  if (p.n <= 16) launch_quant_nt<DT, 1, 2, UP>(p, st);
  else launch_quant_nt<DT, 2, 1, UP>(p, st);
}

hipError_t launch_quant(int dt, const QuantParams& p, hipStream_t st) {
  if (p.n == 0) return hipSuccess;
  if (dt == DT_BF16) {
    if (p.up) launch_quant_dt<DT_BF16, true>(p, st);
    else launch_quant_dt<DT_BF16, false>(p, st);
  } else {
    if (p.up) launch_quant_dt<DT_F32, true>(p, st);
    else launch_quant_dt<DT_F32, false>(p, st);
  }
  return hipGetLastError();
}

}  // namespace lookme
