// Products of few rows, of decoded tokens, with weights of 4 bits and scales (and
// zero points) by groups along K: a projection with its residual sum, or the gate
// and up half of a SwiGLU layer (the form of Eq. 10; the handle's own fusion takes
// bf16 and float32 weights):
//
//   out = round(add + sum_G s_G sum_{k in G} (q_k - z_G) x_k), or
//   out = round(silu(gate) * up) of two such sums.
//
// Bound by the weights' stream out of HBM.  A wave takes 16 weight rows and
// 16 NT tokens on the matrix cores.  A lane's 16 bytes are 32 weights of a row;
// a nibble in a byte of its own is the e4m3 value q / 512, which a conversion
// turns into the float32 q for two of them at a time; q - z, at most 8 bits of
// significand, is exact in bf16.  So every product is exact in float32, the sums
// are float32 sums of these products and nothing else, and the group's scale
// multiplies its sum: no weight is rounded.  (Two instructions for two nibbles
// give 16 + q, with (16 + z) sum x taken off afterwards: no faster, 8192 x 8192 of 1,
// 16 and 64 rows 15.1, 18.5 and 45.1 us against 15.3, 18.5 and 45.3, and its sums
// lose what the result is when sum x is large beside it: relative errors of
// 4e-5 instead of 1e-7 for tokens of mean 5, of 4e-2 where only one token value of
// 12345 stands before a weight of zero.)
// float32 tokens are three bf16 values (8 + 8 + 8 bits of the significand), three
// products a step.
// The scales and zero points of a workgroup's rows wait in LDS as float32.  What a
// call takes beyond its launch is the weights at 5 TB/s, or the instructions (120 a
// wave for 128 x 16 weights, 102 with two row tiles), whichever is longer, and two
// latencies of HBM, while its workgroups are all resident: one to three a CU, by
// their registers.  More of them (there are cols / 16 x n / 16, half as many for
// every second tile a wave has) take their turns.
#include "common.h"
#include "kernels.h"
#include "tile_gemm.h"

namespace lookme {

constexpr int QP_WAVES = 8, QP_THREADS = 64 * QP_WAVES;
constexpr int QP_GROUPS = 128;   // groups whose scales are in LDS at a time

// 8 nibbles less a zero point as bf16, in their order
__device__ __forceinline__ u32x4_t qp_expand(uint32_t u, float z) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const uint32_t even = u & 0x0F0F0F0Fu, odd = (u >> 4) & 0x0F0F0F0Fu;
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 512.f, false);
  const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 512.f, false);
  const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(even, 512.f, true);
  const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(odd, 512.f, true);
  auto pair = [z](float lo, float hi) {   // (the lower halves are zero)
    return __builtin_amdgcn_perm(as_u32(hi - z), as_u32(lo - z), 0x07060302u);
  };
  return u32x4_t{pair(a[0], b[0]), pair(a[1], b[1]), pair(c[0], d[0]), pair(c[1], d[1])};
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

// Eight values of a token as bf16 parts whose sum they are: one part, or for
// float32 three (truncated, so that none overflows; of a value that is not
// finite the later parts are NaN).
template <int DT>
struct QpFrag {
  static constexpr int PARTS = DT == DT_BF16 ? 1 : 3;
  u32x4_t raw[DT == DT_BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p) {
    raw[0] = ld16(p);
    if constexpr (DT == DT_F32) raw[1] = ld16(p + 16);
  }
  __device__ __forceinline__ void split(u32x4_t (&f)[PARTS]) const {
    if constexpr (DT == DT_BF16) {
      f[0] = raw[0];
    } else {
      uint32_t h[3][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = raw[e >> 2][e & 3];
        h[0][e] = u & 0xFFFF0000u;
        const float r1 = as_f32(u) - as_f32(h[0][e]);
        h[1][e] = as_u32(r1) & 0xFFFF0000u;
        h[2][e] = as_u32(r1 - as_f32(h[1][e]));
      }
#pragma unroll
      for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          f[q][e] = __builtin_amdgcn_perm(h[q][2 * e + 1], h[q][2 * e], 0x07060302u);
    }
  }
};

// NT: token tiles of 16.  RW: tiles of 16 weight rows a wave multiplies with the
// same tokens (of each matrix).  SHORT: groups of 32 or 64 (the words of a block
// are transposed so that a product step stays inside one), else of whole
// blocks.  K is split over the workgroup's waves, two blocks of 128 weights in
// flight in each.  lds: the scales of at most QP_GROUPS groups, then the waves'
// sums.
template <int DT, int NT, int RW, bool UP, bool SHORT>
__global__ __launch_bounds__(QP_THREADS) void quant_rows_kernel(QuantParams p) {
  constexpr int ES = DT == DT_BF16 ? 2 : 4;
  constexpr int MATS = UP ? 2 : 1, TILES = MATS * RW;   // tile q RW + i: rows 16 i of matrix q
  constexpr int PARTS = QpFrag<DT>::PARTS;
  static_assert(RW * NT <= QP_WAVES, "a wave an output tile");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  // [group][tile][scale, zero][16 rows]
  float (*sz)[TILES][2][16] = reinterpret_cast<float (*)[TILES][2][16]>(lds);
  f32x4_t* part = reinterpret_cast<f32x4_t*>(lds);
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int c0 = blockIdx.x * (16 * RW);
  const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);
  const int64_t k_bytes = (int64_t)p.k * ES;
  const int groups = p.k / p.group;

  const char* xp[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t t = t0 + 16 * j + n16;
    xp[j] = p.x + (t < p.n ? t : p.n - 1) * k_bytes;
  }
  const char* wp[TILES];
#pragma unroll
  for (int q = 0; q < TILES; ++q) {
    const int c = c0 + 16 * (q % RW) + n16;
    wp[q] = p.m[q / RW].w + (int64_t)(c < p.cols ? c : p.cols - 1) * (p.k / 2);
  }

  f32x4_t acc[TILES][NT];
#pragma unroll
  for (int q = 0; q < TILES; ++q)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // K may end inside the last block of SHORT groups: its chunks past the end are
  // read from clamped addresses, and their sums, whole steps, never used
  constexpr int XB = 8 * ES;   // bytes of 8 values
  const int wchunks = p.k / 32, xchunks = p.k / 8;
  u32x4_t fw[2][TILES];
  QpFrag<DT> fx[2][NT][4];
  auto load_w = [&](int d, int b) {
    int c = 4 * b + g;
    if constexpr (SHORT) c = c < wchunks ? c : wchunks - 1;
#pragma unroll
    for (int q = 0; q < TILES; ++q) fw[d][q] = ld16(wp[q] + c * 16);
  };
  auto load_x = [&](int d, int b) {
    if (!SHORT || 128 * (b + 1) <= p.k) {
      const int off = (16 * b + (SHORT ? g : 4 * g)) * XB;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) fx[d][j][s].load(xp[j] + off + (SHORT ? 4 * s : s) * XB);
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int x = 16 * b + 4 * s + g;
          fx[d][j][s].load(xp[j] + (x < xchunks ? x : xchunks - 1) * XB);
        }
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
      for (int d = 0; d < 2; ++d) {
        if (b0 + d < b1) {
          load_x(d, b0 + d);
          load_w(d, b0 + d);
        }
        asm volatile("" ::: "memory");
      }
    }
    const int first = (int)((int64_t)seg * 128 / p.group);
    const int count = groups - first < QP_GROUPS ? groups - first : QP_GROUPS;
    if (seg != 0) __syncthreads();
    // 16 threads a row
    for (int r = threadIdx.x >> 4; r < 16 * TILES; r += QP_THREADS / 16) {
      const int q = r >> 4;
      int row = c0 + 16 * (q % RW) + (r & 15);
      row = row < p.cols ? row : p.cols - 1;
      const QuantMatrix& m = p.m[q / RW];
      const int64_t at = (int64_t)row * groups + first;
      for (int k = threadIdx.x & 15; k < count; k += 16) {
        if constexpr (DT == DT_BF16)
          sz[k][q][0][r & 15] = bf16lo(reinterpret_cast<const uint16_t*>(m.scale)[at + k]);
        else
          sz[k][q][0][r & 15] = reinterpret_cast<const float*>(m.scale)[at + k];
        sz[k][q][1][r & 15] = m.zero != nullptr ? (float)m.zero[at + k] : 8.f;
      }
    }
    __syncthreads();
    for (int b = b0; b < b1; b += 2) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        if (b + d < b1) {   // the same for the whole wave
          u32x4_t w[TILES];
#pragma unroll
          for (int q = 0; q < TILES; ++q) {
            w[q] = fw[d][q];
            if constexpr (SHORT) qp_transpose(w[q]);
          }
          const int block = b + d;
          // a block's group, among those in LDS; of SHORT ones that of step s (of the
          // steps past K the last one)
          const int whole = SHORT ? 0 : 128 * block / p.group - first;
          auto of = [&](int s) {
            const int grp = (4 * block + s) >> (p.group == 32 ? 0 : 1);
            return (grp < groups ? grp : groups - 1) - first;
          };
          float z[TILES];
          auto zeros = [&](int grp) {
#pragma unroll
            for (int q = 0; q < TILES; ++q) z[q] = sz[grp][q][1][n16];
          };
          f32x4_t sp[TILES][NT];
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < TILES; ++q) sp[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          auto flush = [&](int grp) {   // the group's sums, scaled, into acc
#pragma unroll
            for (int q = 0; q < TILES; ++q) {
              const f32x4_t s = *reinterpret_cast<const f32x4_t*>(&sz[grp][q][0][4 * g]);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[q][j][r] = fmaf(s[r], sp[q][j][r], acc[q][j][r]);
                sp[q][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
              }
            }
          };
          if constexpr (!SHORT) zeros(whole);
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            if constexpr (SHORT)
              if (p.group == 32 || (s & 1) == 0) zeros(of(s));
            u32x4_t a[TILES];
#pragma unroll
            for (int q = 0; q < TILES; ++q) a[q] = qp_expand(w[q][s], z[q]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              u32x4_t f[PARTS];
              fx[d & 1][j][s].split(f);
#pragma unroll
              for (int e = 0; e < PARTS; ++e)
#pragma unroll
                for (int q = 0; q < TILES; ++q)
                  sp[q][j] = mfma_chunk<DT_BF16>(a[q], f[e], sp[q][j]);
            }
            if constexpr (SHORT) {
              // (K may end inside the last block)
              if (128 * block + 32 * s < p.k && (p.group == 32 || (s & 1) != 0)) flush(of(s));
            }
          }
          if constexpr (!SHORT) flush(whole);
        }
        if (b + d + 2 < b1) {
          load_x(d, b + d + 2);
          load_w(d, b + d + 2);
        }
      }
    }
  }

  __syncthreads();   // the scales give way to the sums: [wave][tile][token tile][lane]
  f32x4_t* mine = part + wv * (TILES * NT * 64) + lane;
#pragma unroll
  for (int q = 0; q < TILES; ++q)
#pragma unroll
    for (int j = 0; j < NT; ++j) mine[(q * NT + j) * 64] = acc[q][j];
  __syncthreads();
  if (wv >= RW * NT) return;   // a wave an output tile
  const int i = wv / NT, j = wv % NT;
  f32x4_t sum[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) {
    sum[q] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < QP_WAVES; ++w) {
      const f32x4_t v = part[((w * TILES + q * RW + i) * NT + j) * 64 + lane];
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[q][r] += v[r];
    }
    // an infinity becomes a NaN, as the parts of a float32 one are
#pragma unroll
    for (int r = 0; r < 4; ++r) sum[q][r] = fmaf(sum[q][r], 0.f, sum[q][r]);
  }
  const int col = c0 + 16 * i + 4 * g;
  const int64_t t = t0 + 16 * j + n16;
  if (col >= p.cols || t >= p.n) return;   // cols is a multiple of 4
  const int64_t at = (t * p.cols + col) * ES;
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = UP ? silu_f(sum[0][r]) * sum[MATS - 1][r] : sum[0][r];
  if (p.add != nullptr) {
    float a[4];
    ld_cols<DT, 4>(p.add + at, a);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] += a[r];
  }
  st_cols<DT, 4>(p.out + at, v);
}

template <int DT, int NT, int RW, bool UP>
static hipError_t launch_quant_nt(const QuantParams& p, hipStream_t st) {
  constexpr int TILES = (UP ? 2 : 1) * RW;
  const dim3 grid((unsigned)((p.cols + 16 * RW - 1) / (16 * RW)),
                  (unsigned)((p.n + 16 * NT - 1) / (16 * NT)));
  const int groups = p.k / p.group < QP_GROUPS ? p.k / p.group : QP_GROUPS;
  const size_t scales = (size_t)groups * TILES * 2 * 16 * 4;
  const size_t sums = (size_t)QP_WAVES * TILES * NT * 64 * 16;
  static_assert(QP_GROUPS * TILES * 128 <= 65536 && QP_WAVES * TILES * NT * 1024 <= 65536,
                "dynamic LDS of a launch");
  const size_t lds = scales > sums ? scales : sums;
  if (p.group < 128)
    return launch_kernel(quant_rows_kernel<DT, NT, RW, UP, true>, grid, dim3(QP_THREADS), lds, st,
                         p);
  return launch_kernel(quant_rows_kernel<DT, NT, RW, UP, false>, grid, dim3(QP_THREADS), lds, st, p);
}

// Two row tiles a wave where these are a workgroup for every CU: the tokens,
// which every wave reads from L2 for itself, then serve twice the weights (8192 x
// 8192 of bf16 out of HBM, one tile and two: 1 row 15.0 and 14.6 us, 16 rows 23.9
// and 18.3, 32 rows 36.5 and 25.1; float32 1 row 28.2 and 20.1; 4096 x 4096, 128
// workgroups, 16 rows 8.6 and 10.1).  Gate and up share the tokens already, which
// is enough for few rows (2 x 8192 x 4096 of 4 rows 14.2 and 16.9, of 16 17.4 and
// 17.6, of 32 27.2 and 21.3; float32 of 4 rows 24.5 and 21.3), and with two token
// tiles of float32 two row tiles spill.  Deeper rings (4 blocks: 1 row of 8192 x 8192 14.0 us), 16 waves (1
// row of 1024 x 8192 7.5 and 7.4 us) and no loads for the tokens there are none
// of (the same) were no faster.
template <int DT, bool UP>
static hipError_t launch_quant_dt(const QuantParams& p, hipStream_t st) {
  const int64_t wide = (int64_t)((p.cols + 31) / 32) * ((p.n + 31) / 32);
  const bool two = wide >= 256 && !(UP && (DT == DT_BF16 ? p.n <= 8 : p.n > 16));
  if (p.n <= 16) {
    return two ? launch_quant_nt<DT, 1, 2, UP>(p, st) : launch_quant_nt<DT, 1, 1, UP>(p, st);
  }
  if constexpr (!(UP && DT == DT_F32))
    if (two) return launch_quant_nt<DT, 2, 2, UP>(p, st);
  return launch_quant_nt<DT, 2, 1, UP>(p, st);
}

hipError_t launch_quant(int dt, const QuantParams& p, hipStream_t st) {
  if (p.n == 0) return hipSuccess;
  if (dt == DT_BF16)
    return p.up ? launch_quant_dt<DT_BF16, true>(p, st) : launch_quant_dt<DT_BF16, false>(p, st);
  return p.up ? launch_quant_dt<DT_F32, true>(p, st) : launch_quant_dt<DT_F32, false>(p, st);
}

}  // namespace lookme
