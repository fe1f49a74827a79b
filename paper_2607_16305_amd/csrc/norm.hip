// What follows a layer's injections and products (arXiv 2607.16305, Eq. 2:
// sums into the hidden states): the residual sum of one or several weighted
// parts with the root-mean-square norm of the next block, its output in the
// storage type, or in e4m3 with one scale a row for products in 8 bits:
//
//   s = round(H + sum_j w_j A_j)            stored, and what is normed
//   y = s / sqrt(mean(s^2) + eps) * g
//   out = round(y);  c = max|y| / 448;  out_quant = e4m3(y / c)
//
// A team of threads holds one row in registers (each thread its 16-byte
// chunks), so H and the parts are read once and every output written once:
// HBM-bound: 23040 rows of 2048 in bf16 with one part, the sum and e4m3 out, 60 us,
// 5.5 TB/s read plus written (a large copy reaches 4.9); 8192 rows of 4096 with
// eight weighted parts 146 us, 5.3 TB/s; one row 2.7 us, a launch and two trips to
// memory.  Sums in float32.  448 is the largest e4m3 value; the scale is at
// least 2^-126 so that a row of zeros divides by it.
#include "common.h"
#include "kernels.h"

namespace lookme {

constexpr int RN_THREADS = 256;
constexpr int64_t RN_ROWS = 1 << 23;   // of a launch, which has under 2^32 threads
constexpr float E4M3_MAX = 448.f;

struct NormParams {
  const char* hidden;
  const char* add;         // [n, parts, d] or null
  const float* part_w;     // [n, parts] or null (1)
  const char* weight;      // [d] or null (1)
  char* hidden_out;        // or null
  char* out;               // or null
  char* out_quant;         // or null, with scale_out
  float* scale_out;
  int64_t n, row_bytes;
  int parts, chunks;
  float eps, inv_d;
};

template <int DT>
constexpr int rn_elems() {
  return DT == DT_BF16 ? 8 : 4;   // values of a 16-byte chunk
}

template <int DT>
__device__ __forceinline__ void rn_unpack(u32x4_t v, float (&f)[rn_elems<DT>()]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == DT_BF16) {
      f[2 * k] = bf16lo(v[k]);
      f[2 * k + 1] = bf16hi(v[k]);
    } else {
      f[k] = as_f32(v[k]);
    }
  }
}

template <int DT>
__device__ __forceinline__ u32x4_t rn_pack(const float (&f)[rn_elems<DT>()]) {
  u32x4_t v;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == DT_BF16) v[k] = pack_bf16x2(f[2 * k], f[2 * k + 1]);
    else v[k] = as_u32(f[k]);
  }
  return v;
}

// Adds the parts of chunk c of a row to its values f.  The float32 products go
// to four partial sums (part j to sum j mod 4), which are added before f is:
// four loads and four short chains at a time.  A part of weight 0 counts as
// zero, whatever its row holds (an entry that no product wrote).
template <int DT>
__device__ __forceinline__ void rn_add(const NormParams& p, const char* add, const float* pw,
                                       int c, float (&f)[rn_elems<DT>()]) {
  constexpr int E = rn_elems<DT>();
  float sum[4][E];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) sum[i][e] = 0.f;
  const char* src = add + (int64_t)c * 16;
  auto take = [&](int i, u32x4_t v, float w) {
    float a[E];
    rn_unpack<DT>(v, a);
#pragma unroll
    for (int e = 0; e < E; ++e) sum[i][e] += w != 0.f ? __fmul_rn(w, a[e]) : 0.f;
  };
  int j = 0;
  for (; j + 4 <= p.parts; j += 4) {
    u32x4_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ld16(src + (j + i) * p.row_bytes);
#pragma unroll
    for (int i = 0; i < 4; ++i) take(i, v[i], pw != nullptr ? pw[j + i] : 1.f);
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (j + i < p.parts)
      take(i, ld16(src + (j + i) * p.row_bytes), pw != nullptr ? pw[j + i] : 1.f);
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] += ((sum[0][e] + sum[1][e]) + sum[2][e]) + sum[3][e];
}

// Sum (float) and largest (uint32: the bits of non-negative floats, so that a
// NaN wins) over the T threads of a team; red: a float per wave of the block.
template <int T>
__device__ __forceinline__ float rn_sum(float v, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += red[w];
  }
  return v;
}
template <int T>
__device__ __forceinline__ uint32_t rn_max(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint32_t o = __shfl_xor(v, d, 64);
    v = o > v ? o : v;
  }
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v = red[w] > v ? red[w] : v;
  }
  return v;
}

__device__ __forceinline__ float rn_scale(uint32_t amax_bits) {
  const float c = as_f32(amax_bits) / E4M3_MAX;
  return c < 0x1p-126f ? 0x1p-126f : c;
}

template <int DT>
__device__ __forceinline__ void rn_store_quant(char* row, int c, const float (&y)[rn_elems<DT>()],
                                               float inv) {
  uint32_t q[rn_elems<DT>() / 4];
#pragma unroll
  for (int k = 0; k < rn_elems<DT>() / 4; ++k) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k] * inv, y[4 * k + 1] * inv, 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2] * inv, y[4 * k + 3] * inv, v, true);
    q[k] = (uint32_t)v;
  }
  if constexpr (DT == DT_BF16)
    *reinterpret_cast<uint2*>(row + (int64_t)c * 8) = make_uint2(q[0], q[1]);
  else
    *reinterpret_cast<uint32_t*>(row + (int64_t)c * 4) = q[0];
}

// A row on a team of T threads, at most CH chunks a thread, kept in registers.
template <int DT, int T, int CH, bool ONE>
__global__ __launch_bounds__(T > RN_THREADS ? T : RN_THREADS, CH < 8 || DT == DT_F32 ? 4 : 3)
void residual_norm_kernel(NormParams p) {
  constexpr int E = rn_elems<DT>(), BLOCK = T > RN_THREADS ? T : RN_THREADS;
  __shared__ float red_s[BLOCK / 64];
  __shared__ uint32_t red_m[BLOCK / 64];
  const int t = threadIdx.x & (T - 1);
  const int64_t row = (int64_t)blockIdx.x * (BLOCK / T) + threadIdx.x / T;
  if (row >= p.n) return;   // T < BLOCK: whole waves, and no barrier is used
  const char* h = p.hidden + row * p.row_bytes;
  const char* add = p.add + row * p.parts * p.row_bytes;
  const float* pw = p.part_w != nullptr ? p.part_w + row * p.parts : nullptr;
  float s[CH][E];
  float ss = 0.f;
  // one part: its row is loaded beside H's
  u32x4_t hv[CH], av[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = t + T * i;
    hv[i] = av[i] = u32x4_t{0, 0, 0, 0};
    if (c < p.chunks) {
      hv[i] = ld16(h + (int64_t)c * 16);
      if constexpr (ONE) av[i] = ld16(add + (int64_t)c * 16);
    }
  }
  const float w0 = ONE && pw != nullptr ? pw[0] : 1.f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = t + T * i;
    rn_unpack<DT>(hv[i], s[i]);
    if constexpr (ONE) {
      float a[E];
      rn_unpack<DT>(av[i], a);
#pragma unroll
      for (int e = 0; e < E; ++e) s[i][e] += w0 != 0.f ? __fmul_rn(w0, a[e]) : 0.f;
    } else {
      if (p.parts > 0 && c < p.chunks) rn_add<DT>(p, add, pw, c, s[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = t + T * i;
    const u32x4_t v = rn_pack<DT>(s[i]);
    if (p.hidden_out != nullptr && c < p.chunks)
      st16(p.hidden_out + row * p.row_bytes + (int64_t)c * 16, v);
    rn_unpack<DT>(v, s[i]);
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(s[i][e], s[i][e], ss);
  }
  if (p.out == nullptr && p.out_quant == nullptr) return;   // uniform over the launch
  const float r = rsqrtf(rn_sum<T>(ss, red_s) * p.inv_d + p.eps);
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = t + T * i;
    float g[E];
    if (p.weight != nullptr && c < p.chunks) {
      rn_unpack<DT>(ld16(p.weight + (int64_t)c * 16), g);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = 1.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s[i][e] = s[i][e] * r * g[e];
      const uint32_t a = as_u32(s[i][e]) & 0x7FFFFFFFu;
      if (c < p.chunks) amax = a > amax ? a : amax;   // (a NaN of r reaches the padding too)
    }
    if (p.out != nullptr && c < p.chunks)
      st16(p.out + row * p.row_bytes + (int64_t)c * 16, rn_pack<DT>(s[i]));
  }
  if (p.out_quant == nullptr) return;
  const float scale = rn_scale(rn_max<T>(amax, red_m));
  const float inv = 1.f / scale;
  char* q = p.out_quant + row * (p.row_bytes / (DT == DT_BF16 ? 2 : 4));
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = t + T * i;
    if (c < p.chunks) rn_store_quant<DT>(q, c, s[i], inv);
  }
  if (t == 0) p.scale_out[row] = scale;
}

// Rows too wide for registers: three passes over the row, each thread over its
// own chunks; with hidden_out the later passes read the stored sum back
// (hidden_out may be hidden itself), without it they sum again.
template <int DT>
__global__ __launch_bounds__(RN_THREADS) void residual_norm_wide_kernel(NormParams p) {
  constexpr int E = rn_elems<DT>();
  __shared__ float red_s[RN_THREADS / 64];
  __shared__ uint32_t red_m[RN_THREADS / 64];
  const int64_t row = blockIdx.x;
  const char* h = p.hidden + row * p.row_bytes;
  const char* add = p.add + row * p.parts * p.row_bytes;
  const float* pw = p.part_w != nullptr ? p.part_w + row * p.parts : nullptr;
  char* ho = p.hidden_out != nullptr ? p.hidden_out + row * p.row_bytes : nullptr;
  auto sum = [&](int c, float (&f)[E]) {
    rn_unpack<DT>(ld16(h + (int64_t)c * 16), f);
    rn_add<DT>(p, add, pw, c, f);
    const u32x4_t v = rn_pack<DT>(f);
    rn_unpack<DT>(v, f);
    return v;
  };
  float ss = 0.f;
  for (int c = threadIdx.x; c < p.chunks; c += RN_THREADS) {
    float f[E];
    const u32x4_t v = sum(c, f);
    if (ho != nullptr) st16(ho + (int64_t)c * 16, v);
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(f[e], f[e], ss);
  }
  if (p.out == nullptr && p.out_quant == nullptr) return;
  const float r = rsqrtf(rn_sum<RN_THREADS>(ss, red_s) * p.inv_d + p.eps);
  auto normed = [&](int c, float (&f)[E]) {
    if (ho != nullptr) rn_unpack<DT>(ld16(ho + (int64_t)c * 16), f);
    else sum(c, f);
    float g[E];
    if (p.weight != nullptr) rn_unpack<DT>(ld16(p.weight + (int64_t)c * 16), g);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = f[e] * r * (p.weight != nullptr ? g[e] : 1.f);
  };
  float inv = 0.f;
  if (p.out_quant != nullptr) {
    uint32_t amax = 0;
    for (int c = threadIdx.x; c < p.chunks; c += RN_THREADS) {
      float f[E];
      normed(c, f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t a = as_u32(f[e]) & 0x7FFFFFFFu;
        amax = a > amax ? a : amax;
      }
    }
    const float scale = rn_scale(rn_max<RN_THREADS>(amax, red_m));
    inv = 1.f / scale;
    if (threadIdx.x == 0) p.scale_out[row] = scale;
  }
  for (int c = threadIdx.x; c < p.chunks; c += RN_THREADS) {
    float f[E];
    normed(c, f);
    if (p.out != nullptr) st16(p.out + row * p.row_bytes + (int64_t)c * 16, rn_pack<DT>(f));
    if (p.out_quant != nullptr)
      rn_store_quant<DT>(p.out_quant + row * (p.row_bytes / (DT == DT_BF16 ? 2 : 4)), c, f, inv);
  }
}

template <int DT, int T, int CH>
static hipError_t launch_norm_t(const NormParams& p, hipStream_t st) {
  constexpr int BLOCK = T > RN_THREADS ? T : RN_THREADS;
  const int64_t rows = BLOCK / T;
  const dim3 grid((unsigned)((p.n + rows - 1) / rows));
  if (p.parts == 1)
    return launch_kernel(residual_norm_kernel<DT, T, CH, true>, grid, dim3(BLOCK), 0, st, p);
  return launch_kernel(residual_norm_kernel<DT, T, CH, false>, grid, dim3(BLOCK), 0, st, p);
}

// A wave a row while that is two chunks a thread, else 256 threads; 1024 while
// every row has a CU of its own, where the time is one thread's chain of loads
// (2 rows of 7360 in two parts 8.8 -> 5.1 us, 256 rows of 4096 in eight
// 9.6 -> 7.2; 512 such rows 12.0 -> 13.7).
template <int DT>
static hipError_t launch_norm(const NormParams& p, hipStream_t st) {
  const bool few = p.n <= 256;
  if (p.chunks <= 64) return launch_norm_t<DT, 64, 1>(p, st);
  if (p.chunks <= 128) return launch_norm_t<DT, 64, 2>(p, st);
  if (p.chunks <= 256) return launch_norm_t<DT, 256, 1>(p, st);
  if (p.chunks <= 1024 && few) return launch_norm_t<DT, 1024, 1>(p, st);
  if (p.chunks <= 2048 && few) return launch_norm_t<DT, 1024, 2>(p, st);
  if (p.chunks <= 512) return launch_norm_t<DT, 256, 2>(p, st);
  if (p.chunks <= 1024) return launch_norm_t<DT, 256, 4>(p, st);
  if (p.chunks <= 2048) return launch_norm_t<DT, 256, 8>(p, st);
  return launch_kernel(residual_norm_wide_kernel<DT>, dim3((unsigned)p.n), dim3(RN_THREADS), 0, st,
                       p);
}

hipError_t launch_residual_norm(int dt, int64_t n, int d, const void* hidden, int parts,
                                const void* add, const float* part_w, const void* weight,
                                float eps, void* hidden_out, void* out, void* out_quant,
                                float* scale_out, hipStream_t st) {
  if (n == 0) return hipSuccess;
  NormParams p{};
  p.hidden = static_cast<const char*>(hidden);
  p.add = static_cast<const char*>(add);
  p.part_w = part_w;
  p.weight = static_cast<const char*>(weight);
  p.hidden_out = static_cast<char*>(hidden_out);
  p.out = static_cast<char*>(out);
  p.out_quant = static_cast<char*>(out_quant);
  p.scale_out = scale_out;
  p.row_bytes = (int64_t)d * (dt == DT_BF16 ? 2 : 4);
  p.parts = parts;
  p.chunks = (int)(p.row_bytes / 16);
  p.eps = eps;
  p.inv_d = 1.f / (float)d;
  for (int64_t row = 0; row < n; row += RN_ROWS) {
    p.n = n - row < RN_ROWS ? n - row : RN_ROWS;
    const hipError_t e = dt == DT_BF16 ? launch_norm<DT_BF16>(p, st) : launch_norm<DT_F32>(p, st);
    if (e != hipSuccess) return e;
    const int64_t bytes = RN_ROWS * p.row_bytes;
    p.hidden += bytes;
    if (p.add != nullptr) p.add += bytes * parts;
    if (p.part_w != nullptr) p.part_w += RN_ROWS * parts;
    if (p.hidden_out != nullptr) p.hidden_out += bytes;
    if (p.out != nullptr) p.out += bytes;
    if (p.out_quant != nullptr) {
      p.out_quant += RN_ROWS * d;
      p.scale_out += RN_ROWS;
    }
  }
  return hipSuccess;
}

}  // namespace lookme
