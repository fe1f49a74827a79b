// Queries and keys before attention: the root-mean-square norm of each head with
// the rotation of its positions, in one pass over q and k:
//
//   y = x / sqrt(mean(x^2) + eps) * g           (or y = x)
//   a_i = pos[axis_i] freq_i,  c_i = factor cos a_i,  s_i = factor sin a_i
//   (y_i, y_i') -> (y_i c_i - y_i' s_i, y_i s_i + y_i' c_i)
//
// with i' = i + rot / 2, or for neighbouring pairs 2 i and 2 i + 1; the rest of a
// head keeps y.  Float32 sums and products, one rounding into the output.
//
// The angle is reduced in float64, in turns: pos freq / (2 pi) less the nearest
// whole number, good to 2^-53 of the turns, so a position of 10^6 has the angle
// that a float32 product would miss by 0.03.  What is left is float32 (2^-26 of
// a turn).  A token's angles are computed once for all of its heads.
#include "common.h"
#include "kernels.h"

namespace lookme {

constexpr int HR_THREADS = 256;
constexpr int HR_ANGLES = 256;         // of a workgroup: of one token or of several
constexpr int64_t HR_TOKENS = 1 << 22; // of a launch, which has under 2^32 threads

template <int DT>
constexpr int hr_elems() {
  return DT == DT_BF16 ? 8 : 4;   // values of a 16-byte chunk
}

template <int DT>
__device__ __forceinline__ void hr_unpack(u32x4_t v, float (&f)[hr_elems<DT>()]) {
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
__device__ __forceinline__ u32x4_t hr_pack(const float (&f)[hr_elems<DT>()]) {
  u32x4_t v;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == DT_BF16) v[k] = pack_bf16x2(f[2 * k], f[2 * k + 1]);
    else v[k] = as_u32(f[k]);
  }
  return v;
}

// A head on a team of T lanes, a 16-byte chunk each; a workgroup takes `tokens`
// tokens and all of their heads, or `span` heads of one token.
template <int DT, int T>
__global__ __launch_bounds__(HR_THREADS) void head_norm_rotary_kernel(RotaryParams p) {
  constexpr int E = hr_elems<DT>();
  __shared__ float cs[HR_ANGLES], sn[HR_ANGLES];
  __shared__ float ys[HR_THREADS * E];
  const int half = p.rot / 2;
  const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
  const int tokens = (int)(p.n - t0 < p.tokens ? p.n - t0 : p.tokens);
  for (int i = threadIdx.x; i < tokens * half; i += HR_THREADS) {
    const int t = i / half, k = i - t * half;
    int ax = 0;
    if (p.axis != nullptr) {
      ax = p.axis[k];
      ax = ax < 0 ? 0 : ax >= p.axes ? p.axes - 1 : ax;
    }
    const double turns = (double)p.pos[(int64_t)ax * p.pos_stride + t0 + t] *
                         (double)p.freq[k] * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = c * p.factor;
    sn[i] = s * p.factor;
  }
  __syncthreads();
  const int heads = p.q_heads + p.k_heads;
  const int h0 = blockIdx.y * p.span;
  const int hs = heads - h0 < p.span ? heads - h0 : p.span;
  const int lane = threadIdx.x & (T - 1), team = threadIdx.x / T;
  float* y_team = ys + team * (T * E);
  const int tasks = tokens * hs;
  const bool live = lane < p.chunks;
  for (int task = team; task < tasks; task += HR_THREADS / T) {
    const int t = task / hs, h = h0 + task - t * hs;
    const bool is_k = h >= p.q_heads;
    const RotarySide& side = is_k ? p.k : p.q;
    const int hh = is_k ? h - p.q_heads : h;
    const int64_t at = (int64_t)hh * p.head_bytes + lane * 16;
    float x[E];
    u32x4_t raw{0, 0, 0, 0};
    if (live) raw = ld16(side.x + (t0 + t) * side.stride + at);
    hr_unpack<DT>(raw, x);
    if (p.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int d = T / 2; d > 0; d >>= 1) ss += __shfl_xor(ss, d, 64);
      const float r = rsqrtf(ss * p.inv_d + p.eps);
      float g[E];
      if (side.weight != nullptr && live) {
        hr_unpack<DT>(ld16(side.weight + lane * 16), g);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = 1.f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * r * g[e];
    }
    if (half > 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) y_team[lane * E + e] = x[e];
      // the lanes of a wave run in step; this keeps the compiler from moving the
      // reads before the writes
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const float* c_t = cs + t * half;
      const float* s_t = sn + t * half;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = lane * E + e;
        if (i >= p.rot) continue;
        bool first;
        int other, a;
        if (p.interleaved) {
          first = (i & 1) == 0;
          other = i ^ 1;
          a = i >> 1;
        } else {
          first = i < half;
          other = first ? i + half : i - half;
          a = first ? i : i - half;
        }
        const float z = __fmul_rn(y_team[other], s_t[a]);
        x[e] = fmaf(x[e], c_t[a], first ? -z : z);
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (live) st16(side.out + (t0 + t) * side.out_stride + at, hr_pack<DT>(x));
  }
}

template <int DT>
static hipError_t launch_rotary(RotaryParams p, hipStream_t st) {
  const int T = p.chunks <= 8 ? 8 : p.chunks <= 16 ? 16 : p.chunks <= 32 ? 32 : 64;
  const int teams = HR_THREADS / T, heads = p.q_heads + p.k_heads, half = p.rot / 2;
  p.tokens = 1;
  p.span = teams;
  if (p.n * ((heads + teams - 1) / teams) > 2048) {
    p.span = heads;
    if (half > 0) p.tokens = HR_ANGLES / half;
    if (half == 0 || p.tokens > 8) p.tokens = 8;
  }
  const dim3 grid((unsigned)((p.n + p.tokens - 1) / p.tokens),
                  (unsigned)((heads + p.span - 1) / p.span));
  if (T == 8) return launch_kernel(head_norm_rotary_kernel<DT, 8>, grid, dim3(HR_THREADS), 0, st, p);
  if (T == 16)
    return launch_kernel(head_norm_rotary_kernel<DT, 16>, grid, dim3(HR_THREADS), 0, st, p);
  if (T == 32)
    return launch_kernel(head_norm_rotary_kernel<DT, 32>, grid, dim3(HR_THREADS), 0, st, p);
  return launch_kernel(head_norm_rotary_kernel<DT, 64>, grid, dim3(HR_THREADS), 0, st, p);
}

hipError_t launch_head_norm_rotary(int dt, const RotaryParams& all, hipStream_t st) {
  RotaryParams p = all;
  for (int64_t t = 0; t < all.n; t += HR_TOKENS) {
    p.n = all.n - t < HR_TOKENS ? all.n - t : HR_TOKENS;
    const hipError_t e = dt == DT_BF16 ? launch_rotary<DT_BF16>(p, st) : launch_rotary<DT_F32>(p, st);
    if (e != hipSuccess) return e;
    for (RotarySide* s : {&p.q, &p.k}) {
      s->x += HR_TOKENS * s->stride;
      s->out += HR_TOKENS * s->out_stride;
    }
    if (p.pos != nullptr) p.pos += HR_TOKENS;
  }
  return hipSuccess;
}

}  // namespace lookme
