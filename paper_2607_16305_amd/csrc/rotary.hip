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
// whole number, good to 2^-51 of the turns (two products and the constant round to
// 2^-53 each), so a position of 10^6 has the angle that a float32 product would miss by
// 0.03.  What is left is float32 (2^-26 of a turn).  A token's angles are computed once
// for all of its heads.
//
// Bound by memory: 8192 rows of 40 heads of 128 in bf16, 168 MB read and written, take 33
// us (5.0 TB/s; a large copy reaches 4.9).  Each lane holds its two chunks of 16 bytes
// through norm and rotation, so a head is read and written once and nothing but the
// angles goes through LDS; the next head's loads are on their way meanwhile.  (Heads in
// LDS took 56 us, register pairs without loads past the caches 40.)  One token of 18
// heads: 3.2 us, a launch.  Halves whose boundary is no chunk's take their pairs through LDS:
// the same rows with 100 of 128 elements turned 57 us, with 96 40.
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

// two values to bf16, to nearest even
__device__ __forceinline__ uint32_t hr_bf16x2(float a, float b) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

template <int DT>
__device__ __forceinline__ u32x4_t hr_pack(const float (&f)[hr_elems<DT>()]) {
  u32x4_t v;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == DT_BF16) v[k] = hr_bf16x2(f[2 * k], f[2 * k + 1]);
    else v[k] = as_u32(f[k]);
  }
  return v;
}

// A head on a team of T lanes, two 16-byte chunks each; a workgroup takes `tokens`
// tokens and all of their heads, or `span` heads of one token.  PAIRED: halves whose
// boundary is a chunk's, so a lane's chunks are l and l + half of them and its pairs are
// its own; neighbouring pairs (chunks 2 l and 2 l + 1) are so anyway.  Elsewhere (half
// a multiple of no chunk) the other element comes through LDS.
enum : int { HR_PAIRED = 0, HR_NEIGHBOURS = 1, HR_ODD = 2 };

template <int DT, int T, int MODE, bool STREAM>
__global__ __launch_bounds__(HR_THREADS) void head_norm_rotary_kernel(RotaryParams p) {
  constexpr int E = hr_elems<DT>();
  constexpr int PAD = 16;                      // (read, not used, behind the last angle)
  __shared__ __attribute__((aligned(16))) float cs[HR_ANGLES + PAD], sn[HR_ANGLES + PAD];
  __shared__ __attribute__((aligned(16))) float ys[MODE == HR_ODD ? HR_THREADS * 2 * E : 4];
  const int half = p.rot / 2, half4 = (half + 3) & ~3;
  const int lane = threadIdx.x & (T - 1), team = threadIdx.x / T;
  const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
  const int tokens = (int)(p.n - t0 < p.tokens ? p.n - t0 : p.tokens);
  const int heads = p.q_heads + p.k_heads, h0 = blockIdx.y * p.span;
  const int hs = heads - h0 < p.span ? heads - h0 : p.span;
  const int tasks = tokens * hs;
  // the lane's chunks
  const int pairs = MODE == HR_PAIRED ? half / E : 0;
  const int ca = MODE == HR_PAIRED && lane < pairs ? lane
                 : MODE == HR_PAIRED ? 2 * pairs + 2 * (lane - pairs) : 2 * lane;
  const int cb = MODE == HR_PAIRED && lane < pairs ? lane + pairs : ca + 1;
  const bool live_a = ca < p.chunks, live_b = cb < p.chunks;
  struct Place {
    int64_t row;
    int h;
    bool is_k;
  };
  auto place = [&](int task) {
    const int t = task / hs, h = h0 + task - t * hs;
    const bool is_k = h >= p.q_heads;
    return Place{t0 + t, is_k ? h - p.q_heads : h, is_k};
  };
  auto load = [&](int task, u32x4_t& a, u32x4_t& b) {
    const Place w = place(task);
    const char* x = (w.is_k ? p.k.x + w.row * p.k.stride : p.q.x + w.row * p.q.stride) +
                    (int64_t)w.h * p.head_bytes;
    a = b = u32x4_t{0, 0, 0, 0};
    if (live_a) a = STREAM ? ld16_nt(x + ca * 16) : ld16(x + ca * 16);
    if (live_b) b = STREAM ? ld16_nt(x + cb * 16) : ld16(x + cb * 16);
  };
  u32x4_t na, nb;
  if (team < tasks) load(team, na, nb);        // (on its way during the angles)
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
    cs[t * half4 + k] = c * p.factor;
    sn[t * half4 + k] = s * p.factor;
  }
  __syncthreads();
  float* y_team = ys + (MODE == HR_ODD ? team * (T * 2 * E) : 0);
  for (int task = team; task < tasks; task += HR_THREADS / T) {
    const Place w = place(task);
    const RotarySide& side = w.is_k ? p.k : p.q;
    float a[E], b[E];
    hr_unpack<DT>(na, a);
    hr_unpack<DT>(nb, b);
    const int next = task + HR_THREADS / T;
    if (next < tasks) load(next, na, nb);
    if (p.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(a[e], a[e], ss);
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(b[e], b[e], ss);
#pragma unroll
      for (int d = T / 2; d > 0; d >>= 1) ss += __shfl_xor(ss, d, 64);
      const float r = rsqrtf(ss * p.inv_d + p.eps);
      if (side.weight != nullptr) {
        float g[E];
        hr_unpack<DT>(live_a ? ld16(side.weight + ca * 16) : u32x4_t{0, 0, 0, 0}, g);
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] = a[e] * r * g[e];
        hr_unpack<DT>(live_b ? ld16(side.weight + cb * 16) : u32x4_t{0, 0, 0, 0}, g);
#pragma unroll
        for (int e = 0; e < E; ++e) b[e] = b[e] * r * g[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          a[e] *= r;
          b[e] *= r;
        }
      }
    }
    const float* c_t = cs + (int)(w.row - t0) * half4;
    const float* s_t = sn + (int)(w.row - t0) * half4;
    if constexpr (MODE == HR_ODD) {
      if (half > 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          y_team[lane * 2 * E + e] = a[e];
          y_team[lane * 2 * E + E + e] = b[e];
        }
        // the lanes of a wave run in step; this keeps the compiler from moving the
        // reads before the writes
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        auto turn = [&](int i, float y) {
          if (i >= p.rot) return y;
          const bool first = i < half;
          const int at = first ? i : i - half;
          const float z = y_team[first ? i + half : at] * s_t[at];
          return fmaf(y, c_t[at], first ? -z : z);
        };
#pragma unroll
        for (int e = 0; e < E; ++e) {
          a[e] = turn(lane * 2 * E + e, a[e]);
          b[e] = turn(lane * 2 * E + E + e, b[e]);
        }
        __builtin_amdgcn_wave_barrier();
      }
    } else if (lane * E < half) {
      float c[E], s[E];
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const f32x4_t cv = *reinterpret_cast<const f32x4_t*>(c_t + lane * E + e);
        const f32x4_t sv = *reinterpret_cast<const f32x4_t*>(s_t + lane * E + e);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          c[e + k] = cv[k];
          s[e + k] = sv[k];
        }
      }
      if constexpr (MODE == HR_PAIRED) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float y = a[e];
          a[e] = fmaf(y, c[e], -(b[e] * s[e]));
          b[e] = fmaf(b[e], c[e], y * s[e]);
        }
      } else {
        auto turn = [&](float& y0, float& y1, int i) {
          if (lane * E + i < half) {
            const float y = y0;
            y0 = fmaf(y, c[i], -(y1 * s[i]));
            y1 = fmaf(y1, c[i], y * s[i]);
          }
        };
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          turn(a[e], a[e + 1], e / 2);
          turn(b[e], b[e + 1], E / 2 + e / 2);
        }
      }
    }
    char* out = side.out + w.row * side.out_stride + (int64_t)w.h * p.head_bytes;
    if (live_a) st16(out + ca * 16, hr_pack<DT>(a));
    if (live_b) st16(out + cb * 16, hr_pack<DT>(b));
  }
}

template <int DT, int MODE>
static hipError_t launch_rotary_mode(RotaryParams p, hipStream_t st) {
  const int T = p.chunks <= 8 ? 4 : p.chunks <= 16 ? 8 : p.chunks <= 32 ? 16 : 32;
  const int teams = HR_THREADS / T, heads = p.q_heads + p.k_heads, half4 = (p.rot / 2 + 3) & ~3;
  // few rows: a team a head, so that the launch is as wide as it can be (3001 rows of 16
  // heads of 80 in float32 15 -> 10 us); many: whole tokens, up to 8 for one set of angles
  p.tokens = 1;
  p.span = teams;
  if (p.n * ((heads + teams - 1) / teams) > 2048) {
    p.span = heads;
    const int64_t most = half4 > HR_ANGLES / 8 ? HR_ANGLES / half4 : 8, spread = p.n / 2048;
    p.tokens = (int)(spread < 1 ? 1 : spread < most ? spread : most);
  }
  const dim3 grid((unsigned)((p.n + p.tokens - 1) / p.tokens),
                  (unsigned)((heads + p.span - 1) / p.span));
  const dim3 block(HR_THREADS);
  // rows that the caches cannot have kept are read past them (84 MB 40 -> 34 us; 31 MB, which
  // they have, 10 -> 14)
  if (p.n * heads * p.head_bytes >= (int64_t)1 << 26) {
    if (T == 4)
      return launch_kernel(head_norm_rotary_kernel<DT, 4, MODE, true>, grid, block, 0, st, p);
    if (T == 8)
      return launch_kernel(head_norm_rotary_kernel<DT, 8, MODE, true>, grid, block, 0, st, p);
    if (T == 16)
      return launch_kernel(head_norm_rotary_kernel<DT, 16, MODE, true>, grid, block, 0, st, p);
    return launch_kernel(head_norm_rotary_kernel<DT, 32, MODE, true>, grid, block, 0, st, p);
  }
  if (T == 4)
    return launch_kernel(head_norm_rotary_kernel<DT, 4, MODE, false>, grid, block, 0, st, p);
  if (T == 8)
    return launch_kernel(head_norm_rotary_kernel<DT, 8, MODE, false>, grid, block, 0, st, p);
  if (T == 16)
    return launch_kernel(head_norm_rotary_kernel<DT, 16, MODE, false>, grid, block, 0, st, p);
  return launch_kernel(head_norm_rotary_kernel<DT, 32, MODE, false>, grid, block, 0, st, p);
}

template <int DT>
static hipError_t launch_rotary(const RotaryParams& p, hipStream_t st) {
  if (p.interleaved) return launch_rotary_mode<DT, HR_NEIGHBOURS>(p, st);
  if (p.rot / 2 % hr_elems<DT>() == 0) return launch_rotary_mode<DT, HR_PAIRED>(p, st);
  return launch_rotary_mode<DT, HR_ODD>(p, st);
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
