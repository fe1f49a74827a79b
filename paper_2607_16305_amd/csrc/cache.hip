// Keys and values into the 4-bit cache as they come, and back (cache4.h has the
// format and the places of the bytes).
//
// A block of 32 values of a head is four neighbouring lanes with 8 values each:
// its largest |value| over the four, the scale from its exponent, the codes by the
// conversion of this chip, which rounds to the nearest value, of two as near to
// the even code, and saturates.  Every step is exact but that rounding, so the
// bytes are a function of the 32 values alone.
#include "cache4.h"
#include "kernels.h"

namespace lookme {

constexpr int CW_THREADS = 256;

// 8 values from p (16-byte aligned)
template <int DT>
__device__ __forceinline__ void cw_load(const char* p, float (&x)[8]) {
  const u32x4_t a = ld16(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == DT_BF16) {
      x[2 * k] = bf16lo(a[k]);
      x[2 * k + 1] = bf16hi(a[k]);
    } else {
      x[k] = as_f32(a[k]);
    }
  }
  if constexpr (DT == DT_F32) {
    const u32x4_t b = ld16(p + 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[4 + k] = as_f32(b[k]);
  }
}

// Where slot s of head h is: its tile's address and its token there; false: no
// such slot.
__device__ __forceinline__ bool c4_slot(const CacheParams& p, int64_t s, int h, int64_t* tile,
                                        int* token) {
  if (s < 0 || s >= p.slots_all) return false;
  const int64_t page = s >> p.page_log2;
  const int in = (int)(s & ((1 << p.page_log2) - 1));
  *tile = ((page * p.heads + h) * ((int64_t)1 << (p.page_log2 - 5)) + in / C4_TILE) * 34 * p.d;
  *token = in % C4_TILE;
  return true;
}

// A thread: 8 values of one row's head, of k or of v.
template <int DT, int D>
__global__ __launch_bounds__(CW_THREADS) void cache_write_kernel(CacheParams p) {
  constexpr int L = D / 8;                     // lanes of a head
  const int64_t id = (int64_t)blockIdx.x * CW_THREADS + threadIdx.x;
  const int lane = (int)(id % L);
  const int64_t rest = id / L;
  const int h = (int)(rest % p.heads);
  const int64_t row = rest / p.heads;
  const bool is_v = blockIdx.y != 0;
  int64_t tile = 0;
  int token = 0;
  if (row >= p.n || !c4_slot(p, p.slots[row], h, &tile, &token)) return;   // whole teams of L
  const char* src = is_v ? p.v + row * p.v_stride : p.k + row * p.k_stride;
  float x[8];
  cw_load<DT>(src + ((int64_t)h * D + lane * 8) * (DT == DT_BF16 ? 2 : 4), x);
  uint32_t amax = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t a = as_u32(x[e]) & 0x7FFFFFFFu;
    amax = a > amax ? a : amax;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    const uint32_t o = __shfl_xor(amax, d, 64);
    amax = o > amax ? o : amax;
  }
  const int byte = c4_scale(amax);
  uint32_t w = 0;
  if (byte != C4_NAN) {
    const float s = c4_power(byte);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  }
  uint8_t* t = p.cache + tile;
  const int dim = lane * 8;
  if (!is_v) {
    *reinterpret_cast<uint32_t*>(t + c4_k_code(D, token, dim)) = w;
    if (lane % 4 == 0) t[c4_k_scale(D, token, dim)] = (uint8_t)byte;
  } else {
    if constexpr (D == 64) {   // two units of 4 values
      *reinterpret_cast<uint16_t*>(t + c4_v_code(D, token, dim)) = (uint16_t)w;
      *reinterpret_cast<uint16_t*>(t + c4_v_code(D, token, dim + 4)) = (uint16_t)(w >> 16);
    } else {
      *reinterpret_cast<uint32_t*>(t + c4_v_code(D, token, dim)) = w;
    }
    if (lane % 4 == 0) t[c4_v_scale(D, token, dim)] = (uint8_t)byte;
  }
}

template <int DT, int D>
__global__ __launch_bounds__(CW_THREADS) void cache_read_kernel(CacheParams p) {
  constexpr int L = D / 8;
  const int64_t id = (int64_t)blockIdx.x * CW_THREADS + threadIdx.x;
  const int lane = (int)(id % L);
  const int64_t rest = id / L;
  const int h = (int)(rest % p.heads);
  const int64_t row = rest / p.heads;
  const bool is_v = p.k_out == nullptr || blockIdx.y != 0;
  int64_t tile = 0;
  int token = 0;
  if (row >= p.n || !c4_slot(p, p.slots[row], h, &tile, &token)) return;
  const uint8_t* t = p.cache + tile;
  const int dim = lane * 8;
  uint32_t w;
  int byte;
  if (!is_v) {
    w = *reinterpret_cast<const uint32_t*>(t + c4_k_code(D, token, dim));
    byte = t[c4_k_scale(D, token, dim)];
  } else {
    if constexpr (D == 64) {
      w = *reinterpret_cast<const uint16_t*>(t + c4_v_code(D, token, dim));
      w |= (uint32_t)*reinterpret_cast<const uint16_t*>(t + c4_v_code(D, token, dim + 4)) << 16;
    } else {
      w = *reinterpret_cast<const uint32_t*>(t + c4_v_code(D, token, dim));
    }
    byte = t[c4_v_scale(D, token, dim)];
  }
  const float s = c4_power(byte);
  u32x4_t v;
#pragma unroll
  for (int b = 0; b < 4; ++b) v[b] = c4_pair(w, s, b);
  char* dst = is_v ? p.v_out + row * p.v_stride : p.k_out + row * p.k_stride;
  dst += ((int64_t)h * D + dim) * (DT == DT_BF16 ? 2 : 4);
  if constexpr (DT == DT_BF16) {
    st16(dst, v);
  } else {
    u32x4_t a, b;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      a[2 * k] = as_u32(bf16lo(v[k]));
      a[2 * k + 1] = as_u32(bf16hi(v[k]));
      b[2 * k] = as_u32(bf16lo(v[2 + k]));
      b[2 * k + 1] = as_u32(bf16hi(v[2 + k]));
    }
    st16(dst, a);
    st16(dst + 16, b);
  }
}

constexpr int64_t CW_BLOCKS = 1 << 23;   // of a launch, which has under 2^32 threads

template <int DT, int D>
static hipError_t launch_cache_d(bool write, CacheParams p, hipStream_t st) {
  const int64_t row_threads = (int64_t)p.heads * (D / 8);
  const int64_t most = CW_BLOCKS * CW_THREADS / row_threads;   // rows of a launch
  const unsigned sides = write || (p.k_out != nullptr && p.v_out != nullptr) ? 2 : 1;
  const int64_t n = p.n;
  for (int64_t row = 0; row < n; row += most) {
    p.n = n - row < most ? n - row : most;
    const dim3 grid((unsigned)((p.n * row_threads + CW_THREADS - 1) / CW_THREADS), sides);
    const hipError_t e =
        write ? launch_kernel(cache_write_kernel<DT, D>, grid, dim3(CW_THREADS), 0, st, p)
              : launch_kernel(cache_read_kernel<DT, D>, grid, dim3(CW_THREADS), 0, st, p);
    if (e != hipSuccess) return e;
    p.slots += most;
    if (write) {
      p.k += most * p.k_stride;
      p.v += most * p.v_stride;
    } else {
      if (p.k_out != nullptr) p.k_out += most * p.k_stride;
      if (p.v_out != nullptr) p.v_out += most * p.v_stride;
    }
  }
  return hipSuccess;
}

template <int DT>
static hipError_t launch_cache(bool write, const CacheParams& p, hipStream_t st) {
  if (p.d == 64) return launch_cache_d<DT, 64>(write, p, st);
  if (p.d == 128) return launch_cache_d<DT, 128>(write, p, st);
  return launch_cache_d<DT, 256>(write, p, st);
}

hipError_t launch_cache_write(int dt, const CacheParams& p, hipStream_t st) {
  return dt == DT_BF16 ? launch_cache<DT_BF16>(true, p, st) : launch_cache<DT_F32>(true, p, st);
}

hipError_t launch_cache_read(int dt, const CacheParams& p, hipStream_t st) {
  return dt == DT_BF16 ? launch_cache<DT_BF16>(false, p, st) : launch_cache<DT_F32>(false, p, st);
}

}  // namespace lookme
