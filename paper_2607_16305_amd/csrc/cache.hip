// Keys and values into the 4-bit cache as they come, and back (cache4.h has the
// format and the places of the bytes).
//
// A block of 32 values of a head is four lanes of a wave with 8 values each:
// its largest |value| over the four, the scale from its exponent, the codes by the
// conversion of this chip, which rounds to the nearest value, of two as near to
// the even code, and saturates.  Every step is exact but that rounding, so the
// bytes are a function of the 32 values alone.
//
// Both are bound by memory: 32768 rows of 8 heads of 128 in bf16 are written in 39 us (134
// MB read, 36 written: 4.4 TB/s) and read in 34 (36 read, 134 written: 5.0 TB/s); a large
// copy reaches 4.9.  64 rows take 3 us each, a launch.
#include "cache4.h"
#include "kernels.h"

namespace lookme {

// A workgroup takes 32 rows of a head, of k or of v.  k goes a row at a time; for v,
// where a lane of the attention reads 8 tokens, neighbouring threads take the 8 rows
// that are such a lane's when the rows are a tile: their bytes are neighbours then
// (any other slots are as right, only more scattered; with v a row at a time, each byte of
// a tile's line from another workgroup, the write took 52 us instead of 39).
constexpr int CW_THREADS = 256, CW_ROWS = 32;

// 8 values from p (16-byte aligned)
template <int DT, bool STREAM>
__device__ __forceinline__ void cw_load(const char* p, float (&x)[8]) {
  const u32x4_t a = STREAM ? ld16_nt(p) : ld16(p);
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
    const u32x4_t b = STREAM ? ld16_nt(p + 16) : ld16(p + 16);
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

// Task i of the workgroup's 32 rows by d / 8 chunks of 8 values
template <int D, bool V>
__device__ __forceinline__ void cw_task(int i, int* row, int* dim) {
  constexpr int L = D / 8;                     // chunks of a head
  if constexpr (V) {
    const int c = i / (8 * L), s = i % 8;
    *row = 4 * c + s % 4 + 16 * (s / 4);
    *dim = i / 8 % L * 8;
  } else {
    *row = i / L;
    *dim = i % L * 8;
  }
}

template <int DT, int D, bool V, bool STREAM>
__device__ __forceinline__ void cw_write(const CacheParams& p) {
  constexpr int STEP = V ? 8 : 1, TASKS = CW_ROWS * D / 8 / CW_THREADS;
  const int h = blockIdx.y;
  const int64_t row0 = (int64_t)blockIdx.x * CW_ROWS;
  float x[TASKS][8];
  int64_t tile[TASKS];
  int token[TASKS], dim[TASKS];
  bool live[TASKS];
  // (a row's values do not wait for its slot)
#pragma unroll
  for (int i = 0; i < TASKS; ++i) {
    int row;
    cw_task<D, V>(i * CW_THREADS + threadIdx.x, &row, &dim[i]);
    const int64_t r = row0 + row < p.n ? row0 + row : p.n - 1;
    cw_load<DT, STREAM>((V ? p.v + r * p.v_stride : p.k + r * p.k_stride) +
                    ((int64_t)h * D + dim[i]) * (DT == DT_BF16 ? 2 : 4), x[i]);
    live[i] = c4_slot(p, p.slots[r], h, &tile[i], &token[i]) && row0 + row < p.n;
  }
#pragma unroll
  for (int i = 0; i < TASKS; ++i) {
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = as_u32(x[i][e]) & 0x7FFFFFFFu;
      amax = a > amax ? a : amax;
    }
#pragma unroll
    for (int d = STEP; d < 4 * STEP; d <<= 1) {
      const uint32_t o = __shfl_xor(amax, d, 64);
      amax = o > amax ? o : amax;
    }
    if (!live[i]) continue;
    const int byte = c4_scale(amax);
    uint32_t w = 0;
    if (byte != C4_NAN) {
      const float s = c4_power(byte);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][0], x[i][1], s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][2], x[i][3], s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][4], x[i][5], s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i][6], x[i][7], s, 3);
    }
    uint8_t* t = p.cache + tile[i];
    if constexpr (V && D == 64) {   // two units of 4 values
      *reinterpret_cast<uint16_t*>(t + c4_v_code(D, token[i], dim[i])) = (uint16_t)w;
      *reinterpret_cast<uint16_t*>(t + c4_v_code(D, token[i], dim[i] + 4)) = (uint16_t)(w >> 16);
    } else {
      *reinterpret_cast<uint32_t*>(t + (V ? c4_v_code(D, token[i], dim[i])
                                          : c4_k_code(D, token[i], dim[i]))) = w;
    }
    if (dim[i] % 32 == 0)
      t[V ? c4_v_scale(D, token[i], dim[i]) : c4_k_scale(D, token[i], dim[i])] = (uint8_t)byte;
  }
}

template <int DT, int D, bool STREAM>
__global__ __launch_bounds__(CW_THREADS) void cache_write_kernel(CacheParams p) {
  if (blockIdx.z == 0) cw_write<DT, D, false, STREAM>(p);
  else cw_write<DT, D, true, STREAM>(p);
}

template <int DT, int D, bool V>
__device__ __forceinline__ void cw_read(const CacheParams& p) {
  const int h = blockIdx.y;
  const int64_t row0 = (int64_t)blockIdx.x * CW_ROWS;
#pragma unroll
  for (int i = 0; i < CW_ROWS * D / 8; i += CW_THREADS) {
    int row, dim;
    cw_task<D, V>(i + threadIdx.x, &row, &dim);
    const int64_t r = row0 + row;
    int64_t tile = 0;
    int token = 0;
    if (r >= p.n || !c4_slot(p, p.slots[r], h, &tile, &token)) continue;
    const uint8_t* t = p.cache + tile;
    uint32_t w;
    if constexpr (V && D == 64) {
      w = *reinterpret_cast<const uint16_t*>(t + c4_v_code(D, token, dim));
      w |= (uint32_t)*reinterpret_cast<const uint16_t*>(t + c4_v_code(D, token, dim + 4)) << 16;
    } else {
      w = *reinterpret_cast<const uint32_t*>(
          t + (V ? c4_v_code(D, token, dim) : c4_k_code(D, token, dim)));
    }
    const float s = c4_power(t[V ? c4_v_scale(D, token, dim) : c4_k_scale(D, token, dim)]);
    u32x4_t v;
#pragma unroll
    for (int b = 0; b < 4; ++b) v[b] = c4_pair(w, s, b);
    char* dst = (V ? p.v_out + r * p.v_stride : p.k_out + r * p.k_stride) +
                ((int64_t)h * D + dim) * (DT == DT_BF16 ? 2 : 4);
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
}

template <int DT, int D>
__global__ __launch_bounds__(CW_THREADS) void cache_read_kernel(CacheParams p) {
  if (p.k_out != nullptr && blockIdx.z == 0) cw_read<DT, D, false>(p);
  else cw_read<DT, D, true>(p);
}

template <int DT, int D>
static hipError_t launch_cache_d(bool write, CacheParams p, hipStream_t st) {
  // (a launch has under 2^32 threads)
  const int64_t most = ((int64_t)1 << 22) / p.heads * CW_ROWS;
  const unsigned sides = write || (p.k_out != nullptr && p.v_out != nullptr) ? 2 : 1;
  const int64_t n = p.n;
  // rows that the caches cannot have kept are read past them (32768 rows of 8 heads of
  // 128, 134 MB in all, 44 -> 39 us; ones that they have kept would take longer)
  const bool stream = n * p.heads * D * (DT == DT_BF16 ? 4 : 8) >= (int64_t)1 << 26;
  for (int64_t row = 0; row < n; row += most) {
    p.n = n - row < most ? n - row : most;
    const dim3 grid((unsigned)((p.n + CW_ROWS - 1) / CW_ROWS), (unsigned)p.heads, sides);
    const hipError_t e =
        !write ? launch_kernel(cache_read_kernel<DT, D>, grid, dim3(CW_THREADS), 0, st, p)
        : stream ? launch_kernel(cache_write_kernel<DT, D, true>, grid, dim3(CW_THREADS), 0, st, p)
                 : launch_kernel(cache_write_kernel<DT, D, false>, grid, dim3(CW_THREADS), 0, st, p);
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
