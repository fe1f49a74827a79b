// The key and value cache of 4 bits: where a token's bytes are, and the format of
// its values (cache.hip writes and reads it, attend.hip multiplies with it).
//
// 32 neighbouring values of a head share a scale 2^(byte - 127); a value is 4
// bits, e2m1: a sign and 0, .5, 1, 1.5, 2, 3, 4 or 6.  Such a value times a power
// of two is exact in bf16, so the matrix cores take it without a rounding.
//
// A tile holds 32 tokens of a head, 34 d bytes: codes of k [16 d], codes of v
// [16 d], scales of k [d], scales of v [d], each in the order in which the lanes of
// a wave need them.  With lane = 16 c + j:
//   k is matrix operand [16 tokens, 32 dims] of the scores: the lane of token j
//     holds dims 32 m + 8 c .. + 7 of every m, d / 8 neighbouring bytes;
//   v is operand [16 dims, 32 tokens] of the outputs: the lane's dims are
//     j u .. j u + u - 1 with u = d / 16 (one for each of u products), its tokens
//     4 c .. 4 c + 3 and 16 + 4 c .. + 3, which is where the scores' product
//     leaves the weights of these tokens: 8 units of u / 2 bytes.
#pragma once

#include "common.h"

namespace lookme {

constexpr int C4_TILE = 32;            // tokens
constexpr int C4_NAN = 255;            // scale byte of a block that is not finite
                                       // (so reads any above C4_HIGHEST)
constexpr int C4_LOWEST = 127 - 100;   // smallest scale byte: smaller values become zeros
constexpr int C4_HIGHEST = 127 + 125;  // largest: 6 2^125 is finite, larger values saturate

// bytes within a tile; t: token, in [0, 32)
__host__ __device__ __forceinline__ int c4_k_code(int d, int t, int dim) {
  return t * (d / 2) + dim % 32 / 8 * (d / 8) + dim / 32 * 4 + dim % 8 / 2;
}
__host__ __device__ __forceinline__ int c4_v_code(int d, int t, int dim) {
  const int u = d / 16, lane = t % 16 / 4 * 16 + dim / u, place = t % 4 + 4 * (t / 16);
  return 16 * d + (lane * 8 + place) * (u / 2) + dim % u / 2;
}
__host__ __device__ __forceinline__ int c4_k_scale(int d, int t, int dim) {
  return 32 * d + t * (d / 32) + dim / 32;
}
__host__ __device__ __forceinline__ int c4_v_scale(int d, int t, int dim) {
  return 33 * d + dim / 32 * 32 + t % 16 / 4 * 8 + t % 4 + 4 * (t / 16);
}

// The scale byte of a block from the bits of its largest |value|: the smallest
// 2^E with |value| <= 7 2^E, so that the largest code, 6, is at most the half of
// its step off.
__device__ __forceinline__ int c4_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return C4_NAN;
  const int e = (int)((amax_bits + 0x1FFFFFu) >> 23) - 2;   // mantissa above 1.75: one more
  return e < C4_LOWEST ? C4_LOWEST : e > C4_HIGHEST ? C4_HIGHEST : e;
}
__device__ __forceinline__ float c4_power(int byte) {
  return byte > C4_HIGHEST ? as_f32(0x7FC00000u) : as_f32((uint32_t)byte << 23);
}

// two values from byte SEL of w: bf16, exact
__device__ __forceinline__ uint32_t c4_pair(uint32_t w, float scale, int sel) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  bf16x2_t v;
  switch (sel) {
    case 0: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0); break;
    case 1: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1); break;
    case 2: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2); break;
    default: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3); break;
  }
  return __builtin_bit_cast(uint32_t, v);
}

}  // namespace lookme
