// Attention of a batch's rows over the 4-bit cache of their sequences (cache4.h
// has its format): for row i of a sequence and query head h,
//
//   s_t = scale q[i, h] . k[t, h / G],   p = softmax over the visible t,
//   out[i, h] = sum_t p_t v[t, h / G]
//
// in one pass over the keys with a running maximum and sum.  The G query heads
// of a key head and the rows of a sequence are one list of rows, row r = (row r / G,
// head r % G), 16 of which are a tile of the matrix cores.  The scores are
// taken transposed, S^T = K Q^T: a lane then holds one row's scores of the tokens
// 4 c .. 4 c + 3 and 16 + 4 c .. + 3 (c = lane / 16), which is what the second
// product, out^T = V^T P^T, wants from it, so the weights never leave their
// registers.  The cache is laid out for that: a lane's bytes are neighbours, and
// a conversion makes two bf16 values of a byte and its scale, exactly.
//
// Rounding: k and v are exact, sums and the softmax float32; bf16 rows round their
// weights p to bf16 for the second product (half a step, 2^-8 relative, of independent
// signs; the output has the same step), float32 rows take q and p as three bf16
// values each, which hold all 24 bits.
#include <numeric>
#include <type_traits>

#include "cache4.h"
#include "dtl.h"
#include "kernels.h"

namespace lookme {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// Fewest tiles of a work unit; the rescaling waits until a maximum has grown by
// 2^AT_SLACK.
constexpr int AT_MIN_TILES = 4;
constexpr float AT_SLACK = 8.f;
// Scaled scores beyond this leave a weight's exponent to the rounding of the maximum.  Float32
// scores that differ are 2^6 apart there, so that any scale that keeps the maximum exact gives
// their weights: the next power of two.
constexpr float AT_WIDE = 1073741824.f;
constexpr int AT_UNITS_OF_SEQ = 1 << 24;
constexpr int AT_INLINE = 64;    // sequences that a unit looks at by itself

// ---------------------------------------------------------------------------
// work units: (sequence, key head, block of rows, part of the keys)
// ---------------------------------------------------------------------------
struct AttendSeq {
  int q0, rows, len;   // first row, rows, visible length
};

__device__ __forceinline__ AttendSeq at_seq(const AttendParams& p, int b) {
  AttendSeq s;
  s.q0 = b;
  s.rows = 1;
  if (p.q_offsets != nullptr) {
    const int a = p.q_offsets[b], e = p.q_offsets[b + 1];
    s.q0 = a < 0 ? 0 : a > p.n ? p.n : a;
    const int end = e > p.n ? p.n : e;
    s.rows = end > s.q0 ? end - s.q0 : 0;
  }
  const int64_t held = (int64_t)p.max_pages << p.page_log2;
  const int len = p.lengths[b];
  s.len = len < 0 ? 0 : len > held ? (int)held : len;
  return s;
}

struct AttendUnit {
  AttendSeq seq;
  int b, local, splits;   // sequence, index among its units, parts of its keys
  int part;               // index among the units whose keys are cut, of its sequence's first
};

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// The workspace: p.target 2 units' outputs [BR, D], their rows' (maximum, sum), then the plan:
// whether keys are cut and the count of units, and of every sequence where its units and
// its parts begin and the parts of its keys
template <int D, int BR>
__device__ __forceinline__ float* at_sums(const AttendParams& p) {
  return p.part + (int64_t)2 * p.target * BR * D;
}
struct AttendCut {
  uint32_t unit;     // its first unit (where attend_plan_kernel has written it)
  int part;          // index among the units whose keys are cut, of its first one
  int splits, pad;   // parts of its keys
};
struct AttendHead {
  int cut;
  uint32_t units;
  int pad[2];
};
template <int D, int BR>
__device__ __forceinline__ AttendHead* at_head(const AttendParams& p) {
  return reinterpret_cast<AttendHead*>(at_sums<D, BR>(p) + (int64_t)2 * p.target * BR * 2);
}
template <int D, int BR>
__device__ __forceinline__ AttendCut* at_cuts(const AttendParams& p) {
  return reinterpret_cast<AttendCut*>(at_head<D, BR>(p) + 1);
}

// Inclusive sum over the 1024 threads of a workgroup, and the sum of all (wrapping: what
// offsets that are not ascending give is checked where it is used)
__device__ __forceinline__ uint32_t at_block_scan(uint32_t v, int* sums, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  if (lane == 63) sums[wave] = (int)v;
  __syncthreads();
  uint32_t off = 0, sum = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) off += (uint32_t)sums[w];
    sum += (uint32_t)sums[w];
  }
  __syncthreads();
  *all = sum;
  return v + off;
}

// Blocks of BR rows of a sequence, of all its key heads
template <int BR>
__device__ __forceinline__ int at_blocks(const AttendParams& p, const AttendSeq& s) {
  return (int)(((int64_t)s.rows * (p.q_heads / p.kv_heads) + BR - 1) / BR) * p.kv_heads;
}
__device__ __forceinline__ int at_tiles(const AttendSeq& s) {
  return (s.len + C4_TILE - 1) / C4_TILE;
}

// Tiles of a part of the keys, of sequences with `blocks` blocks of rows, `work` tiles of
// them in all and `longest` of one: parts of about the same size, so that there are about
// p.target units whatever the lengths, or everything, where the longest sequence keeps its
// workgroups less than it costs to join parts.
template <int BR>
__device__ __forceinline__ int at_chunk(const AttendParams& p, int blocks, float work,
                                        float longest) {
  if ((longest - work / (float)p.target) * p.tile_us <= p.join_us) return 0x7FFFFFFF;
  // Parts are rounded up, half a part a block: of units of 32 to 64 rows, which are long
  // in their beginning and end, none is to be left for a second round (15 x 40 rows over
  // 6700 tokens 43 -> 35 us; units of 16 rows even out better without: 276 and 300)
  const float room = BR > 16 && BR < 128 ? 0.5f * fminf((float)blocks, (float)p.target) : 0.f;
  const float c = ceilf(work / ((float)p.target - room));
  return c < (float)AT_MIN_TILES ? AT_MIN_TILES : c > 1e9f ? 1000000000 : (int)c;
}

// The last of `count` entries whose key (ascending) is at most x, 64 at a time; 0 where
// none is
template <class F>
__device__ __forceinline__ int at_search(int count, F at_most) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, b = lo + lane * step;
    const uint64_t found = __ballot(b < hi && at_most(b)) | 1u;
    lo += (63 - __clzll((long long)found)) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Unit `unit` of the batch, the same for every lane of the wave.  64 sequences are looked
// at by the lanes of every wave.  More would cost each of the many units that they are as
// much as its work (1024 rows of 500 tokens 215 us, 4096 1983): with whole keys a unit
// finds its sequence by q_offsets alone, from a count of blocks that never is too small,
// and where they may be cut attend_plan_kernel has written where each one begins (107 to
// 117 us and 435 to 502).
template <int D, int BR>
__device__ __forceinline__ bool at_unit(const AttendParams& p, int unit, AttendUnit* u) {
  const int lane = threadIdx.x & 63;
  if (p.batch <= AT_INLINE) {
    AttendSeq s{0, 0, 0};
    if (lane < p.batch) s = at_seq(p, lane);
    const int mine = at_blocks<BR>(p, s), tiles = at_tiles(s);
    const int blocks = wave_sum(mine < AT_UNITS_OF_SEQ ? mine : AT_UNITS_OF_SEQ);
    int chunk = 0x7FFFFFFF;
    if (p.target > 0) {
      float longest = mine > 0 ? (float)tiles : 0.f;
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) longest = fmaxf(longest, __shfl_xor(longest, d, 64));
      // (alike in every lane, and known to be: what follows stays in scalar registers)
      chunk = __builtin_amdgcn_readfirstlane(
          at_chunk<BR>(p, blocks, wave_sum((float)mine * (float)tiles), longest));
      if (unit == 0 && threadIdx.x == 0) at_head<D, BR>(p)->cut = chunk != 0x7FFFFFFF;
    }
    if (chunk == 0x7FFFFFFF) {
      // without a cut the blocks of rows of one key head read the same keys: a
      // neighbourhood of units for each XCD, so that they meet in its L2
      unit = __builtin_amdgcn_readfirstlane(xcd_remap(unit, blocks));
      if (unit < 0) return false;
    }
    const int splits = tiles > chunk ? (tiles + chunk - 1) / chunk : 1;
    const int64_t all = (int64_t)mine * splits;
    const int units = all > AT_UNITS_OF_SEQ ? AT_UNITS_OF_SEQ : (int)all;
    const int cut = splits > 1 ? units : 0;
    const int incl = wave_scan_incl(units), cut_incl = wave_scan_incl(cut);
    const uint64_t found = __ballot(unit < incl);
    if (found == 0) return false;
    const int l = __ffsll((unsigned long long)found) - 1;
    u->b = l;
    u->seq.q0 = __builtin_amdgcn_readlane(s.q0, l);
    u->seq.rows = __builtin_amdgcn_readlane(s.rows, l);
    u->seq.len = __builtin_amdgcn_readlane(s.len, l);
    u->splits = __builtin_amdgcn_readlane(splits, l);
    u->local = unit - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(units, l));
    u->part = __builtin_amdgcn_readlane(cut_incl, l) - __builtin_amdgcn_readlane(cut, l);
    if (p.target > 0 && u->local == 0 && threadIdx.x == 0) {
      AttendCut* c = at_cuts<D, BR>(p) + l;
      c->part = u->part;
      c->splits = u->splits;
    }
    return true;
  }
  const AttendCut* cuts = at_cuts<D, BR>(p);
  uint32_t first;
  int count = 0;
  if (p.target > 0) {
    const AttendHead* head = at_head<D, BR>(p);
    const uint32_t units = head->units;
    if (head->cut == 0) unit = __builtin_amdgcn_readfirstlane(xcd_remap(unit, (int)units));
    if (unit < 0 || (uint32_t)unit >= units) return false;
    u->b = at_search(p.batch, [&](int b) { return cuts[b].unit <= (uint32_t)unit; });
    first = cuts[u->b].unit;
    u->part = cuts[u->b].part;
    u->splits = cuts[u->b].splits;
  } else {
    // Sequence b's blocks, of one key head, begin at or behind (q0 G + b pad) / BR: with pad =
    // BR - gcd(G, BR), that leaves it room for its last, partial block
    const int G = p.q_heads / p.kv_heads;
    auto begin = [&](int b) {
      int64_t q0 = b;
      if (p.q_offsets != nullptr) {
        const int a = p.q_offsets[b];
        q0 = a < 0 ? 0 : a > p.n ? p.n : a;
      }
      return (int)((q0 * G + (int64_t)b * p.pad) / BR);
    };
    unit = __builtin_amdgcn_readfirstlane(xcd_remap(unit, begin(p.batch) * p.kv_heads));
    if (unit < 0) return false;
    const int slot = unit / p.kv_heads;
    u->b = at_search(p.batch, [&](int b) { return begin(b) <= slot; });
    first = (uint32_t)(begin(u->b) * p.kv_heads);
    count = begin(u->b + 1) * p.kv_heads - (int)first;
    u->part = 0;
    u->splits = 1;
  }
  u->seq = at_seq(p, u->b);
  const int blocks = at_blocks<BR>(p, u->seq);
  u->local = (int)((uint32_t)unit - first);
  if (p.target == 0) {
    // (by key head: its blocks, then what was left over)
    const int slots = count / p.kv_heads, each = blocks / p.kv_heads;
    if (u->local < 0 || u->local >= count) return false;
    const int h = u->local / slots, x = u->local - h * slots;
    u->local = h * each + x;
    if (x >= each) return false;
  }
  u->seq.q0 = __builtin_amdgcn_readfirstlane(u->seq.q0);
  u->seq.rows = __builtin_amdgcn_readfirstlane(u->seq.rows);
  u->seq.len = __builtin_amdgcn_readfirstlane(u->seq.len);
  u->splits = __builtin_amdgcn_readfirstlane(u->splits);
  u->part = __builtin_amdgcn_readfirstlane(u->part);
  u->local = __builtin_amdgcn_readfirstlane(u->local);
  return u->local >= 0 && u->local < (int64_t)blocks * u->splits;
}

// The plan of a call of more than AT_INLINE sequences whose keys may be cut, by one workgroup
template <int D, int BR>
__global__ __launch_bounds__(1024) void attend_plan_kernel(AttendParams p) {
  __shared__ float works[16], longs[16];
  __shared__ int sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float work = 0.f, longest = 0.f;
  int64_t mine = 0;
  for (int b = threadIdx.x; b < p.batch; b += 1024) {
    const AttendSeq s = at_seq(p, b);
    const int n = at_blocks<BR>(p, s);
    mine += n;
    work += (float)n * (float)at_tiles(s);
    longest = fmaxf(longest, n > 0 ? (float)at_tiles(s) : 0.f);
  }
  // (what is not more than the launch's units; offsets that are not ascending may give more)
  const int some = wave_sum((int)(mine < 1 << 20 ? mine : 1 << 20));
  work = wave_sum(work);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) longest = fmaxf(longest, __shfl_xor(longest, d, 64));
  if (lane == 0) {
    works[wave] = work;
    longs[wave] = longest;
    sums[wave] = some;
  }
  __syncthreads();
  int blocks = 0;
  work = longest = 0.f;
  for (int w = 0; w < 16; ++w) {
    work += works[w];
    longest = fmaxf(longest, longs[w]);
    blocks += sums[w];
  }
  __syncthreads();
  const int chunk = at_chunk<BR>(p, blocks, work, longest);
  AttendCut* cuts = at_cuts<D, BR>(p);
  uint32_t before = 0, parts = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    AttendSeq s{0, 0, 0};
    if (b < p.batch) s = at_seq(p, b);
    const int tiles = at_tiles(s), splits = tiles > chunk ? (tiles + chunk - 1) / chunk : 1;
    const uint32_t units = (uint32_t)at_blocks<BR>(p, s) * (uint32_t)splits;
    const uint32_t cut = splits > 1 ? units : 0;
    uint32_t all, all_cut;
    const uint32_t at = before + at_block_scan(units, sums, &all) - units;
    const uint32_t part = parts + at_block_scan(cut, sums, &all_cut) - cut;
    if (b < p.batch) cuts[b] = AttendCut{at, (int)part, splits, 0};
    before += all;
    parts += all_cut;
  }
  if (threadIdx.x == 0) *at_head<D, BR>(p) = AttendHead{parts > 0, before, {0, 0}};
}

// ---------------------------------------------------------------------------
// a tile of 32 tokens in a lane's registers
// ---------------------------------------------------------------------------
template <int D>
struct AttendTile {
  static constexpr int U = D / 16, M = D / 32;
  uint32_t k[2][M], v[U], ks[2][(M + 3) / 4], vs[2];
};

template <int N>
__device__ __forceinline__ void at_load_words(uint32_t (&w)[N], const uint8_t* p) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const u32x2_t v = *reinterpret_cast<const u32x2_t*>(p);
    w[0] = v[0];
    w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4_t v = ld16(p + 16 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
    }
  }
}

template <int D>
__device__ __forceinline__ void at_load(AttendTile<D>& t, const uint8_t* tile) {
  const uint32_t lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
#pragma unroll
  for (int s = 0; s < 2; ++s)
    at_load_words(t.k[s], tile + (16 * s + j) * (D / 2) + c * (D / 8));
  at_load_words(t.v, tile + 16 * D + (c * 16 + j) * (D / 4));
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint8_t* at = tile + 32 * D + (16 * s + j) * (D / 32);
    if constexpr (D == 64) t.ks[s][0] = *reinterpret_cast<const uint16_t*>(at);
    else at_load_words(t.ks[s], at);
  }
  at_load_words(t.vs, tile + 33 * D + j * (D / 16) / 32 * 32 + c * 8);
}

// The scale of byte i of w: the conversion takes a float's exponent and nothing else of
// it, so the other bytes may stand in its sign and significand (255: NaN)
__device__ __forceinline__ float at_scale(uint32_t w, int i) {
  return as_f32(i == 3 ? w >> 1 : w << (23 - 8 * i));
}

// x as `terms` bf16 values that add up to it
template <int DT>
constexpr int at_terms() {
  return DT == DT_BF16 ? 1 : 3;
}

__device__ __forceinline__ uint32_t at_pack(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

template <int DT>
__device__ __forceinline__ void at_split(float a, float b, uint32_t (&w)[at_terms<DT>()]) {
  w[0] = at_pack(a, b);
  if constexpr (DT == DT_F32) {
    a -= bf16lo(w[0]);
    b -= bf16hi(w[0]);
    w[1] = at_pack(a, b);
    w[2] = at_pack(a - bf16lo(w[1]), b - bf16hi(w[1]));
  }
}

// at_split of float32 of any size: also where it is infinite, or finite and the nearest bf16
// is not, its first value is then what it begins with
__device__ __forceinline__ void at_split_any(float a, float b, uint32_t (&w)[3]) {
  auto first = [](float x, uint32_t near) {
    return (near & 0x7FFFu) == 0x7F80u ? as_u32(x) >> 16 : near;
  };
  const uint32_t near = at_pack(a, b);
  w[0] = first(a, near & 0xFFFFu) | first(b, near >> 16) << 16;
  a = fabsf(a) == INFINITY ? 0.f : a - bf16lo(w[0]);
  b = fabsf(b) == INFINITY ? 0.f : b - bf16hi(w[0]);
  w[1] = at_pack(a, b);
  w[2] = at_pack(a - bf16lo(w[1]), b - bf16hi(w[1]));
}

// The largest of the four lanes that hold a row
__device__ __forceinline__ float at_row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// Weight of a part whose maximum is m, of M over all (both in powers of two)
__device__ __forceinline__ float at_weight(float m, float M) {
  return m == -INFINITY ? 0.f : exp2f(m - M);
}

// ---------------------------------------------------------------------------
// a wave's rows, RT tiles of 16: running maxima and sums over the tokens so far
// ---------------------------------------------------------------------------
// A lane holds, of row j of each tile, dims (4 c + i) u + m in acc[.][m][i]; the
// sum of the row's weights is acc[.][u], the product with a row of ones, which
// the matrix cores do while the vector instructions are what is short.
template <int D, int RT>
struct AttendRows {
  static constexpr int U = D / 16;
  f32x4_t acc[RT][U + 1];
  float top[RT], next[RT], base[RT];   // maximum, where it is renewed, in powers of two
  float scl[RT];                       // that a score has for a power of two
  int last[RT];                        // the last token that the row sees

  __device__ __forceinline__ void clear(float scale) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      top[rt] = next[rt] = -INFINITY;
      base[rt] = 0.f;
      scl[rt] = scale;
#pragma unroll
      for (int m = 0; m <= U; ++m) acc[rt][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }

  // scores of the tile from token t0 that a row does not see
  __device__ __forceinline__ void mask(f32x4_t (&s)[RT][2], int t0) const {
    const int c = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + 16 * half + 4 * c + i > last[rt]) s[rt][half][i] = -INFINITY;
  }

  // NaN into the dims of the blocks of v that are not finite (a byte above C4_HIGHEST among
  // the tile's scales) of rows that see them.  The products take such blocks as zeros, which
  // would meet weights of 0 otherwise.
  __device__ __forceinline__ void holes(const uint8_t* scales, int t0) {
    const int c = (threadIdx.x & 63) >> 4;
    uint32_t nan_rows[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) nan_rows[rt] = 0;
    for (int g = 0; g < D / 32; ++g) {
      uint32_t vs[2];
      at_load_words(vs, scales + g * 32 + c * 8);
      for (int x = 0; x < 8; ++x) {
        const bool hole = ((vs[x / 4] >> (8 * (x % 4))) & 0xFFu) > (uint32_t)C4_HIGHEST;
        const int token = t0 + 4 * c + x % 4 + 16 * (x / 4);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          nan_rows[rt] |= (hole && token <= last[rt] ? 1u : 0u) << g;
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      nan_rows[rt] |= __shfl_xor(nan_rows[rt], 16, 64);
      nan_rows[rt] |= __shfl_xor(nan_rows[rt], 32, 64);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((nan_rows[rt] >> ((4 * c + i) * U / 32)) & 1u)
#pragma unroll
          for (int m = 0; m < U; ++m) acc[rt][m][i] = as_f32(0x7FC00000u);
    }
  }

  // The maximum is renewed, and what there is rescaled, only when a score has passed
  // it by 2^AT_SLACK: the weights stay far from float32's ends, and most tiles need
  // neither.
  __device__ __forceinline__ void renew(const f32x4_t (&s)[RT][2], const AttendParams& p,
                                        float slack) {
    float mx[RT];
    bool grown = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mx[rt] = s[rt][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx[rt] = fmaxf(mx[rt], s[rt][e / 4][e % 4]);
      grown |= mx[rt] > next[rt];
    }
    if (__builtin_expect(__any(grown), 0)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float now = fmaxf(top[rt], at_row_max(mx[rt]));
        // (finite, so that scaled scores past float32 are what their infinities would be:
        // minus weighs 0, plus gives NaN)
        const bool wide = now != -INFINITY && fabsf(now * p.scale_log2) > AT_WIDE;
        scl[rt] = wide ? p.scale_wide : p.scale_log2;
        const float b = now == -INFINITY ? 0.f
                                         : fminf(fmaxf(now * scl[rt], -__FLT_MAX__), __FLT_MAX__);
        const float f = top[rt] == -INFINITY ? 0.f : exp2f(base[rt] - b);
        top[rt] = now;
        next[rt] = now + slack;
        base[rt] = b;
#pragma unroll
        for (int m = 0; m <= U; ++m) acc[rt][m] *= f;
      }
    }
  }

  // Scores into weights 2^(s scl - base)
  template <int DT>
  __device__ __forceinline__ void weights(const f32x4_t (&s)[RT][2],
                                          u32x4_t (&w)[RT][at_terms<DT>()]) const {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float e[8];
#pragma unroll
      for (int x = 0; x < 8; ++x)
        e[x] = __builtin_amdgcn_exp2f(fmaf(s[rt][x / 4][x % 4], scl[rt], -base[rt]));
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        uint32_t o[at_terms<DT>()];
        at_split<DT>(e[2 * x], e[2 * x + 1], o);
#pragma unroll
        for (int k = 0; k < at_terms<DT>(); ++k) w[rt][k][x] = o[k];
      }
    }
  }

  // acc[.][m] += v^T w
  template <int TERMS>
  __device__ __forceinline__ void add(int m, u32x4_t v, const u32x4_t (&w)[RT][TERMS]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int k = TERMS - 1; k >= 0; --k)
        acc[rt][m] = mfma_chunk<DT_BF16>(v, w[rt][k], acc[rt][m]);
  }
  template <int TERMS>
  __device__ __forceinline__ void add_ones(const u32x4_t (&w)[RT][TERMS]) {
    add(U, u32x4_t{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, w);
  }

  __device__ __forceinline__ float ref(int rt) const {
    return top[rt] == -INFINITY ? -INFINITY : base[rt];
  }

  // Joins tile rt of a wave that left its rows at `other` (acc, then ref); ref_rt: this
  // wave's, renewed
  static constexpr int LEFT = RT * ((U + 1) * 1024 + 256);   // bytes
  __device__ __forceinline__ void leave(char* to, const float (&refs)[RT]) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      reinterpret_cast<float*>(to + RT * (U + 1) * 1024)[rt * 64 + lane] = refs[rt];
#pragma unroll
      for (int m = 0; m <= U; ++m)
        reinterpret_cast<f32x4_t*>(to)[(rt * (U + 1) + m) * 64 + lane] = acc[rt][m];
    }
  }
  __device__ __forceinline__ void join(const char* from, float (&refs)[RT]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float other = reinterpret_cast<const float*>(from + RT * (U + 1) * 1024)[rt * 64 + lane];
      const float most = fmaxf(refs[rt], other);
      const float a = at_weight(refs[rt], most), b = at_weight(other, most);
      refs[rt] = most;
#pragma unroll
      for (int m = 0; m <= U; ++m)
        acc[rt][m] = acc[rt][m] * a +
                     reinterpret_cast<const f32x4_t*>(from)[(rt * (U + 1) + m) * 64 + lane] * b;
    }
  }
};

// What the waves of a unit know of it
struct AttendBlock {
  AttendUnit u;
  int G, R, blk, h, split;   // heads of a key head, rows, block of rows, key head, part of the keys
  int first, end;            // the part's tiles
};

template <int D, int BR>
__device__ __forceinline__ bool at_block(const AttendParams& p, AttendBlock* k) {
  if (!at_unit<D, BR>(p, blockIdx.x, &k->u)) return false;
  k->G = p.q_heads / p.kv_heads;
  k->R = k->u.seq.rows * k->G;
  const int blocks = (k->R + BR - 1) / BR, hs = k->u.local / blocks;
  k->blk = blocks - 1 - k->u.local % blocks;     // the longest first
  k->h = hs / k->u.splits;
  k->split = hs % k->u.splits;
  const int end_row = k->blk * BR + BR < k->R ? k->blk * BR + BR : k->R;
  const int seen = p.causal ? k->u.seq.len - k->u.seq.rows + (end_row - 1) / k->G + 1 : k->u.seq.len;
  const int tiles = seen > 0 ? (seen + C4_TILE - 1) / C4_TILE : 0;   // (early rows may see none)
  const int per = (tiles + k->u.splits - 1) / k->u.splits;
  k->first = k->split * per;
  k->end = k->first + per < tiles ? k->first + per : tiles;
  return true;
}

// The last token that row r sees
__device__ __forceinline__ int at_last(const AttendParams& p, const AttendBlock& k, int r) {
  return p.causal ? k.u.seq.len - k.u.seq.rows + r / k.G : k.u.seq.len - 1;
}

// Where the block's tiles are
template <int D>
struct AttendPages {
  // (scalar loads, which the counts of loads in flight below leave out)
  typedef const __attribute__((address_space(4))) int32_t* scalar_ptr_t;
  scalar_ptr_t pages;
  const uint8_t* head;       // the key head's tiles of page 0
  int64_t page_bytes;
  int tiles_log2, num_pages;

  __device__ __forceinline__ AttendPages(const AttendParams& p, const AttendBlock& k)
      : pages((scalar_ptr_t)(uintptr_t)(p.pages + (int64_t)k.u.b * p.max_pages)),
        head(p.cache + ((int64_t)k.h << (p.page_log2 - 5)) * (34 * D)),
        page_bytes(((int64_t)p.kv_heads << (p.page_log2 - 5)) * (34 * D)),
        tiles_log2(p.page_log2 - 5), num_pages(p.num_pages) {}
  __device__ __forceinline__ int id(int t) const { return pages[t >> tiles_log2]; }
  __device__ __forceinline__ bool held(int id) const { return id >= 0 && id < num_pages; }
  __device__ __forceinline__ const uint8_t* tile(int t, int id) const {
    return head + (held(id) ? id : 0) * page_bytes + (t & ((1 << tiles_log2) - 1)) * (34 * D);
  }
};

// The queries of RT tiles from row row0 as matrix operands
template <int DT, int D, int RT>
__device__ __forceinline__ void at_queries(const AttendParams& p, const AttendBlock& k, int row0,
                                           u32x4_t (&q)[RT][D / 32][at_terms<DT>()]) {
  constexpr int TERMS = at_terms<DT>(), ES = DT == DT_BF16 ? 2 : 4;
  const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
  // `any`: by at_split_any
  auto load = [&](auto any, int rt) {
    const int r = row0 + rt * 16 + j, i = r < k.R ? r / k.G : 0;
    const char* src = p.q + (k.u.seq.q0 + i) * p.q_stride +
                      ((int64_t)k.h * k.G + (r < k.R ? r - i * k.G : 0)) * D * ES;
    float most = 0.f;
#pragma unroll
    for (int m = 0; m < D / 32; ++m) {
      if constexpr (DT == DT_BF16) {
        q[rt][m][0] = r < k.R ? ld16(src + (32 * m + 8 * c) * 2) : u32x4_t{0, 0, 0, 0};
      } else {
        u32x4_t a{0, 0, 0, 0}, b{0, 0, 0, 0};
        if (r < k.R) {
          a = ld16(src + (32 * m + 8 * c) * 4);
          b = ld16(src + (32 * m + 8 * c) * 4 + 16);
        }
        const f32x4_t af = __builtin_bit_cast(f32x4_t, a), bf = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(fmaxf(most, fabsf(af[e])), fabsf(bf[e]));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t w[TERMS], x[TERMS];
          if constexpr (decltype(any)::value) {
            at_split_any(af[2 * e], af[2 * e + 1], w);
            at_split_any(bf[2 * e], bf[2 * e + 1], x);
          } else {
            at_split<DT>(af[2 * e], af[2 * e + 1], w);
            at_split<DT>(bf[2 * e], bf[2 * e + 1], x);
          }
#pragma unroll
          for (int n = 0; n < TERMS; ++n) {
            q[rt][m][n][e] = w[n];
            q[rt][m][n][2 + e] = x[n];
          }
        }
      }
    }
    return most;
  };
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float most = load(std::false_type(), rt);
    constexpr float BF16_MOST = 0x1.fep127f;
    if constexpr (DT == DT_F32)
      if (__builtin_expect(__any(most > BF16_MOST), 0)) load(std::true_type(), rt);
  }
  // (waited for here, once: the compiler would wait for every load in the loop)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
      for (int n = 0; n < TERMS; ++n) asm volatile("" : "+v"(q[rt][m][n]));
}

// The outputs of a wave's rows, or what a part of the keys gives for them
template <int DT, int D, int RT, int BR>
__device__ __forceinline__ void at_store(const AttendParams& p, const AttendBlock& k, int row0,
                                         const AttendRows<D, RT>& a, const float (&refs)[RT]) {
  constexpr int U = D / 16, ES = DT == DT_BF16 ? 2 : 4;
  const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + j;
    if (r >= k.R) continue;
    const float sum = a.acc[rt][U][0];
    if (k.u.splits > 1) {
      const int64_t at = (int64_t)(k.u.part + k.u.local) * BR + (r - k.blk * BR);
      float* dst = p.part + at * D + 4 * c * U;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < U; m += 4)
          *reinterpret_cast<f32x4_t*>(dst + i * U + m) =
              f32x4_t{a.acc[rt][m][i], a.acc[rt][m + 1][i], a.acc[rt][m + 2][i],
                      a.acc[rt][m + 3][i]};
      if (c == 0)
        reinterpret_cast<f32x2_t*>(at_sums<D, BR>(p))[at] = f32x2_t{refs[rt], sum};
      continue;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int i = r / k.G;
    char* dst = p.out + (int64_t)(k.u.seq.q0 + i) * p.out_stride +
                ((int64_t)k.h * k.G + (r - i * k.G)) * D * ES + 4 * c * U * ES;
    float o[4 * U];
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
      for (int m = 0; m < U; ++m) o[i4 * U + m] = a.acc[rt][m][i4] * inv;
#pragma unroll
    for (int x = 0; x < 4 * U * ES / 16; ++x) {
      u32x4_t v;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if constexpr (DT == DT_BF16) v[n] = at_pack(o[8 * x + 2 * n], o[8 * x + 2 * n + 1]);
        else v[n] = as_u32(o[4 * x + n]);
      }
      st16(dst + 16 * x, v);
    }
  }
}

// Whether one of 8 scale bytes is above C4_HIGHEST (its complement below 3): 255, or what no
// write leaves, 253 and 254, whose larger values bf16 cannot hold
__device__ __forceinline__ bool at_hole(const uint32_t (&vs)[2]) {
  const uint32_t a = ~vs[0], b = ~vs[1];
  constexpr uint32_t BELOW = (255 - C4_HIGHEST) * 0x01010101u;
  return ((((a - BELOW) & ~a) | ((b - BELOW) & ~b)) & 0x80808080u) != 0;
}

// Zeros in the place of the lane's tokens whose block of v is not finite, or which lie
// behind the last one, where anything may be
template <int D>
__device__ __forceinline__ void at_fill_holes(uint32_t (&v)[D / 16], uint32_t (&vs)[2], int t0,
                                              int len) {
  constexpr int U = D / 16;
  const int c = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const int token = t0 + 4 * c + x % 4 + 16 * (x / 4), bit = 8 * (x % 4);
    asm volatile("");   // (rare: not to be turned into selects on everybody's way)
    if (token >= len || ((vs[x / 4] >> bit) & 0xFFu) > (uint32_t)C4_HIGHEST) {
      vs[x / 4] = (vs[x / 4] & ~(0xFFu << bit)) | (127u << bit);
      if constexpr (U == 4) {
        v[x / 2] &= x % 2 == 0 ? 0xFFFF0000u : 0x0000FFFFu;
      } else {
#pragma unroll
        for (int w = 0; w < U / 8; ++w) v[x * (U / 8) + w] = 0;
      }
    }
  }
}

// Operand m = 2 b and 2 b + 1 of v: byte b of a token's unit holds these dims
template <int D>
__device__ __forceinline__ void at_v_operands(const uint32_t (&v)[D / 16], const uint32_t (&vs)[2],
                                              int b, u32x4_t* lo, u32x4_t* hi) {
  uint32_t pair[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const int byte = x * (D / 32) + b;
    pair[x] = c4_pair(v[byte / 4], at_scale(vs[x / 4], x % 4), byte % 4);
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    (*lo)[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x05040100u);
    (*hi)[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x07060302u);
  }
}

__device__ __forceinline__ u32x4_t at_k_operand(uint32_t k, float scale) {
  return u32x4_t{c4_pair(k, scale, 0), c4_pair(k, scale, 1), c4_pair(k, scale, 2),
                 c4_pair(k, scale, 3)};
}

// ---------------------------------------------------------------------------
// few rows a key head (a decode step, some tokens more): RT tiles of 16 a unit, its waves
// along the tokens
// ---------------------------------------------------------------------------
constexpr int AF_WAVES = 4;
// Waves a SIMD, as the registers allow (rt: tiles of 16 rows a unit)
constexpr int af_occupancy(int dt, int d, int rt) {
  if (rt > 2) return 2;
  if (rt == 2) return dt == DT_F32 ? (d == 64 ? 2 : 1) : d == 64 ? 3 : d == 128 ? 2 : 1;
  return d == 64 ? 4 : d == 128 ? 3 : dt == DT_BF16 ? 2 : 1;
}
// tiles of a wave's ring in LDS, one of them being multiplied
constexpr int af_ring(int d) { return d == 64 ? 4 : 2; }

// A tile on its way into LDS: 1 KB an instruction, the last one on some of the lanes
template <int D>
constexpr int at_instr() {
  return 34 * D / 1024 + 1;
}
template <int D>
__device__ __forceinline__ void at_issue(const uint8_t* tile, char* dst) {
  const int lane = threadIdx.x & 63;
  constexpr int FULL = 34 * D / 1024, REST = 34 * D % 1024 / 16;
#pragma unroll
  for (int i = 0; i < FULL; ++i) load_lds16_nt(tile + i * 1024 + lane * 16, dst + i * 1024);
  if (lane < REST) load_lds16_nt(tile + FULL * 1024 + lane * 16, dst + FULL * 1024);
}

// Bound by memory for a row or two a key head, by vector instructions from there on (two
// values an unpacking instruction, an exponential a score).  A row of 64 heads over 131072
// tokens of 8 key heads of 128, 4 sequences (570 MB), takes 97 us, 5.9 TB/s; the same
// stream with the arithmetic left out takes 93.  What carried it there (us of that case): tiles in
// registers, waited for one by one 160 and in turns 134; each wave's own ring in LDS,
// filled past the registers and without barriers, 120; nontemporal loads and the rows'
// sums in the matrix cores 104; rare cases (masks, blocks that are not finite) out of
// everybody's way 97.  Rings of 3 tiles and 8 waves were no faster.  64 sequences of up to
// 8192 tokens, 290 MB, take 54.  300 rows of 16 heads of 64 over up to 2880 tokens, 8
// sequences, take 36 to 40: matrix cores 0.21, the rest unpacking, exponentials and the
// uneven end.
template <int DT, int D, int RT>
__global__ __launch_bounds__(64 * AF_WAVES, af_occupancy(DT, D, RT))
void attend_few_kernel(AttendParams p) {
  constexpr int U = D / 16, M = D / 32, BR = 16 * RT, TERMS = at_terms<DT>();
  constexpr int NB = af_ring(D), TILE = 34 * D;
  constexpr int RING = AF_WAVES * NB * TILE, JOIN = AF_WAVES / 2 * AttendRows<D, RT>::LEFT;
  // the waves' rings of tiles, then what they join
  __shared__ __attribute__((aligned(1024))) char smem[RING > JOIN ? RING : JOIN];
  const int lane = threadIdx.x & 63, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  AttendBlock k;
  if (!at_block<D, BR>(p, &k)) return;
  const int row0 = k.blk * BR;
  AttendRows<D, RT> rows;
  rows.clear(p.scale_log2);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + j;
    rows.last[rt] = r < k.R ? at_last(p, k, r) : -1;
  }
  const int full = at_last(p, k, row0);      // every row sees the tokens up to here
  const float slack = fminf(AT_SLACK / p.scale_log2, 1e38f);
  const AttendPages<D> pages(p, k);

  // The wave's own ring: NB - 1 tiles on their way while one is multiplied, no barrier,
  // the page of the next one ahead of them.  `bad`: bit i, the tile i turns ahead is on
  // no page.
  char* ring = smem + wave * (NB * TILE);
  uint32_t bad = 0;
  int t = k.first + wave, slot = 0;
  int id = t < k.end ? pages.id(t) : 0;
  auto issue = [&](int x, int at) {
    at_issue<D>(pages.tile(x, id), ring + at * TILE);
    bad |= (pages.held(id) ? 0u : 1u) << (NB - 1);
    id = pages.id(x + AF_WAVES < k.end ? x + AF_WAVES : x);
  };
#pragma unroll
  for (int i = 0; i < NB - 1; ++i) {
    bad >>= 1;
    if (t + i * AF_WAVES < k.end) issue(t + i * AF_WAVES, i);
  }
  u32x4_t q[RT][M][TERMS];
  at_queries<DT, D, RT>(p, k, row0, q);
  for (; t < k.end; t += AF_WAVES) {
    bad >>= 1;
    if (t + (NB - 1) * AF_WAVES < k.end) {
      issue(t + (NB - 1) * AF_WAVES, slot == 0 ? NB - 1 : slot - 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 1) * at_instr<D>()) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    if ((bad & 1u) == 0) {
      const uint8_t* tile = reinterpret_cast<const uint8_t*>(ring + slot * TILE);
      AttendTile<D> cur;
      at_load(cur, tile);
      const int t0 = t * C4_TILE;
      f32x4_t s[RT][2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][half] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const u32x4_t kv = at_k_operand(cur.k[half][m], at_scale(cur.ks[half][m / 4], m % 4));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x)
              s[rt][half] = mfma_chunk<DT_BF16>(kv, q[rt][m][x], s[rt][half]);
        }
      }
      const bool hole = __any(at_hole(cur.vs));
      if (__builtin_expect(hole || t0 + C4_TILE - 1 > full, 0)) {
        rows.mask(s, t0);
        if (hole) rows.holes(tile + 33 * D, t0);
        at_fill_holes<D>(cur.v, cur.vs, t0, k.u.seq.len);
      }
      rows.renew(s, p, slack);
      u32x4_t w[RT][TERMS];
      rows.template weights<DT>(s, w);
      rows.add_ones(w);
#pragma unroll
      for (int b = 0; b < U / 2; ++b) {
        u32x4_t lo, hi;
        at_v_operands<D>(cur.v, cur.vs, b, &lo, &hi);
        rows.add(2 * b, lo, w);
        rows.add(2 * b + 1, hi, w);
      }
    }
    slot = slot == NB - 1 ? 0 : slot + 1;
    asm volatile("" ::: "memory");
  }

  float refs[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) refs[rt] = rows.ref(rt);
  __syncthreads();   // the rings are free for the join
#pragma unroll
  for (int step = AF_WAVES / 2; step > 0; step >>= 1) {
    char* left = smem + (wave & (step - 1)) * AttendRows<D, RT>::LEFT;
    if (wave >= step && wave < 2 * step) rows.leave(left, refs);
    __syncthreads();
    if (wave < step) rows.join(left, refs);
    if (step > 1) __syncthreads();
  }
  if (wave == 0) at_store<DT, D, RT, BR>(p, k, row0, rows, refs);
}

// ---------------------------------------------------------------------------
// many rows a key head (prefill, cross attention): the waves of a workgroup along
// the rows, RT tiles of 16 each; a tile of the cache is unpacked once, a quarter by
// each wave, and read as matrix operands from LDS
// ---------------------------------------------------------------------------
constexpr int AM_WAVES = 4;
// As many row tiles as leave two waves a SIMD (bf16, 256 dims, 2 x 3954 rows over 9178
// tokens x 4 heads: one 382 us, two and one wave 519; float32, 128 dims: one 185, two 201)
constexpr int am_row_tiles(int dt, int d) { return dt == DT_BF16 && d == 128 ? 2 : 1; }

// A wave's share of a tile of 128 or 256 dims: D / 64 of the D / 16 operands of k, D / 128
// of the D / 32 pairs of operands of v
template <int D>
struct AttendShare {
  static constexpr int M = D / 32, U = D / 16;
  static constexpr int KN = D / 64, VN = D / 128;
  uint32_t k[KN], ks, v[U];
  uint32_t at_k, at_ks, at_v, at_vs;   // of the lane's bytes in a tile
  uint32_t ks_shift;                   // of its scales of k in their word
  __device__ __forceinline__ AttendShare(int wave) {
    const uint32_t lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
    const uint32_t half = wave >> 1, m0 = (wave & 1) * KN;
    at_k = (16 * half + j) * (D / 2) + c * (D / 8) + 4 * m0;
    at_ks = 32 * D + (16 * half + j) * M + m0;
    ks_shift = at_ks % 4 * 8;
    at_ks -= at_ks % 4;
    at_v = 16 * D + (c * 16 + j) * (D / 4);
    at_vs = 33 * D + j * U / 32 * 32 + c * 8;
  }
  __device__ __forceinline__ void load_k(const uint8_t* tile) {
    at_load_words(k, tile + at_k);
    ks = *reinterpret_cast<const uint32_t*>(tile + at_ks);
  }
  __device__ __forceinline__ void load_v(const uint8_t* tile) { at_load_words(v, tile + at_v); }
  __device__ __forceinline__ void load_scales(const uint8_t* tile, uint32_t (&vs)[2]) const {
    at_load_words(vs, tile + at_vs);
  }
  // operands at lds + n 1024
  __device__ __forceinline__ void unpack_k(char* lds, int wave) const {
    char* to = lds + (threadIdx.x & 63) * 16;
#pragma unroll
    for (int n = 0; n < KN; ++n)
      st16(to + (wave * KN + n) * 1024, at_k_operand(k[n], at_scale(ks >> ks_shift, n)));
  }
  __device__ __forceinline__ void unpack_v(char* lds, int wave, const uint32_t (&vs)[2]) const {
    char* to = lds + (threadIdx.x & 63) * 16;
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int b = wave * VN + n;      // byte b of every token's unit, as byte 0
      uint32_t pair[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        uint32_t word;
        if constexpr (U == 8) word = v[x];
        else word = b < 4 ? v[2 * x] : v[2 * x + 1];
        pair[x] = c4_pair(word >> (8 * (b & 3)), at_scale(vs[x / 4], x % 4), 0);
      }
      u32x4_t lo, hi;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        lo[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x05040100u);
        hi[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x07060302u);
      }
      st16(to + 2 * b * 1024, lo);
      st16(to + (2 * b + 1) * 1024, hi);
    }
  }
};

// Bound by the issue of instructions: the matrix cores are busy 0.44 of the time and vector
// instructions take 0.54 (2 x 4096 rows of 16 heads of 128, 4 key heads, at the end of 8192
// tokens: 414 to 507 us from card to card, 995 to 813 TFLOP/s).  Steps (us of that case):
// unpacking in every wave 1226, turns in registers 822, shared through LDS with the blocks of
// a key head on one XCD 587, the next tile's scores beside this one's weights and no
// copies of registers 560, rare cases out of the way 502.  Codes through a ring in LDS 605;
// three row tiles 617, one and more waves 613.
template <int DT, int D>
__global__ __launch_bounds__(64 * AM_WAVES, 2)
void attend_many_kernel(AttendParams p) {
  constexpr int U = D / 16, M = D / 32, TERMS = at_terms<DT>(), RT = am_row_tiles(DT, D);
  constexpr int BR = 16 * RT * AM_WAVES, STAGE = 4 * M * 1024;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  const int lane = threadIdx.x & 63, j = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  AttendBlock k;
  if (!at_block<D, BR>(p, &k)) return;
  const int row0 = k.blk * BR + wave * RT * 16;
  AttendRows<D, RT> rows;
  rows.clear(p.scale_log2);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + j;
    rows.last[rt] = r < k.R ? at_last(p, k, r) : -1;
  }
  const int full = row0 < k.R ? at_last(p, k, row0) : -1;   // every row sees the tokens up to here
  const float slack = fminf(AT_SLACK / p.scale_log2, 1e38f);
  const AttendPages<D> pages(p, k);

  // In one turn, of tile t: the scores of tile t + 1 (matrix cores) beside the weights of t
  // (vector instructions), then the outputs of t beside the unpacking of k of t + 2 and
  // v of t + 1 into the halves of LDS that were read before the last barrier: a half is
  // never written before one that follows its last reading.  One barrier a turn, and one
  // between the scores of the first tile and turn 0.
  char* const lds_k = smem;
  char* const lds_v = smem + STAGE;
  constexpr int HALF = STAGE / 2;
  AttendShare<D> share(wave);
  u32x4_t q[RT][M][TERMS];
  const int turns = k.end - k.first;
  if (turns > 0) {
    auto at = [&](int i) { return k.first + (i < turns ? i : turns - 1); };
    auto scores = [&](f32x4_t (&s)[RT][2], const char* ops) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][half] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const u32x4_t kv = ld16(ops + (half * M + m) * 1024 + lane * 16);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x)
              s[rt][half] = mfma_chunk<DT_BF16>(kv, q[rt][m][x], s[rt][half]);
        }
      }
    };
    // a tile's scores as its rows see them; a tile on no page is seen by none
    auto seen = [&](f32x4_t (&s)[RT][2], int i, int id) {
      const int t0 = (k.first + i) * C4_TILE;
      if (__builtin_expect(t0 + C4_TILE - 1 > full || !pages.held(id), 0))
        rows.mask(s, pages.held(id) ? t0 : 0x7FFFFF00);
      rows.renew(s, p, slack);
    };
    bool hole, hole1;   // in v of tiles i and i + 1
    auto mend = [&](int i, bool hole, uint32_t (&vs)[2]) {
      const int t0 = (k.first + i) * C4_TILE;
      if (__builtin_expect(hole || t0 + C4_TILE > k.u.seq.len, 0))
        at_fill_holes<D>(share.v, vs, t0, k.u.seq.len);
    };
    uint32_t vs_even[2], vs_odd[2];
    f32x4_t s_even[RT][2], s_odd[RT][2];
    int id = pages.id(at(0)), id1 = pages.id(at(1)), id2 = pages.id(at(2));
    const uint8_t* tile = pages.tile(at(0), id);
    share.load_k(tile);
    share.load_v(tile);
    share.load_scales(tile, vs_odd);
    at_queries<DT, D, RT>(p, k, row0, q);
    share.unpack_k(lds_k, wave);
    hole = __any(at_hole(vs_odd));
    mend(0, hole, vs_odd);
    share.unpack_v(lds_v, wave, vs_odd);
    tile = pages.tile(at(1), id1);
    share.load_k(tile);
    share.load_v(tile);
    share.load_scales(tile, vs_even);
    share.unpack_k(lds_k + HALF, wave);
    tile = pages.tile(at(2), id2);
    share.load_k(tile);
    share.load_scales(tile, vs_odd);
    __syncthreads();
    scores(s_even, lds_k);
    __syncthreads();   // (turn 0 writes k of tile 2 where these were read)
    seen(s_even, 0, id);
    hole1 = __any(at_hole(vs_even));
    // (even and odd turns: what is loaded or computed for a later one keeps its registers)
    auto turn = [&](auto odd, int i, const f32x4_t (&s)[RT][2], f32x4_t (&ahead)[RT][2],
                    uint32_t (&vs)[2], const uint32_t (&vs_next)[2]) {
      constexpr int HERE = decltype(odd)::value ? HALF : 0, THERE = HALF - HERE;
      mend(i + 1, hole1, vs);
      const int id3 = pages.id(at(i + 3));
      scores(ahead, lds_k + THERE);
      u32x4_t w[RT][TERMS];
      rows.template weights<DT>(s, w);
      const char* ops = lds_v + HERE + lane * 16;
      rows.add_ones(w);
#pragma unroll
      for (int m = 0; m < U; ++m) rows.add(m, ld16(ops + m * 1024), w);
      share.unpack_k(lds_k + HERE, wave);
      share.unpack_v(lds_v + THERE, wave, vs);
      const bool hole2 = __any(at_hole(vs_next));   // (these have come, the loads below have not)
      share.load_v(tile);
      tile = pages.tile(at(i + 3), id3);
      share.load_k(tile);
      share.load_scales(tile, vs);
      if (__builtin_expect(hole, 0)) {
        if (pages.held(id))
          rows.holes(pages.tile(at(i), id) + 33 * D, (k.first + i) * C4_TILE);
      }
      __syncthreads();
      seen(ahead, i + 1, id1);   // (behind the last tile: of no use, and of no harm)
      hole = hole1;
      hole1 = hole2;
      id = id1;
      id1 = id2;
      id2 = id3;
    };
    int i = 0;
    while (true) {
      turn(std::false_type(), i, s_even, s_odd, vs_even, vs_odd);
      if (++i == turns) break;
      turn(std::true_type(), i, s_odd, s_even, vs_odd, vs_even);
      if (++i == turns) break;
    }
  }
  float refs[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) refs[rt] = rows.ref(rt);
  at_store<DT, D, RT, BR>(p, k, row0, rows, refs);
}

// Joins the parts of a row's keys: W waves a row and query head, 64 parts at a time
// whose weights the lanes compute side by side (250 parts one after the other took 25 us,
// so 6).  Bound by latency, 4 to 5 us of which 2.7 are a launch.  Rows from `from` on, of all
// rows' query heads.
template <int DT, int D, int BR, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void attend_join_kernel(AttendParams p,
                                                                            int from) {
  constexpr int E = D / 64, AHEAD = 8;     // values of a lane, parts on their way
  typedef float fe_t __attribute__((ext_vector_type(E)));
  __shared__ fe_t accs[W][64];
  __shared__ float ms[W], ls[W];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = from + (W == 1 ? blockIdx.x * 4 + wave : blockIdx.x);
  if (at >= p.n * p.q_heads) return;
  const int row = at / p.q_heads, head = at - row * p.q_heads, G = p.q_heads / p.kv_heads;
  if (at_head<D, BR>(p)->cut == 0) return;
  // the row's sequence
  const int b = p.q_offsets == nullptr
                    ? row : at_search(p.batch, [&](int i) { return p.q_offsets[i] <= row; });
  const AttendSeq s = at_seq(p, b);
  if (row < s.q0 || row >= s.q0 + s.rows) return;
  const int part = at_cuts<D, BR>(p)[b].part, splits = at_cuts<D, BR>(p)[b].splits;
  if (splits <= 1 || splits > 2 * p.target) return;
  const int blocks = (s.rows * G + BR - 1) / BR;
  const int h = head / G, r = (row - s.q0) * G + head - h * G, blk = r / BR;
  const int64_t first = ((int64_t)part + (int64_t)h * splits * blocks + (blocks - 1 - blk)) * BR +
                        (r - blk * BR);
  const int64_t step = (int64_t)blocks * BR;
  // (sequences that share rows can be more units than the launch has: then one may not
  // have written where its parts are)
  if (part < 0 || first + (splits - 1) * step >= (int64_t)2 * p.target * BR) return;
  const f32x2_t* sums = reinterpret_cast<const f32x2_t*>(at_sums<D, BR>(p));
  const fe_t* outs = reinterpret_cast<const fe_t*>(p.part) + lane;
  float m = -INFINITY, sum = 0.f;
  fe_t acc = {};
  const int mine = W == 1 ? splits : (splits - wave + W - 1) / W;   // parts wave, wave + W, ..
  auto part_of = [&](int i) { return first + (int64_t)(W == 1 ? i : wave + i * W) * step; };
  for (int i0 = 0; i0 < mine; i0 += 64) {
    const int n = mine - i0 < 64 ? mine - i0 : 64;
    f32x2_t ml = {-INFINITY, 0.f};
    if (lane < n) ml = sums[part_of(i0 + lane)];
    fe_t v[AHEAD];
    auto load = [&](int i) {
#pragma unroll
      for (int x = 0; x < AHEAD; ++x)
        if (i + x < n) v[x] = outs[part_of(i0 + i + x) * 64];
    };
    load(0);
    auto of_lane = [](float y, int l) { return as_f32(__builtin_amdgcn_readlane(as_u32(y), l)); };
    float most = ml[0];
    if (n <= AHEAD) {
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) most = fmaxf(x == 0 ? m : most, of_lane(ml[0], x));
    } else {
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
      most = fmaxf(most, m);
    }
    const float f = at_weight(m, most), w = at_weight(ml[0], most);
    m = most;
    sum *= f;
    acc *= f;
    for (int i = 0; i < n; i += AHEAD) {
      if (i > 0) load(i);
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        if (i + x >= n) break;
        const float g = of_lane(w, i + x);
        sum = fmaf(of_lane(ml[1], i + x), g, sum);
        acc += v[x] * g;
      }
    }
  }
  if constexpr (W > 1) {
    accs[wave][lane] = acc;
    if (lane == 0) {
      ms[wave] = m;
      ls[wave] = sum;
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int x = 1; x < W; ++x) {
      const float most = fmaxf(m, ms[x]), a = at_weight(m, most), c = at_weight(ms[x], most);
      m = most;
      sum = sum * a + ls[x] * c;
      acc = acc * a + accs[x][lane] * c;
    }
  }
  acc *= sum == 0.f ? 0.f : 1.f / sum;
  constexpr int ES = DT == DT_BF16 ? 2 : 4;
  char* dst = p.out + row * p.out_stride + ((int64_t)head * D + E * lane) * ES;
  if constexpr (DT == DT_F32) {
    *reinterpret_cast<fe_t*>(dst) = acc;
  } else {
    typedef __bf16 be_t __attribute__((ext_vector_type(E)));
    *reinterpret_cast<be_t*>(dst) = __builtin_convertvector(acc, be_t);
  }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------
static int many_block(int dt, int d) {
  return 16 * AM_WAVES * am_row_tiles(dt, d);
}

// Row tiles of a unit of attend_few_kernel for `rows` rows of a sequence and key head; 0:
// attend_many_kernel.  A few-rows unit unpacks a tile of the cache once for its 16 to 48
// rows, without a barrier; a many-rows unit once for 64 or 128, through LDS.  Two tiles keep
// two or three waves a SIMD, three save a block where two would hold padding.  Both sides
// (us, 16 sequences x 8192 tokens x 4 heads of 128): 32 rows, two tiles and many 33 and 55;
// 48 rows, three, two and many 36, 41, 57; 64 rows 50, 41, 60; 80 rows 50, 67, 62; 128 rows 83,
// 68, 70; 200 rows of 32 x 16 heads over 1500 tokens 145, 161, 138; 16 x 8 heads of 256
// over 4096 tokens: 36 rows, two and many 68 and 83, 100 rows 126 and 107; float32, 128
// dims: 36 rows 62 and 67, 2048 rows 404 and 337; 256 dims, one and many: 36 rows 123 and
// 129, 1024 rows 455 and 456.  64 dims have no many-rows kernel: 2048 rows took it 127 us,
// two tiles take 107 and four 101, but 300 rows of 8 x 16 heads over 2880 tokens 40 and
// 45, 64 rows of 20 x 16 heads over 4000 34 and 50 (float32 219 with it, two tiles 182).
static int few_tiles(int dt, int d, int64_t rows) {
  if (rows <= 16 || (dt == DT_F32 && d == 256)) return 1;
  if (rows <= 32 || d == 64) return 2;
  if (dt == DT_F32 || d == 256) return rows <= 64 ? 2 : 0;
  return rows <= 48 ? 3 : rows <= 64 ? 2 : rows <= 96 ? 3 : 0;
}

// The keys are cut where that saves more than it costs.  It saves a unit's turns (tile_us a
// tile, in microseconds) as far as the blocks of rows leave workgroups free; it costs a
// launch, and each row's parts written and read again.  (500 rows of 500 tokens: 20 us
// whole, 24 cut; 64 rows of 1024 tokens 12 and 17; a row of 2048 tokens 16 and 10; 11
// sequences of up to 32000 tokens x 64 heads 340 and 282.)  Here the lengths are not known,
// only what the page table could hold: the call gets a join where the keys would be cut
// were they all that long, or where one long sequence among short ones could keep a few
// workgroups busy by itself (one of 131072 tokens among 127 of 1000, 8 key heads: 631 us
// whole, 64 cut; units of many rows only in the first case); the kernel then decides by
// the lengths (at_unit), and a join with nothing to do takes 4 to 5 us with the plan (64
// rows of 1000 tokens 12 -> 18).  Units are of one size for all sequences, from the mean of
// their rows: single rows beside a long block of rows take units of many rows too, whole
// where that block fills the chip.
AttendPlan attend_plan(int dt, int64_t n, int batch, int q_heads, int kv_heads, int d,
                       int64_t tokens) {
  const int64_t rows = n * (q_heads / kv_heads), each = (rows + batch - 1) / batch;
  AttendPlan a{};
  a.tiles = few_tiles(dt, d, each);
  // many rows, but too few for most of the chip, over few tokens: more and shorter units
  // (500 rows of 8 heads over 500 tokens 12 us, as many rows 20)
  const int64_t large = ((each + many_block(dt, d) - 1) / many_block(dt, d)) * batch * kv_heads;
  if (a.tiles == 0 && large <= 120 && tokens <= 64 * C4_TILE) a.tiles = 2;
  a.block = a.tiles > 0 ? 16 * a.tiles : many_block(dt, d);
  // (one round of resident workgroups; 512 of 128 rows and 128 dims are 68 MB)
  a.target = a.tiles > 0 ? 256 * af_occupancy(dt, d, a.tiles) : d == 128 ? 480 : 448;
  a.tile_us = a.tiles > 0 ? 0.18f * (1 + a.tiles) / AF_WAVES : 0.5f;
  a.join_us = (float)((double)n * q_heads * d * 16 / 2.5e6);
  const double turns = (double)((tokens + C4_TILE - 1) / C4_TILE) * a.tile_us;
  const double blocks = (double)((each + a.block - 1) / a.block) * kv_heads;   // of a sequence
  if ((1.0 - blocks * batch / a.target) * turns <= 4.0 + a.join_us &&
      (a.tiles == 0 || batch > 1 << 17 ||
       (1.0 - blocks / a.target) * turns <= 40.0 + a.join_us))
    a.target = 0;
  a.units = (rows / a.block + batch) * kv_heads + (a.target > 0 ? a.target + 64 : 0);
  return a;
}

size_t attend_workspace(int dt, int64_t n, int batch, int q_heads, int kv_heads, int d,
                        int64_t tokens) {
  const AttendPlan a = attend_plan(dt, n, batch, q_heads, kv_heads, d, tokens);
  return a.target == 0 ? 0 : (size_t)2 * a.target * a.block * (d + 2) * 4 +
                               sizeof(AttendHead) + sizeof(AttendCut) * batch;
}

template <int D, int BR>
static hipError_t launch_plan(const AttendParams& p, hipStream_t st) {
  if (p.target == 0 || p.batch <= AT_INLINE) return hipSuccess;
  return launch_kernel(attend_plan_kernel<D, BR>, dim3(1), dim3(1024), 0, st, p);
}

// A wave a row: 64 threads each, and a launch has under 2^32
template <int DT, int D, int BR>
static hipError_t launch_join(const AttendParams& p, hipStream_t st) {
  constexpr int64_t MOST = 1 << 25;
  const int64_t rows = (int64_t)p.n * p.q_heads;
  for (int64_t from = 0; from < rows; from += MOST) {
    const int64_t n = rows - from < MOST ? rows - from : MOST;
    const dim3 grid((unsigned)((n + 3) / 4));
    const hipError_t e =
        launch_kernel(attend_join_kernel<DT, D, BR, 1>, grid, dim3(256), 0, st, p, (int)from);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int DT, int D, int RT>
static hipError_t launch_few(const AttendPlan& a, const AttendParams& p, dim3 grid, hipStream_t st) {
  hipError_t e = launch_plan<D, 16 * RT>(p, st);
  if (e == hipSuccess)
    e = launch_kernel(attend_few_kernel<DT, D, RT>, grid, dim3(64 * AF_WAVES), 0, st, p);
  if (e != hipSuccess || a.target == 0) return e;
  // a wave a row where that fills the chip, else as many as do
  const int64_t rows = (int64_t)p.n * p.q_heads;
  if (rows >= 2048) return launch_join<DT, D, 16 * RT>(p, st);
  const dim3 each((unsigned)rows);
  // (42 rows with up to 250 parts each took 25 us with four waves a row, 6 with
  // sixteen; 16 rows of 16 parts 4.4 and 5.4)
  const int64_t even = a.target / ((int64_t)p.batch * p.kv_heads),
                held = ((int64_t)p.max_pages << p.page_log2) / (C4_TILE * AT_MIN_TILES);
  if (rows < 512 && even > 32 && held > 32)
    return launch_kernel(attend_join_kernel<DT, D, 16 * RT, 16>, each, dim3(1024), 0, st, p, 0);
  return launch_kernel(attend_join_kernel<DT, D, 16 * RT, 4>, each, dim3(256), 0, st, p, 0);
}

template <int DT, int D>
static hipError_t launch_attend_d(AttendParams p, hipStream_t st) {
  const AttendPlan a = attend_plan(DT, p.n, p.batch, p.q_heads, p.kv_heads, D,
                                   (int64_t)p.max_pages << p.page_log2);
  p.target = a.target;
  p.tile_us = a.tile_us;
  p.join_us = a.join_us;
  p.pad = a.block - std::gcd(p.q_heads / p.kv_heads, a.block);
  const dim3 grid((unsigned)((a.units + 7) / 8 * 8));
  // (what few_tiles chooses, and nothing else, is built)
  if (a.tiles == 1) return launch_few<DT, D, 1>(a, p, grid, st);
  if constexpr (DT == DT_BF16 || D < 256)
    if (a.tiles == 2) return launch_few<DT, D, 2>(a, p, grid, st);
  if constexpr (DT == DT_BF16 && D == 128)
    if (a.tiles == 3) return launch_few<DT, D, 3>(a, p, grid, st);
  if constexpr (D == 128 || (DT == DT_BF16 && D == 256)) {
    constexpr int BLOCK = 16 * AM_WAVES * am_row_tiles(DT, D);
    hipError_t e = launch_plan<D, BLOCK>(p, st);
    if (e == hipSuccess)
      e = launch_kernel(attend_many_kernel<DT, D>, grid, dim3(64 * AM_WAVES), 0, st, p);
    if (e != hipSuccess || a.target == 0) return e;
    return launch_join<DT, D, BLOCK>(p, st);
  }
  return hipErrorInvalidValue;   // (few_tiles gives no 0 there)
}

hipError_t launch_attend(int dt, int d, AttendParams p, hipStream_t st) {
  if (dt == DT_BF16) {
    if (d == 64) return launch_attend_d<DT_BF16, 64>(p, st);
    if (d == 128) return launch_attend_d<DT_BF16, 128>(p, st);
    return launch_attend_d<DT_BF16, 256>(p, st);
  }
  if (d == 64) return launch_attend_d<DT_F32, 64>(p, st);
  if (d == 128) return launch_attend_d<DT_F32, 128>(p, st);
  return launch_attend_d<DT_F32, 256>(p, st);
}

}  // namespace lookme
