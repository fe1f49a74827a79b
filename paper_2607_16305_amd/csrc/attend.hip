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
constexpr int AT_UNITS_OF_SEQ = 1 << 24;

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
  int64_t part;           // index among the units whose keys are cut
};

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Unit `unit` of the batch, the same for every lane of the wave.  The keys of all
// sequences are cut into parts of about the same size, so that there are about
// p.target units in all, whatever the lengths.  ROWS: a unit is a row of blocks
// all of whose parts count as one (for joining them).
template <int BR>
__device__ __forceinline__ bool at_unit(const AttendParams& p, int64_t unit, bool joined,
                                        AttendUnit* u) {
  const int lane = threadIdx.x & 63, G = p.q_heads / p.kv_heads;
  float work = 0.f;
  if (p.target > 0) {
    for (int b = lane; b < p.batch; b += 64) {
      const AttendSeq s = at_seq(p, b);
      const int64_t blocks = ((int64_t)s.rows * G + BR - 1) / BR;
      work += (float)blocks * (float)((s.len + C4_TILE - 1) / C4_TILE);
    }
    work = wave_sum(work) * (float)p.kv_heads;
  } else {
    // without a cut the blocks of rows of one key head read the same keys: a
    // neighbourhood of units for each XCD, so that they meet in its L2
    int all = 0;
    for (int b = lane; b < p.batch; b += 64)
      all += (int)(((int64_t)at_seq(p, b).rows * G + BR - 1) / BR * p.kv_heads);
    unit = __builtin_amdgcn_readfirstlane(xcd_remap((int)unit, wave_sum(all)));
    if (unit < 0) return false;
  }
  int chunk = 0x7FFFFFFF;
  if (p.target > 0) {
    const float c = ceilf(work / (float)p.target);
    chunk = c < (float)AT_MIN_TILES ? AT_MIN_TILES : c > 1e9f ? 1000000000 : (int)c;
  }
  int64_t before = 0, parts = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    AttendSeq s{0, 0, 0};
    int units = 0, splits = 1, cut = 0;
    if (b0 + lane < p.batch) {
      s = at_seq(p, b0 + lane);
      const int64_t blocks = ((int64_t)s.rows * G + BR - 1) / BR * p.kv_heads;
      const int tiles = (s.len + C4_TILE - 1) / C4_TILE;
      splits = tiles > chunk ? (tiles + chunk - 1) / chunk : 1;
      const int64_t all = blocks * splits;
      const int most = all > AT_UNITS_OF_SEQ ? AT_UNITS_OF_SEQ : (int)all;
      cut = splits > 1 ? most : 0;
      units = joined ? (int)blocks : most;
    }
    const int incl = wave_scan_incl(units), cut_incl = wave_scan_incl(cut);
    const bool here = unit < before + incl;
    const uint64_t found = __ballot(here);
    if (found != 0) {
      const int l = __ffsll((unsigned long long)found) - 1;
      u->b = b0 + l;
      u->seq.q0 = __builtin_amdgcn_readlane(s.q0, l);
      u->seq.rows = __builtin_amdgcn_readlane(s.rows, l);
      u->seq.len = __builtin_amdgcn_readlane(s.len, l);
      u->splits = __builtin_amdgcn_readlane(splits, l);
      u->local = (int)(unit - before - (__builtin_amdgcn_readlane(incl, l) -
                                        __builtin_amdgcn_readlane(units, l)));
      u->part = parts + __builtin_amdgcn_readlane(cut_incl, l) - __builtin_amdgcn_readlane(cut, l);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
    parts += __builtin_amdgcn_readlane(cut_incl, 63);
  }
  return false;
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
  const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
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

__device__ __forceinline__ uint32_t at_byte(uint32_t w, int i) { return (w >> (8 * i)) & 0xFFu; }

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

// The largest of the four lanes that hold a row
__device__ __forceinline__ float at_row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float at_row_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Weight of a part whose maximum is m, of M over all (both in powers of two)
__device__ __forceinline__ float at_weight(float m, float M) {
  return m == -INFINITY ? 0.f : exp2f(m - M);
}

// ---------------------------------------------------------------------------
// RT tiles of 16 rows a wave, WR waves along the rows, WT along the tokens
// ---------------------------------------------------------------------------
constexpr int at_waves(int dt, int d, int rt) {
  const int bf16 = d == 64 ? (rt == 1 ? 4 : 3) : d == 128 ? (rt == 1 ? 3 : 2) : rt == 1 ? 2 : 1;
  return dt == DT_BF16 || bf16 == 1 ? bf16 : bf16 - 1;
}
// tiles of a wave's ring in LDS, one of them being multiplied
constexpr int at_ring(int dt, int d) { return d == 64 ? 4 : d == 128 ? 3 : 2; }

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
  for (int i = 0; i < FULL; ++i) load_lds16(tile + i * 1024 + lane * 16, dst + i * 1024);
  if (lane < REST) load_lds16(tile + FULL * 1024 + lane * 16, dst + FULL * 1024);
}

template <int DT, int D, int RT, int WR, int WT>
__global__ __launch_bounds__(64 * WR * WT, at_waves(DT, D, RT)) void attend_kernel(AttendParams p) {
  constexpr int U = D / 16, M = D / 32, BR = 16 * RT * WR, TERMS = at_terms<DT>();
  constexpr int ES = DT == DT_BF16 ? 2 : 4;
  // the waves' rings of tiles, then what they join
  constexpr int NB = at_ring(DT, D), TILE = 34 * D;
  constexpr int JOIN = WT > 1 ? WT / 2 * WR * RT * (U * 1024 + 512) : 16;
  constexpr int RING = WT > 1 ? WT * WR * NB * TILE : 16;
  __shared__ __attribute__((aligned(1024))) char smem[RING > JOIN ? RING : JOIN];
  const int lane = threadIdx.x & 63, j = lane & 15, c = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % WT, wr = wave / WT;
  const int G = p.q_heads / p.kv_heads;

  AttendUnit u;
  if (!at_unit<BR>(p, blockIdx.x, false, &u)) return;
  const int R = u.seq.rows * G, blocks = (R + BR - 1) / BR;
  const int blk = blocks - 1 - u.local % blocks;     // the longest first
  const int hs = u.local / blocks, split = hs % u.splits, h = hs / u.splits;

  // rows, their last visible token, their queries
  const int row0 = blk * BR + wr * RT * 16;
  const int shift = u.seq.len - u.seq.rows;
  auto last_of = [&](int r) { return p.causal ? shift + r / G : u.seq.len - 1; };
  const int end_row = row0 + 16 * RT < R ? row0 + 16 * RT : R;
  const int block_end = blk * BR + BR < R ? blk * BR + BR : R;
  int last[RT];
  u32x4_t q[RT][M][TERMS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + j;
    last[rt] = r < R ? last_of(r) : -1;
  }
  auto load_q = [&]() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = row0 + rt * 16 + j, i = r < R ? r / G : 0;
      const char* src = p.q + (u.seq.q0 + i) * p.q_stride +
                        ((int64_t)h * G + (r < R ? r - i * G : 0)) * D * ES;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if constexpr (DT == DT_BF16) {
          q[rt][m][0] = r < R ? ld16(src + (32 * m + 8 * c) * 2) : u32x4_t{0, 0, 0, 0};
        } else {
          u32x4_t a{0, 0, 0, 0}, b{0, 0, 0, 0};
          if (r < R) {
            a = ld16(src + (32 * m + 8 * c) * 4);
            b = ld16(src + (32 * m + 8 * c) * 4 + 16);
          }
          const f32x4_t af = __builtin_bit_cast(f32x4_t, a), bf = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t w[TERMS], x[TERMS];
            at_split<DT>(af[2 * e], af[2 * e + 1], w);
            at_split<DT>(bf[2 * e], bf[2 * e + 1], x);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
              q[rt][m][k][e] = w[k];
              q[rt][m][k][2 + e] = x[k];
            }
          }
        }
      }
    }
    // (waited for here, once: the compiler would wait for every load in the loop)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int k = 0; k < TERMS; ++k) asm volatile("" : "+v"(q[rt][m][k]));
  };

  f32x4_t acc[RT][U];
  float top[RT], top_next[RT], base[RT], sum[RT];   // maximum; where it is renewed; in powers of two
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = top_next[rt] = -INFINITY;
    base[rt] = sum[rt] = 0.f;
#pragma unroll
    for (int m = 0; m < U; ++m) acc[rt][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float scl = p.scale_log2, slack = AT_SLACK / scl;

  // the part's tiles, of which this wave takes every WT-th
  const int seen = last_of(block_end - 1) + 1;       // (rows before the first token see none)
  const int block_tiles = seen > 0 ? (seen + C4_TILE - 1) / C4_TILE : 0;
  const int per = (block_tiles + u.splits - 1) / u.splits;
  const int first = split * per;
  int end = first + per < block_tiles ? first + per : block_tiles;
  if (row0 < R) {
    const int own = last_of(end_row - 1) / C4_TILE + 1;   // no less than the block's first rows'
    end = own < end ? own : end;
  } else {
    end = first;
  }
  const int full = row0 < R ? last_of(row0) : -1;    // every row sees the tokens up to here
  const int tiles_log2 = p.page_log2 - 5;
  // (scalar loads, which the counts of loads in flight below leave out)
  typedef const __attribute__((address_space(4))) int32_t* scalar_ptr_t;
  const scalar_ptr_t pages = (scalar_ptr_t)(uintptr_t)(p.pages + (int64_t)u.b * p.max_pages);
  auto page_of = [&](int t) { return pages[t >> tiles_log2]; };
  auto held = [&](int id) { return id >= 0 && id < p.num_pages; };
  auto tile_at = [&](int t, int id) {
    const int64_t page = held(id) ? id : 0;
    return p.cache + (((page * p.kv_heads + h) << tiles_log2) + (t & ((1 << tiles_log2) - 1))) *
                         (int64_t)(34 * D);
  };
  auto step = [&](AttendTile<D>& cur, int t, const uint8_t* tile) {
    // scores of 32 tokens
    f32x4_t s[RT][2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][half] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const float scale = at_scale(cur.ks[half][m / 4], m % 4);
        u32x4_t k;
#pragma unroll
        for (int b = 0; b < 4; ++b) k[b] = c4_pair(cur.k[half][m], scale, b);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int x = TERMS - 1; x >= 0; --x)
            s[rt][half] = mfma_chunk<DT_BF16>(k, q[rt][m][x], s[rt][half]);
      }
    }
    // tokens that a row does not see, and, where a block of v is not finite (or
    // behind the last token, where anything may be), values that must not meet the
    // weight 0
    const int t0 = t * C4_TILE;
    const bool edge = t0 + C4_TILE - 1 > full;
    if (edge) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (t0 + 16 * half + 4 * c + i > last[rt]) s[rt][half][i] = -INFINITY;
    }
    // (a byte of 255: its complement is 0)
    const uint32_t inv0 = ~cur.vs[0], inv1 = ~cur.vs[1];
    const uint32_t holes = (((inv0 - 0x01010101u) & ~inv0) | ((inv1 - 0x01010101u) & ~inv1)) &
                           0x80808080u;
    uint32_t nan_rows[RT];
    const bool careful = __any(holes != 0 || t0 + C4_TILE > u.seq.len);
    if (careful) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) nan_rows[rt] = 0;
      for (int g = 0; g < M; ++g) {
        uint32_t vs[2];
        at_load_words(vs, tile + 33 * D + g * 32 + c * 8);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const bool hole = at_byte(vs[x / 4], x % 4) == C4_NAN;
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
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int token = t0 + 4 * c + x % 4 + 16 * (x / 4);
        if (token >= u.seq.len || at_byte(cur.vs[x / 4], x % 4) == C4_NAN) {
          const int bit = 8 * (x % 4);
          cur.vs[x / 4] = (cur.vs[x / 4] & ~(0xFFu << bit)) | (127u << bit);
          if constexpr (U == 4) {
            cur.v[x / 2] &= x % 2 == 0 ? 0xFFFF0000u : 0x0000FFFFu;
          } else {
#pragma unroll
            for (int w = 0; w < U / 8; ++w) cur.v[x * (U / 8) + w] = 0;
          }
        }
      }
    }
    // running maximum
    float mx[RT];
    bool grown = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mx[rt] = s[rt][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx[rt] = fmaxf(mx[rt], s[rt][e / 4][e % 4]);
      grown |= mx[rt] > top_next[rt];
    }
    if (__any(grown)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float now = fmaxf(top[rt], at_row_max(mx[rt]));
        const float b = now == -INFINITY ? 0.f : now * scl;
        const float f = top[rt] == -INFINITY ? 0.f : exp2f(base[rt] - b);
        top[rt] = now;
        top_next[rt] = now + slack;
        base[rt] = b;
        sum[rt] *= f;
#pragma unroll
        for (int m = 0; m < U; ++m) acc[rt][m] *= f;
      }
    }
    // weights
    u32x4_t w[RT][TERMS];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float e[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        e[x] = __builtin_amdgcn_exp2f(fmaf(s[rt][x / 4][x % 4], scl, -base[rt]));
        sum[rt] += e[x];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        uint32_t o[TERMS];
        at_split<DT>(e[2 * x], e[2 * x + 1], o);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) w[rt][k][x] = o[k];
      }
    }
    // outputs: byte b of a token's unit holds the lane's dims 2 b and 2 b + 1
#pragma unroll
    for (int b = 0; b < U / 2; ++b) {
      uint32_t pair[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int byte = x * (U / 2) + b;
        pair[x] = c4_pair(cur.v[byte / 4], at_scale(cur.vs[x / 4], x % 4), byte % 4);
      }
      u32x4_t lo, hi;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        lo[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x05040100u);
        hi[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], 0x07060302u);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int k = TERMS - 1; k >= 0; --k) {
          acc[rt][2 * b] = mfma_chunk<DT_BF16>(lo, w[rt][k], acc[rt][2 * b]);
          acc[rt][2 * b + 1] = mfma_chunk<DT_BF16>(hi, w[rt][k], acc[rt][2 * b + 1]);
        }
    }
  };

  int t = first + wt;
  if constexpr (WT > 1) {
    // The wave's own ring: NB - 1 tiles on their way while one is multiplied, no
    // barrier, the page of the next one ahead of them.  `bad`: bit i, the tile i turns
    // ahead is on no page.
    char* ring = smem + wave * (NB * TILE);
    uint32_t bad = 0;
    int id = t < end ? page_of(t) : 0, slot = 0;
    auto issue = [&](int x, int at) {
      at_issue<D>(tile_at(x, id), ring + at * TILE);
      bad |= (held(id) ? 0u : 1u) << (NB - 1);
      id = page_of(x + WT < end ? x + WT : x);
    };
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) {
      bad >>= 1;
      if (t + i * WT < end) issue(t + i * WT, i);
    }
    load_q();
    for (; t < end; t += WT) {
      bad >>= 1;
      if (t + (NB - 1) * WT < end) {
        issue(t + (NB - 1) * WT, slot == 0 ? NB - 1 : slot - 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 1) * at_instr<D>()) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      if ((bad & 1u) == 0) {
        AttendTile<D> cur;
        const uint8_t* tile = reinterpret_cast<const uint8_t*>(ring + slot * TILE);
        at_load(cur, tile);
        step(cur, t, tile);
      }
      slot = slot == NB - 1 ? 0 : slot + 1;
      asm volatile("" ::: "memory");
    }
    __syncthreads();   // the rings are free for the join
  } else {
    // Two tiles in registers by turns: one is multiplied while the other is on its
    // way, and the page of the one after it
    AttendTile<D> even, odd;
    if (t < end) {
      load_q();
      int id = page_of(t), next = page_of(t + WT < end ? t + WT : t);
      at_load(even, tile_at(t, id));
      while (true) {
        int after = page_of(t + 2 * WT < end ? t + 2 * WT : t);
        if (t + WT < end) at_load(odd, tile_at(t + WT, next));
        if (held(id)) step(even, t, tile_at(t, id));
        t += WT;
        if (t >= end) break;
        id = page_of(t + 2 * WT < end ? t + 2 * WT : t);
        if (t + WT < end) at_load(even, tile_at(t + WT, after));
        if (held(next)) step(odd, t, tile_at(t, next));
        t += WT;
        if (t >= end) break;
        next = id;
        id = after;
      }
    }
  }

  // the waves along the tokens join
  float ref[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] = at_row_sum(sum[rt]);
    ref[rt] = top[rt] == -INFINITY ? -INFINITY : base[rt];
  }
  if constexpr (WT > 1) {
#pragma unroll
    for (int step = WT / 2; step > 0; step >>= 1) {
      char* slot = smem + (wr * (WT / 2) + (wt & (step - 1))) * (RT * (U * 1024 + 512));
      f32x4_t* join = reinterpret_cast<f32x4_t*>(slot) + lane;
      float* ml = reinterpret_cast<float*>(slot + RT * U * 1024) + lane;
      if (wt >= step && wt < 2 * step) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          ml[rt * 128] = ref[rt];
          ml[rt * 128 + 64] = sum[rt];
#pragma unroll
          for (int m = 0; m < U; ++m) join[(rt * U + m) * 64] = acc[rt][m];
        }
      }
      __syncthreads();
      if (wt < step) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float other = ml[rt * 128], most = fmaxf(ref[rt], other);
          const float a = at_weight(ref[rt], most), b = at_weight(other, most);
          ref[rt] = most;
          sum[rt] = sum[rt] * a + ml[rt * 128 + 64] * b;
#pragma unroll
          for (int m = 0; m < U; ++m) acc[rt][m] = acc[rt][m] * a + join[(rt * U + m) * 64] * b;
        }
      }
      if (step > 1) __syncthreads();
    }
    if (wt != 0) return;
  }

  // a lane holds dims 4 c u .. 4 c u + 4 u - 1 of its rows
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = row0 + rt * 16 + j;
    if (r >= R) continue;
    if (u.splits > 1) {
      const int64_t at = (u.part + u.local) * BR + (r - blk * BR);
      float* dst = p.part + at * D + 4 * c * U;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < U; m += 4)
          *reinterpret_cast<f32x4_t*>(dst + i * U + m) =
              f32x4_t{acc[rt][m][i], acc[rt][m + 1][i], acc[rt][m + 2][i], acc[rt][m + 3][i]};
      if (c == 0) {
        float* ml = p.part + (int64_t)2 * p.target * BR * D + at * 2;
        ml[0] = ref[rt];
        ml[1] = sum[rt];
      }
      continue;
    }
    const float inv = sum[rt] == 0.f ? 0.f : 1.f / sum[rt];
    char* dst = p.out + (int64_t)(u.seq.q0 + r / G) * p.out_stride + ((int64_t)h * G + r % G) * D * ES + 4 * c * U * ES;
    float o[4 * U];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int m = 0; m < U; ++m) o[i * U + m] = acc[rt][m][i] * inv;
#pragma unroll
    for (int x = 0; x < 4 * U * ES / 16; ++x) {
      u32x4_t v;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (DT == DT_BF16) v[k] = at_pack(o[8 * x + 2 * k], o[8 * x + 2 * k + 1]);
        else v[k] = as_u32(o[4 * x + k]);
      }
      st16(dst + 16 * x, v);
    }
  }
}

// Joins the parts of a row's keys: a workgroup a row and query head.
template <int DT, int D, int BR>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendParams p) {
  constexpr int ES = DT == DT_BF16 ? 2 : 4, L = D / 4, N = 256 / L;
  __shared__ f32x4_t accs[N][L];
  __shared__ float ms[N], ls[N];
  const int G = p.q_heads / p.kv_heads;
  const int row = blockIdx.x / p.q_heads, head = blockIdx.x % p.q_heads;   // (of all n rows)
  // the row's sequence
  const int lane64 = threadIdx.x & 63;
  int b = row;
  if (p.q_offsets != nullptr) {
    b = -1;
    for (int b0 = 0; b0 < p.batch && b < 0; b0 += 64) {
      bool mine = false;
      if (b0 + lane64 < p.batch) {
        const AttendSeq s = at_seq(p, b0 + lane64);
        mine = row >= s.q0 && row < s.q0 + s.rows;
      }
      const uint64_t found = __ballot(mine);
      if (found != 0) b = b0 + __ffsll((unsigned long long)found) - 1;
    }
    if (b < 0) return;
  }
  // the sequence's first unit, by the search that found the units
  const AttendSeq s = at_seq(p, b);
  AttendUnit u;
  int64_t first = 0;
  for (int a = lane64; a < b; a += 64) {
    const AttendSeq o = at_seq(p, a);
    first += ((int64_t)o.rows * G + BR - 1) / BR * p.kv_heads;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) first += __shfl_xor((long long)first, d, 64);
  if (!at_unit<BR>(p, first, true, &u) || u.splits <= 1) return;
  const int R = s.rows * G, blocks = (R + BR - 1) / BR;
  const int h = head / G, r = (row - s.q0) * G + head % G, blk = r / BR;
  const int l = threadIdx.x % L, g = threadIdx.x / L;
  const float* ml = p.part + (int64_t)2 * p.target * BR * D;
  float m = -INFINITY, sum = 0.f;
  f32x4_t acc{0.f, 0.f, 0.f, 0.f};
  for (int x = g; x < u.splits; x += N) {
    const int64_t unit = u.part + ((int64_t)h * u.splits + x) * blocks + (blocks - 1 - blk);
    const int64_t at = unit * BR + (r - blk * BR);
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p.part + at * D + 4 * l);
    const float om = ml[2 * at], ol = ml[2 * at + 1];
    const float most = fmaxf(m, om), a = at_weight(m, most), c = at_weight(om, most);
    m = most;
    sum = sum * a + ol * c;
    acc = acc * a + v * c;
  }
  accs[g][l] = acc;
  if (l == 0) {
    ms[g] = m;
    ls[g] = sum;
  }
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int x = 1; x < N; ++x) {
    const float most = fmaxf(m, ms[x]), a = at_weight(m, most), c = at_weight(ms[x], most);
    m = most;
    sum = sum * a + ls[x] * c;
    acc = acc * a + accs[x][l] * c;
  }
  acc *= sum == 0.f ? 0.f : 1.f / sum;
  char* dst = p.out + row * p.out_stride + ((int64_t)head * D + 4 * l) * ES;
  if constexpr (DT == DT_BF16)
    *reinterpret_cast<uint2*>(dst) = make_uint2(at_pack(acc[0], acc[1]), at_pack(acc[2], acc[3]));
  else
    *reinterpret_cast<f32x4_t*>(dst) = acc;
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------
struct AttendPlan {
  bool rows;        // many rows a sequence: the waves of a workgroup share the keys
  int block;        // rows of a unit
  int target;       // units that the cut aims at; 0: no cut
  int64_t units;    // workgroups
};

template <int DT, int D>
constexpr int at_row_tiles() {
  return DT == DT_F32 && D == 256 ? 1 : 2;
}

static AttendPlan attend_plan(int dt, int64_t n, int batch, int q_heads, int kv_heads, int d,
                              int64_t tokens) {
  const int G = q_heads / kv_heads;
  AttendPlan a{};
  a.rows = n * G > (int64_t)16 * batch;
  a.block = !a.rows ? 16 : dt == DT_F32 && d == 256 ? 64 : 128;
  const int64_t whole = (n * G / a.block + batch) * kv_heads;
  a.target = a.rows ? 240 : 1024;
  if (whole >= a.target || tokens <= AT_MIN_TILES * C4_TILE) a.target = 0;
  a.units = whole + (a.target > 0 ? a.target + 64 : 0);
  return a;
}

size_t attend_workspace(int dt, int64_t n, int batch, int q_heads, int kv_heads, int d,
                        int64_t tokens) {
  const AttendPlan a = attend_plan(dt, n, batch, q_heads, kv_heads, d, tokens);
  return (size_t)2 * a.target * a.block * (d + 2) * 4;
}

template <int DT, int D>
static hipError_t launch_attend_d(AttendParams p, hipStream_t st) {
  const AttendPlan a = attend_plan(DT, p.n, p.batch, p.q_heads, p.kv_heads, D,
                                   (int64_t)p.max_pages << p.page_log2);
  p.target = a.target;
  const dim3 grid((unsigned)((a.units + 7) / 8 * 8));
  constexpr int RT = at_row_tiles<DT, D>();
  const hipError_t e =
      a.rows ? launch_kernel(attend_kernel<DT, D, RT, 4, 1>, grid, dim3(256), 0, st, p)
             : launch_kernel(attend_kernel<DT, D, 1, 1, 4>, grid, dim3(256), 0, st, p);
  if (e != hipSuccess || a.target == 0) return e;
  const dim3 rows((unsigned)((int64_t)p.n * p.q_heads));
  return a.rows ? launch_kernel(attend_join_kernel<DT, D, 64 * RT>, rows, dim3(256), 0, st, p)
                : launch_kernel(attend_join_kernel<DT, D, 16>, rows, dim3(256), 0, st, p);
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
