// attend_rows.h -- attention of query rows over a pool's blocks (library-internal):
// tiles of keys and values in LDS, the products, the running softmax, and the
// walk over a sequence's keys, for many rows and for few.
//
// One pass over the keys with a running maximum and sum: for each tile of
// keys, s = q.k, m' = max(m, s), p = exp(scale (s - m')), and the output and
// the sum of weights so far are scaled by exp(scale (m - m')) before the
// tile's p v and p are added.  A long axis is split over workgroups; the
// parts (output not divided by its sum, maximum, sum) are joined by the same
// rule.
//
// Products run on the matrix cores as 32 x 32 x 16 bf16 with the query rows
// as columns: S^T = K Q^T and O^T = V^T P^T.  A lane then holds one query row
// (column lane % 32), so the running maximum and sum are lane values, and the
// accumulator's layout of S^T (keys 8 (r / 4) + 4 (lane / 32) + r % 4) is, with
// the keys of a contraction step taken in that order, already the operand
// layout of P^T: weights go from one product to the next without leaving the
// lane.  V^T's operand comes from V's rows in LDS by transposing reads.
//
// The query rows of a sequence that read one KV head are its tokens x the
// group of query heads, packed: a tile of 32 columns is filled by several
// heads of one token, and K and V are read once for all heads of a group.
#ifndef CLAIMKV_ATTEND_ROWS_H
#define CLAIMKV_ATTEND_ROWS_H

#include <type_traits>

#include "pool_view.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNoMax = -__builtin_inff();

// A part's maximum where the row sees keys and every score is -infinity: above
// kNoMax, which is left for rows that see nothing, and no higher than any score.
constexpr float kLeast = -3.402823466e38f;

// What a row of keys or values reads where there is none: 16 bytes of zeros
// (positions past the range: their weight is 0, and 0 x 0 adds nothing), then
// 16 bytes that are NaN in bf16 and in e4m3 (keys of a missing block).
__device__ __align__(32) const uint32_t kFill[8] = {0, 0, 0, 0, ~0u, ~0u, ~0u, ~0u};

struct Args {
  // rows
  const uint16_t* q;
  uint16_t* out;
  uint64_t q_row, q_head, out_row, out_head;
  uint32_t rows, num_seqs, group, heads;  // heads: KV heads
  const uint32_t *ids, *offsets;
  // blocks
  uint32_t max_seqs, max_blocks;
  const uint32_t *tables, *lengths, *prefix;
  uint32_t prefix_tokens;
  uint32_t bs, bs_magic, nb;
  uint32_t chunk_bytes, token_bytes;
  const uint8_t *k, *v;  // the layer's planes
  // scores
  float c;        // scale * k_scale * log2(e): weights are powers of two
  float margin;   // a maximum is followed once scores pass it by 2^8
  float v_scale;
  // parts
  uint32_t own_splits, prefix_splits, tiles;
  float* part_o;   // [row][query head][split][dim]
  float2* part_ml;  // [row][query head][split]: maximum, sum
};

// With windows, a row at position P sees P - window + 1 .. P and the first `sinks`.
struct WindowArgs : Args {
  uint32_t window, sinks;
  uint32_t room;    // positions that a table has: a row at one of them or later sees it
  float* part_sum;  // [row][query head][split]: the sum of the weights before rounding
  float* lse;       // [row][query head], or none
};

template <bool WIN>
using ArgsOf = std::conditional_t<WIN, WindowArgs, Args>;

// Which keys of a tile a row sees: the first `hi`, or with a window those of `bits`.
// part(x): of the keys from x on.
template <bool WIN>
struct Seen {
  int hi;
  __device__ __forceinline__ Seen part(int x) const { return {hi - x}; }
  __device__ __forceinline__ bool key(int x) const { return x < hi; }
  __device__ __forceinline__ bool all(int keys) const { return !(hi < keys); }
};

template <>
struct Seen<true> {
  uint64_t bits;
  __device__ __forceinline__ Seen part(int x) const { return {bits >> x}; }
  __device__ __forceinline__ bool key(int x) const { return bits >> x & 1; }
  static __device__ __forceinline__ uint64_t first(uint32_t n) { return n < 64 ? (1ull << n) - 1 : ~0ull; }
  __device__ __forceinline__ bool all(int keys) const { return !(~bits & first(keys)); }
};

// A query row of this lane.
struct Row {
  bool valid;
  uint32_t row, head;  // packed row, query head
  uint32_t limit;      // positions below it are seen
};

// What the row's results are divided by turns into: 0 for a row that sees nothing.
// One that sees keys of score -infinity alone has 0 / 0, as its formula does.
__device__ __forceinline__ float over_sum(float x, float sum, bool sees) { return sees ? x / sum : 0.0f; }

// The logarithm of a row's sum of exponentials: -infinity for one that sees
// nothing, or scores of -infinity alone.
__device__ __forceinline__ void write_lse(const WindowArgs& a, uint32_t row, uint32_t head, float m, float sum) {
  if (!a.lse) return;
  constexpr float kLn2 = 0.693147180559945309f;
  const float x = sum == 0.0f ? kNoMax : __builtin_fmaf(m, a.c, log2f(sum)) * kLn2;
  a.lse[(uint64_t)row * a.heads * a.group + head] = x;
}

// A value that all lanes of the wave have, for the scalar unit.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename T>
__device__ __forceinline__ T* uniform(T* p) {
  const uint64_t x = (uint64_t)p;
  return (T*)((uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x));
}

// Keys lo .. hi - 1 of one list of blocks.
struct Range {
  const uint32_t* list;
  uint32_t entries;
  uint32_t lo, hi;
};

// The groups of KEYS keys that a tile of rows with windows reads, each aligned to
// its size: n0 from position f0 on, of which all rows see the first `full` whole,
// then n1 from b0 on, where windows begin, then the first ones of the sequence.
// What is seen by all comes first, as the order of keys does not matter to a sum.
struct Walk {
  uint32_t f0, n0, b0, n1, full;
  uint32_t from, count;  // this split's groups
  uint32_t end;          // positions from here on are not read
};

template <uint32_t KEYS>
__device__ __forceinline__ uint32_t walk_pos(const Walk& w, uint32_t n) {
  const uint32_t x = w.from + n;
  return x < w.n0 ? w.f0 + x * KEYS : x < w.n0 + w.n1 ? w.b0 + (x - w.n0) * KEYS : (x - w.n0 - w.n1) * KEYS;
}

// Rows at positions first .. last of a sequence, each with its window and the first
// keys; `last` < 0: nothing is seen.  Of positions past the table, the first is read
// by all rows that have come so far: a wrong length cannot hold the GPU.
template <uint32_t KEYS>
__device__ __forceinline__ Walk make_walk(const WindowArgs& a, int64_t first, int64_t last, uint32_t split,
                                          uint32_t splits) {
  Walk w;
  w.end = last < 0 ? 0 : last < (int64_t)a.room ? (uint32_t)(last + 1) : a.room + 1;
  const auto begins = [&](int64_t p) { return p + 1 - a.window < (int64_t)a.room ? p + 1 - a.window : a.room; };
  const int64_t low = begins(first), high = begins(last);  // where windows begin
  const uint32_t few = a.sinks < w.end ? a.sinks : w.end;
  uint32_t n2 = (few + KEYS - 1) / KEYS;  // groups of the first keys
  const uint32_t begin = low > 0 ? (uint32_t)low / KEYS : 0;
  const uint32_t groups = w.end / KEYS + (w.end % KEYS != 0);
  uint32_t b = begin > n2 ? begin : n2;
  b = b < groups ? b : groups;
  n2 = n2 < b ? n2 : b;
  // from `f` on, all rows' windows have begun; below `t`, none has ended
  uint32_t f = high > 0 ? (uint32_t)(high / KEYS + (high % KEYS != 0)) : 0;
  const int64_t least = first + 1 < (int64_t)w.end ? first + 1 : w.end;
  const uint32_t t = least > 0 ? (uint32_t)(least / KEYS) : 0;
  f = f > b ? f : b;
  if (f >= t) f = b;
  w.full = f < t && high <= (int64_t)f * KEYS ? t - f : 0;
  w.f0 = f * KEYS;
  w.n0 = groups - f;
  w.b0 = b * KEYS;
  w.n1 = f - b;
  const uint32_t all = w.n0 + w.n1 + n2;
  uint32_t share = (all + splits - 1) / splits;
  w.from = share * split < all ? share * split : all;
  w.count = all - w.from < share ? all - w.from : share;
  w.full = w.full > w.from ? w.full - w.from : 0;
  w.full = w.full < w.count ? w.full : w.count;
  w.f0 = uniform(w.f0);
  w.n0 = uniform(w.n0);
  w.b0 = uniform(w.b0);
  w.n1 = uniform(w.n1);
  w.full = uniform(w.full);
  w.from = uniform(w.from);
  w.count = uniform(w.count);
  w.end = uniform(w.end);
  return w;
}

__device__ __forceinline__ void split_pos(const Args& a, uint32_t pos, uint32_t* block,
                                          uint32_t* token) {
  // floor(pos / bs): the multiplier is rounded down, so the quotient is right
  // or one too small for every 32-bit position
  uint32_t q = __umulhi(pos, a.bs_magic), r = pos - q * a.bs;
  if (r >= a.bs) {
    ++q;
    r -= a.bs;
  }
  *block = q;
  *token = r;
}

// In place of a row's byte in a plane: nothing is there (its weight is 0), or
// its block is missing.
constexpr uint64_t kZeros = ~0ull, kNaNs = ~1ull;

// ------------------------------------------------------------ tiles in LDS
//
// A tile is whole rows one after another, the 16-byte chunks of a row
// exchanged by an exclusive or with bits of the row's number, so that every
// way of reading it touches all banks equally.

// Rows of D bf16 values read by 32 x 32 products: K by 32 rows x one chunk, V
// by 8 rows x 64 bytes.
template <int D>
struct WideSwizzle {
  static __device__ __forceinline__ constexpr uint32_t k(uint32_t row) {
    return D == 128 ? row & 15 : (row >> 1) & 7;
  }
  static __device__ __forceinline__ constexpr uint32_t v(uint32_t row) {
    return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
  }
};

// Rows of BYTES bytes, as they are in the pool, read by 16 x 16 products: 16
// rows x 32 or 64 bytes.
template <int BYTES>
struct NarrowSwizzle {
  static __device__ __forceinline__ constexpr uint32_t k(uint32_t row) {
    return BYTES == 256 ? row & 15 : BYTES == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
  }
  static __device__ __forceinline__ constexpr uint32_t v(uint32_t row) { return k(row); }
};

typedef const __attribute__((address_space(3))) u32x4 lds_words;
typedef const __attribute__((address_space(3))) u32x2 lds_pair;

__device__ __forceinline__ uint32_t lds_address(const uint8_t* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p;
}

// A wave's 64 lanes copy 16 bytes each to 1024 bytes of LDS from `to` (the same
// on all lanes).  Nothing waits for it here: wait_loads() does.  (The builtin
// makes the compiler wait for the copy at the next LDS read of any buffer.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is named so that no value is kept in it
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(from), "s"(to)
               : "memory", "m0");
}

// The same from one base for the wave and an offset for each lane.
__device__ __forceinline__ void copy_to_lds(const uint8_t* base, uint32_t lane_offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(lane_offset), "s"(base), "s"(to)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Eight e4m3 bytes to eight bf16 values: every one is exact.
__device__ __forceinline__ u32x4 widen(uint32_t a, uint32_t b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const auto two = [](uint32_t w, auto hi) {
    const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, decltype(hi)::value);
    return __builtin_bit_cast(uint32_t, x);
  };
  return u32x4{two(a, std::false_type{}), two(a, std::true_type{}), two(b, std::false_type{}),
               two(b, std::true_type{})};
}

// Moves KEYS rows of BYTES bytes of one plane into a tile with THREADS threads,
// straight to LDS; or (WIDEN) e4m3 rows into registers by issue(), and widened
// to bf16 into LDS by land().
//
// WITHIN says which rows surely lie in one block of the cache, so that they
// share a table entry and a base address on the scalar unit: those of one
// load instruction of a wave (4 of 256 bytes to 16 of 64: their number divides
// the block size), or all of a wave's tile (KEYS divides it); otherwise each
// lane has its own.  16384 causal tokens, 32 heads over 8 of 128, blocks of 16:
// 2.40 ms with lanes of their own, 2.01 ms with loads.
enum Within : int { kLanes = 0, kLoads = 1, kTiles = 2 };

template <int BYTES, bool WIDEN, int KEYS, int THREADS, Within WITHIN, typename Swizzle>
struct Stage {
  static constexpr int kRowLanes = BYTES / 16;  // lanes of one row
  static constexpr int kWaveRows = 64 / kRowLanes;
  static constexpr int kRows = THREADS / kRowLanes;  // rows of one step
  static constexpr int kSteps = KEYS / kRows ? KEYS / kRows : 1;
  static constexpr int kLooks = WITHIN == kTiles ? 1 : kSteps;  // table entries of a tile
  static constexpr bool kScalar = WITHIN != kLanes;
  static_assert(WIDEN || KEYS % kRows == 0, "tiles are filled by whole steps");
  static_assert(WITHIN != kTiles || (THREADS == 64 && !WIDEN), "a wave's own tile");

  struct Held {  // e4m3 bytes on their way
    u32x4 r[WIDEN ? kSteps : 1];
  };

  // The rows of one tile, a wave's first of each look or a lane's own: where
  // they are in the list of blocks, and its entries once they are read.
  struct Rows {
    uint32_t at[kLooks], token[kLooks], entry[kLooks];
  };

  // Where they are in a plane.
  struct Places {
    uint64_t byte[kLooks];
    uint32_t entry[kLooks];
    uint32_t left;  // rows of the tile that the range has
  };

  uint32_t t, wave, k_off, v_off;  // a lane's place in its wave's rows, or in its row
  uint32_t step;                   // bytes from one step's rows to the next (kTiles)

  __device__ __forceinline__ Stage(const Args& a, uint32_t thread) : t(thread) {
    wave = THREADS == 64 ? 0 : uniform(thread >> 6);
    const uint32_t row = thread / kRowLanes, chunk = thread % kRowLanes;
    k_off = (WIDEN ? chunk : chunk ^ Swizzle::k(row)) * 16;
    v_off = (WIDEN ? chunk : chunk ^ Swizzle::v(row)) * 16;
    if (kScalar) {
      k_off += row % kWaveRows * a.token_bytes;
      v_off += row % kWaveRows * a.token_bytes;
    }
    step = kWaveRows * a.token_bytes;
  }

  __device__ __forceinline__ uint32_t row(int i) const {
    return i * kRows + (kScalar ? wave * kWaveRows : t / kRowLanes);
  }

  __device__ __forceinline__ void first(const Args& a, uint32_t pos, Rows& r) const {
#pragma unroll
    for (int i = 0; i < kLooks; ++i) {
      split_pos(a, pos + row(i), &r.at[i], &r.token[i]);
      if (kScalar) {
        r.at[i] = uniform(r.at[i]);
        r.token[i] = uniform(r.token[i]);
      }
    }
  }

  // The rows `keys` positions on: add_blocks = keys / bs, add_tokens = keys % bs.
  __device__ __forceinline__ void next(const Args& a, uint32_t add_blocks, uint32_t add_tokens,
                                       Rows& r) const {
#pragma unroll
    for (int i = 0; i < kLooks; ++i) {
      r.token[i] += add_tokens;
      const bool over = r.token[i] >= a.bs;
      r.token[i] = over ? r.token[i] - a.bs : r.token[i];
      r.at[i] += add_blocks + over;
    }
  }

  __device__ __forceinline__ void look(const Range& g, Rows& r) const {
    typedef const __attribute__((address_space(4))) uint32_t* scalar_list;
#pragma unroll
    for (int i = 0; i < kLooks; ++i) {
      r.entry[i] = CLAIM_NONE;
      if (kScalar) {
        // past the list: its last entry is read in its place
        const uint32_t at = r.at[i] < g.entries ? r.at[i] : g.entries - 1;
        const uint32_t entry = ((scalar_list)g.list)[at];
        r.entry[i] = r.at[i] < g.entries ? entry : CLAIM_NONE;
      } else if (r.at[i] < g.entries) {
        r.entry[i] = g.list[r.at[i]];
      }
    }
  }

  __device__ __forceinline__ Places place(const Args& a, const Rows& r, uint32_t left) const {
    Places p;
    p.left = left;
#pragma unroll
    for (int i = 0; i < kLooks; ++i) {
      p.entry[i] = r.entry[i] < a.nb ? r.entry[i] : CLAIM_NONE;
      p.byte[i] = (uint64_t)r.entry[i] * a.chunk_bytes + (uint64_t)r.token[i] * a.token_bytes;
    }
    return p;
  }

  template <bool KEY>
  __device__ __forceinline__ void issue(const uint8_t* plane, const Places& p, uint8_t* tile,
                                        Held& held) const {
    bool fine = p.left >= KEYS;  // every row is in the range and has a block
#pragma unroll
    for (int i = 0; i < kLooks; ++i) fine &= p.entry[i] != CLAIM_NONE;
    const bool all = kScalar ? fine : __all(fine);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (WIDEN && KEYS < kRows && i * kRows + t / kRowLanes >= KEYS) break;
      const int l = WITHIN == kTiles ? 0 : i;
      const uint32_t to = lds_address(tile) + i * THREADS * 16 + wave * 1024;
      // the first row of a step has a swizzle of its own where a step is less than 16 rows
      uint32_t off = KEY ? k_off : v_off;
      if (!WIDEN) off ^= (KEY ? Swizzle::k(i * kRows) : Swizzle::v(i * kRows)) * 16;
      if (WITHIN == kTiles) off += i * step;
      const uint8_t* base = plane + p.byte[l];
      if (all) {
        if constexpr (WIDEN)
          held.r[i] = *(const u32x4*)((kScalar ? uniform(base) : base) + off);
        else if constexpr (kScalar)
          copy_to_lds(uniform(base), off, to);
        else
          copy_to_lds(base + off, to);
      } else {
        const bool there = i * kRows + t / kRowLanes < p.left;
        const uint8_t* from = there && p.entry[l] != CLAIM_NONE
                                  ? base + off
                                  : (const uint8_t*)kFill + (KEY && there ? 16 : 0);
        if constexpr (WIDEN)
          held.r[i] = *(const u32x4*)from;
        else
          copy_to_lds(from, to);
      }
    }
  }

  template <bool KEY>
  __device__ __forceinline__ void land(const Held& held, uint8_t* tile) const {
    if constexpr (WIDEN) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const uint32_t row = i * kRows + t / kRowLanes, chunk = 2 * (t % kRowLanes);
        if (KEYS < kRows && row >= KEYS) break;
        const uint32_t x = KEY ? Swizzle::k(row) : Swizzle::v(row);
        uint8_t* to = tile + row * BYTES * 2;
        *(u32x4*)(to + (chunk ^ x) * 16) = widen(held.r[i].x, held.r[i].y);
        *(u32x4*)(to + ((chunk + 1) ^ x) * 16) = widen(held.r[i].z, held.r[i].w);
      }
    }
  }
};

// Everything that this wave has asked memory for has arrived.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
}

// All but the last N copies to LDS have arrived.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N < 64, "");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0F70);
  asm volatile("" ::: "memory");
}

// This wave's LDS reads and writes are done.
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------- one wave's 32 rows

__device__ __forceinline__ float across_halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float across_halves_add(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D>
struct Wave {
  bf16x8 q[D / 16];
  f32x16 o[D / 32];
  float m, l;  // the maximum is the row's; the sum this lane's half of the keys
  uint32_t k_lane, v_lane;  // this lane's place in a tile of K, of V

  __device__ __forceinline__ void start(const Args& a, const Row& r) {
    const uint32_t h = (threadIdx.x >> 5) & 1;
    const uint16_t* src = a.q + r.row * a.q_row + r.head * a.q_head + 8 * h;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      u32x4 w = {0, 0, 0, 0};
      if (r.valid) w = *(const u32x4*)(src + 16 * t);
      q[t] = __builtin_bit_cast(bf16x8, w);
    }
#pragma unroll
    for (int j = 0; j < D / 32; ++j) o[j] = f32x16{};
    m = kNoMax;
    l = 0;
    const uint32_t lane = threadIdx.x & 63, row = lane & 31;
    k_lane = row * D * 2 + ((h ^ WideSwizzle<D>::k(row)) << 4);
    const uint32_t key = 4 * h + ((lane & 15) >> 2);
    v_lane = key * D * 2 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ WideSwizzle<D>::v(key)) << 4) +
             (lane & 1) * 8;
  }

  // V^T's operand: 32 values of D from 32 j, keys in the order of P^T's
  static __device__ __forceinline__ bf16x8 v_operand(uint32_t at, int u, int t, int j) {
    typedef __attribute__((address_space(3))) s16x4* p4;
    const uint32_t x = (at ^ (j << 6)) + (32 * u + 16 * t) * D * 2;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)x);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(x + 8 * D * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }

  // Scores of a tile of 32 U keys.
  template <int U>
  __device__ __forceinline__ void scores(const uint8_t* lk, f32x16 (&s)[U]) const {
    // chunk 2 t + h of row lane % 32: the swizzle leaves t an exclusive or
    uint32_t at = lds_address(lk) + k_lane;
    asm volatile("" : "+v"(at));  // eight exclusive ors a tile, not eight registers all along
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] = f32x16{};
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4 w = *(const lds_words*)(uintptr_t)((at ^ (t << 5)) + 32 * u * D * 2);
        s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), q[t], s[u], 0, 0, 0);
      }
  }

  // Takes out the keys of the tile that the row does not see.
  template <int U, bool WIN>
  __device__ __forceinline__ void mask(f32x16 (&s)[U], const Seen<WIN>& seen) const {
    const int h = (threadIdx.x >> 5) & 1;
    const Seen<WIN> mine = seen.part(4 * h);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[u][r] = mine.key(32 * u + 8 * (r / 4) + r % 4) ? s[u][r] : kNoMax;
  }

  // Weights of a tile, and the running maximum and sum.
  template <int U>
  __device__ __forceinline__ void weights(const Args& a, const f32x16 (&s)[U], bf16x8 (&p)[U][2]) {
    float top = kNoMax;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
    top = across_halves_max(top);
    // the maximum in use is only followed once scores pass it by 2^8: weights
    // up to 256 keep their precision, and most tiles scale nothing
    if (__any(top > m + a.margin || m == kNoMax)) {
      const float to = fmaxf(m, top);
      const float base = to == kNoMax ? 0.0f : to;
      const float f = __builtin_amdgcn_exp2f((m - base) * a.c);
      l *= f;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) o[j] *= f;
      m = to;
    }
    const float mc = m == kNoMax ? 0.0f : m * a.c;
    float sum[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        // the sum takes the weight before it is rounded: the rounded one costs
        // 6 % of the kernel's time, for an error of 2.1e-3 in place of 2.2e-3
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][r], a.c, -mc));
        sum[r & 1] += e;
        p[u][r / 8][r % 8] = (__bf16)e;
      }
    l += sum[0] + sum[1];
  }

  template <int U>
  __device__ __forceinline__ void values(const uint8_t* lv, const bf16x8 (&p)[U][2]) {
    uint32_t at = lds_address(lv) + v_lane;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(at, u, t, j), p[u][t], o[j], 0, 0, 0);
  }

  // values() of one tile of 64 keys, then scores() of another: operands are
  // read from LDS four products ahead of their use.
  __device__ __forceinline__ void multiply(const uint8_t* lv, const bf16x8 (&p)[2][2], const uint8_t* lk,
                                           f32x16 (&s)[2]) {
    values<2>(lv, p);
    scores<2>(lk, s);
    constexpr int kV = D / 32, kAll = D / 8, kRead = 0x100, kMul = 0x8;  // products of a step of V; of K
    __builtin_amdgcn_sched_group_barrier(kRead, 8, 0);
#pragma unroll
    for (int i = 0; i < 4 * kV - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMul, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
    }
#pragma unroll
    for (int i = 0; i < kAll; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMul, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMul, 4, 0);
  }

  // A whole tile of which the lane's row sees the keys `seen`.
  template <int U, bool WIN>
  __device__ __forceinline__ void tile(const Args& a, const uint8_t* lk, const uint8_t* lv,
                                       const Seen<WIN>& seen, bool bad = true) {
    f32x16 s[U];
    bf16x8 p[U][2];
    scores<U>(lk, s);
    const bool masked = __any(!seen.all(32 * U));
    if (masked) mask<U>(s, seen);
    weights<U>(a, s, p);
    if (masked && bad && nonfinite<U>(lv))
      values_seen<U>(lv, p, seen);
    else
      values<U>(lv, p);
  }

  // Whether the tile of V holds an infinity or a NaN: a weight of 0 does not
  // take it out of the product.
  static __device__ __forceinline__ bool nonfinite(u32x4 w) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
    return bad;
  }

  template <int U>
  __device__ __forceinline__ bool nonfinite(const uint8_t* lv) const {
    bool bad = false;
#pragma unroll 1
    for (uint32_t at = (threadIdx.x & 63) * 16; at < 32 * U * D * 2; at += 1024)
      bad |= nonfinite(*(const u32x4*)(lv + at));
    return __any(bad);
  }

  // values() where V holds infinities or NaN that some rows do not see: one
  // key's product at a time, kept by the rows that see the key.
  template <int U, bool WIN>
  __device__ __forceinline__ void values_seen(const uint8_t* lv, const bf16x8 (&p)[U][2],
                                              const Seen<WIN>& seen) {
    const uint32_t at = lds_address(lv) + v_lane, h = (threadIdx.x >> 5) & 1;
#pragma unroll 1
    for (uint32_t key = 0; key < 32 * U; ++key) {
      // the key's element of an operand: half (key / 4) % 2, place (key / 8) % 2 * 4 + key % 4
      const uint32_t place = (key >> 3 & 1) * 4 + (key & 3);
      const uint32_t half = (key >> 2 & 1) == h ? 0xFFFFu << (place & 1) * 16 : 0;
      u32x4 only, w = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) only[i] = place / 2 == (uint32_t)i ? half : 0;
#pragma unroll
      for (int x = 0; x < 2 * U; ++x)
        if (key / 16 == (uint32_t)x) w = __builtin_bit_cast(u32x4, p[x / 2][x % 2]);
      const bf16x8 weight = __builtin_bit_cast(bf16x8, w & only);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const u32x4 v = __builtin_bit_cast(u32x4, v_operand(at + key / 16 * 16 * D * 2, 0, 0, j)) & only;
        const f32x16 with = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), weight, o[j], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = seen.key((int)key) ? with[r] : o[j][r];
      }
    }
  }

  // The rows' parts for the joining kernel: through LDS of the wave's own (32
  // rows of D floats), so that whole rows are stored at a time.
  template <bool WIN>
  __device__ __forceinline__ void finish_part(const ArgsOf<WIN>& a, const Row& r, bool sees, uint32_t split,
                                              uint32_t splits, uint8_t* lds) {
    const uint32_t lane = threadIdx.x & 63, h = lane >> 5, row = lane & 31;
    const float sum = across_halves_add(l);
    uint64_t at = ((uint64_t)r.row * a.heads * a.group + r.head) * splits + split;
    if (r.valid && h == 0) a.part_ml[at] = float2{sees ? fmaxf(m, kLeast) : m, sum};
    if constexpr (WIN)
      if (r.valid && h == 0) a.part_sum[at] = sum;
    if (!r.valid || sum == 0.0f) at = ~0ull;
    constexpr uint32_t kChunks = D / 4;  // 16-byte chunks of a row, exchanged by its number
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t chunk = (8 * j + 2 * g + h) ^ (row & (kChunks - 1));
        *(f32x4*)(lds + (row * kChunks + chunk) * 16) =
            f32x4{o[j][4 * g], o[j][4 * g + 1], o[j][4 * g + 2], o[j][4 * g + 3]};
      }
    wait_lds();
#pragma unroll
    for (uint32_t i = 0; i < 32 * kChunks / 64; ++i) {
      const uint32_t x = i * 64 + lane, from = x / kChunks, chunk = x % kChunks;
      const f32x4 w = *(const f32x4*)(lds + (from * kChunks + (chunk ^ (from & (kChunks - 1)))) * 16);
      const uint64_t to = (uint64_t)__shfl((uint32_t)(at >> 32), from) << 32 | __shfl((uint32_t)at, from);
      if (to != ~0ull) *(f32x4*)(a.part_o + to * D + chunk * 4) = w;
    }
  }

  // The rows' results.
  template <bool WIN>
  __device__ __forceinline__ void finish(const ArgsOf<WIN>& a, const Row& r, bool sees) {
    const uint32_t h = (threadIdx.x >> 5) & 1;
    const float sum = across_halves_add(l);
    if (!r.valid) return;
    if constexpr (WIN)
      if (h == 0) write_lse(a, r.row, r.head, m, sum);
    const float f = over_sum(a.v_scale, sum, sees);
    uint16_t* dst = a.out + r.row * a.out_row + r.head * a.out_head + 4 * h;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (__bf16)(o[j][4 * g + i] * f);
        *(bf16x4*)(dst + 32 * j + 8 * g) = w;
      }
  }
};

// ------------------------------------------------------------- work items

// A tile of M packed query rows (token x query head of the group) that read
// the same keys, and one split's share of those keys: all of it the wave's.
struct Tile {
  bool prefix, any;    // any: the tile has rows
  uint32_t first, n;   // own: the sequence's first row and how many it has
  uint32_t x0, all;    // the tile's first packed row, and how many there are
  int64_t len;         // own: the sequence's tokens
  uint32_t kv_head;
  Range range;
  Walk walk;  // with windows, in place of the range's positions
};

// The last sequence whose tiles start at or before `tile`.  Sequence s starts
// at tile floor(first row x group / M) + s: an ascending bound that leaves
// every sequence the tiles it needs.
template <int M>
__device__ __forceinline__ uint32_t first_tile(const Args& a, uint32_t s) {
  return a.offsets[s] * a.group / M + s;  // rows x group fits 32 bits
}

template <int M>
__device__ __forceinline__ uint32_t find_tile(const Args& a, uint32_t tile) {
  uint32_t lo = 0, hi = a.num_seqs;
  const uint32_t lane = threadIdx.x & 63;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64, s = lo + lane * step;
    const uint64_t m = __ballot(s < hi && first_tile<M>(a, s) <= tile);
    lo += (m ? 63u - (uint32_t)__builtin_clzll(m) : 0u) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return uniform(lo);
}

// The item `place` where tiles of longer sequences come before those of shorter
// ones, and a sequence's late tiles, which see the most, before its early ones:
// a workgroup that starts late has little left to do.  A lane holds a sequence
// and counts the tiles of those before it.  Ragged prompts of up to 1500 tokens
// behind up to 4000, 28 query heads over 4 of 128: 8 of them 302 us so and 320 us
// in the order they come in, 12 of them in e4m3 331 and 342 us.
constexpr uint32_t kOrdered = 64;  // sequences at most

struct Ordered {
  bool any;
  uint32_t part, first, n, id, len;
};

template <int M>
__device__ __forceinline__ Ordered ordered_tile(const Args& a, uint32_t place) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t first = 0, n = 0, id = 0, len = 0;
  if (lane < a.num_seqs) {
    first = a.offsets[lane];
    n = a.offsets[lane + 1] - first;
    id = a.ids ? a.ids[lane] : lane;
    // offsets that run backwards or past the rows give the sequence none
    if (first > a.rows || n > a.rows - first) n = 0;
    if (id < a.max_seqs) len = a.lengths[id];
  }
  const uint32_t mine = (n * a.group + M - 1) / M;
  // one number decides: the length (beyond 2^26 all are alike), then the lane
  const uint32_t key = (len < 1u << 26 ? len : (1u << 26) - 1) << 6 | (63 - lane);
  uint32_t before = 0;
  for (uint32_t s0 = 0; s0 < a.num_seqs; s0 += 8) {
#pragma unroll
    for (uint32_t s = s0; s < s0 + 8; ++s) {  // lanes without a sequence have no tiles
      const uint32_t tiles = __builtin_amdgcn_readlane(mine, s);
      before += (uint32_t)__builtin_amdgcn_readlane(key, s) > key ? tiles : 0;
    }
  }
  const uint64_t m = __ballot(place - before < mine);
  const uint32_t s = m ? (uint32_t)__builtin_ctzll(m) : 0;
  Ordered r;
  r.any = m != 0;
  r.part = __builtin_amdgcn_readlane(before + mine, s) - 1 - place;
  r.first = __builtin_amdgcn_readlane(first, s);
  r.n = __builtin_amdgcn_readlane(n, s);
  r.id = __builtin_amdgcn_readlane(id, s);
  r.len = __builtin_amdgcn_readlane(len, s);
  return r;
}

// ORDERED: `tile` is a place in the order above where there is one.
template <int M, bool ORDERED, uint32_t KEYS, bool WIN>
__device__ __forceinline__ Tile make_tile(const ArgsOf<WIN>& a, bool prefix, uint32_t tile, uint32_t split,
                                          uint32_t splits, uint32_t kv_head, uint32_t align) {
  Tile it;
  it.prefix = prefix;
  it.kv_head = kv_head;
  int64_t top;  // what the tile's last row sees
  uint32_t lo = 0;
  if (prefix) {
    it.first = it.n = 0;
    it.len = 0;
    it.x0 = tile * M;
    it.all = a.rows * a.group;
    it.any = it.x0 < it.all;
    it.range.list = a.prefix;
    it.range.entries = a.prefix_tokens / a.bs;
    top = a.prefix_tokens;
  } else {
    uint32_t part, id, len;
    if (ORDERED && a.offsets && a.num_seqs <= kOrdered) {
      const Ordered r = ordered_tile<M>(a, tile);
      it.any = r.any;
      it.first = r.first;
      it.n = r.n;
      part = r.part;
      id = r.id;
      len = r.len;
    } else {
      if (ORDERED) tile = a.tiles - 1 - tile;  // late rows first
      uint32_t s;
      if (a.offsets) {
        s = find_tile<M>(a, tile);
        const uint32_t from = a.offsets[s], start = first_tile<M>(a, s);
        it.first = from;
        it.n = a.offsets[s + 1] - from;
        part = tile - start;
        // offsets that run backwards or past the rows give the sequence none
        it.any = tile >= start && from <= a.rows && it.n <= a.rows - from;
      } else {
        const uint32_t per = (a.group + M - 1) / M;
        s = per == 1 ? tile : tile / per;
        part = tile - s * per;
        it.first = s;
        it.n = 1;
        it.any = s < a.num_seqs;
        if (!it.any) s = 0;
      }
      id = a.ids ? a.ids[s] : s;
      len = id < a.max_seqs ? a.lengths[id] : 0;
    }
    it.all = it.any ? it.n * a.group : 0;
    it.any = it.any && part <= it.all / M;
    it.x0 = it.any ? part * M : 0;
    it.any = it.any && it.x0 < it.all;
    it.len = len;
    it.range.list = a.tables + (uint64_t)(id < a.max_seqs ? id : 0) * a.max_blocks;
    it.range.entries = a.max_blocks;
    lo = a.prefix_tokens;
    const uint32_t last = it.x0 + M < it.all ? it.x0 + M : it.all;
    top = it.any ? it.len - it.n + (last + a.group - 1) / a.group : 0;
  }
  if constexpr (WIN) {
    const int64_t first = it.any ? it.len - it.n + it.x0 / a.group : -1;
    it.walk = make_walk<KEYS>(a, first, top - 1, split, splits);
    it.range.list = uniform(it.range.list);
    it.range.entries = uniform(it.range.entries);
    return it;
  }
  // a row that sees a position past the table is NaN whatever else it sees:
  // one such position is enough, and a wrong length cannot hold the GPU
  uint64_t end = (uint64_t)a.max_blocks * a.bs;
  end = end > a.prefix_tokens ? end : a.prefix_tokens;
  end = end < 0xFFFFF000u ? end : 0xFFFFF000u;
  if (top > (int64_t)end + 1) top = (int64_t)end + 1;
  // this split's share of the keys from lo to the last row's limit
  const uint32_t keys = top > (int64_t)lo ? (uint32_t)(top - lo) : 0;
  uint32_t share = keys, from = 0;
  if (splits > 1) {
    share = (uint32_t)(((uint64_t)keys + splits - 1) / splits + align - 1) / align * align;
    from = (uint64_t)share * split < keys ? share * split : keys;
  }
  const uint32_t to = keys - from < share ? keys : from + share;
  it.range.lo = uniform(lo + from);
  it.range.hi = uniform(lo + to);
  it.range.list = uniform(it.range.list);
  it.range.entries = uniform(it.range.entries);
  return it;
}

// Row r of the tile.
__device__ __forceinline__ Row row_at(const Args& a, const Tile& it, uint32_t r) {
  Row row;
  const uint32_t x = it.x0 + r;
  row.valid = it.any && x < it.all;
  row.row = row.head = row.limit = 0;
  if (!row.valid) return row;
  uint32_t i = x / a.group, n = it.n;
  row.head = it.kv_head * a.group + (x - i * a.group);
  row.row = it.first + i;
  int64_t len = it.len;
  if (it.prefix) {
    uint32_t s = row.row;
    n = 1;
    i = 0;
    if (a.offsets) {
      uint32_t lo = 0, hi = a.num_seqs;
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.offsets[mid] <= row.row) lo = mid; else hi = mid;
      }
      s = lo;
      n = a.offsets[s + 1] - a.offsets[s];
      i = row.row - a.offsets[s];
    }
    const uint32_t id = a.ids ? a.ids[s] : s;
    len = id < a.max_seqs ? a.lengths[id] : 0;
  }
  int64_t limit = len - n + i + 1;
  if (it.prefix && limit > a.prefix_tokens) limit = a.prefix_tokens;
  row.limit = limit > 0 ? (uint32_t)(limit < 0xFFFFFFFF ? limit : 0xFFFFFFFF) : 0;
  return row;
}

// The most and the least that valid rows of `lanes` neighbouring lanes see.
__device__ __forceinline__ void seen_by_wave(const Row& row, int lanes, uint32_t* most, uint32_t* least) {
  uint32_t hi = row.valid ? row.limit : 0, lo = row.valid ? row.limit : ~0u;
  for (int d = 1; d < lanes; d <<= 1) {
    const uint32_t x = __shfl_xor(hi, d), y = __shfl_xor(lo, d);
    hi = x > hi ? x : hi;
    lo = y < lo ? y : lo;
  }
  *most = uniform(hi);
  *least = uniform(lo);
}

__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);  // no work of one phase moves into the other
  wait_lds();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The weights are made here, whatever the compiler thinks of later places.
__device__ __forceinline__ void hold(bf16x8 (&p)[2][2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 w = __builtin_bit_cast(u32x4, p[i / 2][i % 2]);
    asm volatile("" : "+v"(w));
    p[i / 2][i % 2] = __builtin_bit_cast(bf16x8, w);
  }
}

// Which of the `keys` positions from `pos` on the row sees.
template <bool WIN>
__device__ __forceinline__ Seen<WIN> seen_of(const ArgsOf<WIN>& a, const Row& r, uint32_t pos, uint32_t keys) {
  const auto upto = [&](uint32_t end) { return end <= pos ? 0 : end - pos < keys ? end - pos : keys; };
  if constexpr (WIN) {
    uint32_t low = r.limit > a.window ? r.limit - a.window : 0;
    low = low < a.room ? low : a.room;
    const auto below = [&](uint32_t end) { return Seen<true>::first(upto(end)); };
    return {below(r.limit) & (~below(low) | below(a.sinks))};
  } else {
    return {(int)upto(r.limit)};
  }
}

// ----------------------------------------------------------- many query rows
//
// WAVES waves of 32 rows share each tile of 64 keys.  The tiles that every row
// sees in full take two phases each: a wave multiplies (the weights of the
// tile before with V, then the queries with K), then it turns the scores into
// weights and begins the copy of a tile two further on.  Half of the waves,
// one on each SIMD, are one phase ahead of their partners on the SIMDs, so
// matrix cores and vector units are both busy all the time.  The tiles that
// some row does not see in full come last, one after another.
//
// In wave terms: M(n) reads tile n of K and n - 1 of V, W(n) makes weights of
// tile n and asks for tile n + 3 of K and n + 2 of V.  bf16 copies go to LDS and
// are waited for at the end of W(n + 1); e4m3 bytes stop in registers and land
// in W(n + 1).  A ring of four tiles: what W(n) fills was last read in M(n - 1),
// by every wave before any is in W(n), and is read first in M(n + 3), after a
// barrier that every wave reaches with its copies done.
//
// Why 256 rows and 64 keys: a wave's scores, outputs and queries fill its 256
// registers, a key comes from L2 once for 256 rows, and the ring of K and V is
// 128 KiB, one workgroup to a CU.  Bound by the matrix cores, at the clock that
// power leaves them: 16384 causal tokens, 32 query heads over 8 of 128, take 1.93
// ms, 1.14 PFLOP/s of the pairs that are seen, the matrix cores 55 % busy at 1.9
// GHz and no bank conflicts (a bf16 product of 8192 x 8192 matrices reaches 1.12
// PFLOP/s on the same card, of 16384 x 16384 1.36).

template <int D, int WAVES>
struct Many {
  static constexpr int kKeys = 64, kTile = kKeys * D * 2, kAhead = 3;
  struct Lds {
    __align__(1024) uint8_t k[(kAhead + 1) * kTile];
    __align__(1024) uint8_t v[(kAhead + 1) * kTile];
    uint32_t least[WAVES];
  };
  struct WithBad : Lds {
    uint32_t bad[2][WAVES];  // what of a tile of V each wave brought holds an infinity or a NaN
  };
};

template <int D, bool E4M3, int WAVES, Within WITHIN, bool WIN = false>
__device__ __forceinline__ void many_rows(const ArgsOf<WIN>& a, bool prefix, uint32_t b,
                                          std::conditional_t<WIN, typename Many<D, WAVES>::WithBad,
                                                             typename Many<D, WAVES>::Lds>& shared) {
  using F = Many<D, WAVES>;
  constexpr int M = WAVES * 32, kKeys = F::kKeys, kTile = F::kTile, kAhead = F::kAhead;
  using St = Stage<D * (E4M3 ? 1 : 2), E4M3, kKeys, WAVES * 64, WITHIN, WideSwizzle<D>>;
  uint8_t *const lk = shared.k, *const lv = shared.v;
  auto& least = shared.least;
  const uint32_t t = threadIdx.x;
  const uint32_t kv_head = b % a.heads;  // one head's keys stay in one die's cache where heads = 8
  b /= a.heads;
  const uint32_t splits = prefix ? a.prefix_splits : a.own_splits;
  const uint32_t split = b % splits;
  const Tile it = make_tile<M, true, kKeys, WIN>(a, prefix, b / splits, split, splits, kv_head, kKeys);
  if (!it.any) return;
  const uint64_t head_bytes = (uint64_t)kv_head * D * (E4M3 ? 1 : 2);
  const uint8_t *k = a.k + head_bytes, *v = a.v + head_bytes;
  const uint32_t lo = it.range.lo, hi = it.range.hi;
  const St st(a, t);
  typename St::Held kh, vh;
  typename St::Rows rows;
  typename St::Places kp, vp;
  const uint32_t add_blocks = kKeys / a.bs, add_tokens = kKeys % a.bs;
  const auto left = [&](uint32_t tile) {  // rows of the tile that the range has
    if constexpr (WIN) {
      const uint32_t from = walk_pos<kKeys>(it.walk, tile);
      return tile < it.walk.count && from < it.walk.end ? it.walk.end - from : 0;
    }
    const uint32_t from = lo + tile * kKeys;
    return from < hi ? hi - from : 0;
  };
  const auto next = [&](uint32_t tile, typename St::Rows& r) {  // of tile `tile`, after the one before it
    if (WIN)
      st.first(a, walk_pos<kKeys>(it.walk, tile), r);
    else
      st.next(a, add_blocks, add_tokens, r);
  };
  // copies begin before anything else: tiles 0 and 1 of K and 0 of V, then
  // what W(-1) would have asked for, 2 of K and 1 of V
  {
    typename St::Rows ahead[kAhead];
    typename St::Held first[2];
    st.first(a, WIN ? walk_pos<kKeys>(it.walk, 0) : lo, rows);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      ahead[i] = rows;
      st.look(it.range, ahead[i]);
      next(i + 1, rows);
    }
    st.look(it.range, rows);
    vp = st.place(a, ahead[0], left(0));
    kp = st.place(a, ahead[1], left(1));
    st.template issue<true>(k, vp, lk, first[0]);
    st.template issue<false>(v, vp, lv, vh);
    st.template issue<true>(k, kp, lk + kTile, first[1]);
    st.template land<true>(first[0], lk);
    st.template land<false>(vh, lv);
    st.template land<true>(first[1], lk + kTile);
    vp = kp;
    kp = st.place(a, ahead[2], left(2));
    st.template issue<true>(k, kp, lk + 2 * kTile, kh);
    st.template issue<false>(v, vp, lv + kTile, vh);
  }
  const Row row = row_at(a, it, (t >> 6) * 32 + (t & 31));
  Wave<D> w;
  w.start(a, row);
  uint32_t wave_hi, wave_least, full;
  if constexpr (WIN) {
    wait_loads();
    meet();
    full = it.walk.full;
  } else {
    seen_by_wave(row, 32, &wave_hi, &wave_least);
    // whole tiles that every row of the workgroup sees
    if ((t & 63) == 0) least[t >> 6] = wave_least;
    wait_loads();
    meet();
    uint32_t below = hi;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) below = least[i] < below ? least[i] : below;
    full = uniform(below > lo ? (below - lo) / kKeys : 0);
  }

  uint32_t now = 0, n = 0;  // tile n is at `now` in the ring
  const auto before = [&](uint32_t x) { return x ? x - kTile : kAhead * kTile; };
  const auto fetch = [&] {
    const uint32_t to = before(now);  // tile n + 3 of K takes the place of n - 1
    if (E4M3) {  // what W(n - 1) asked for: tile n + 2 of K, n + 1 of V
      st.template land<true>(kh, lk + before(to));
      st.template land<false>(vh, lv + before(before(to)));
    }
    vp = kp;
    kp = st.place(a, rows, left(n + kAhead));
    st.template issue<true>(k, kp, lk + to, kh);
    st.template issue<false>(v, vp, lv + before(to), vh);
    next(n + kAhead + 1, rows);
    st.look(it.range, rows);
  };
  const auto step = [&] {
    now = now == kAhead * kTile ? 0 : now + kTile;
    ++n;
  };
  if (full) {
    if (uniform(t >> 6) >= WAVES / 2) meet();  // these waves are a phase behind
    f32x16 s[2];
    bf16x8 p[2][2];
    const auto weigh = [&] {
      fetch();
      w.template weights<2>(a, s, p);
      step();
      // all but what was asked for just now; and no work moves behind the barrier
      if (!E4M3) wait_copies<2 * St::kSteps>();
      hold(p);
      meet();
    };
    w.template scores<2>(lk, s);
    meet();
    weigh();
#pragma unroll 1
    while (n < full) {
      __builtin_amdgcn_s_setprio(0);
      w.multiply(lv + before(now), p, lk + now, s);
      __builtin_amdgcn_s_setprio(1);
      meet();
      weigh();
    }
    w.template values<2>(lv + before(now), p);
    wait_loads();
    if (uniform(t >> 6) < WAVES / 2) meet();
    meet();
  }
  if constexpr (WIN) {
    // A window has more tiles with a mask than a diagonal has: each wave looks through
    // what it brought of V itself, and copies are waited for a tile after they began.
    const auto look = [&](uint32_t tile, uint32_t at) {  // tile `tile` of V, at `at` in the ring
      bool bad = false;
      if (E4M3) {  // a thread's own row, as land() wrote it
#pragma unroll
        for (int i = 0; i < St::kSteps; ++i) {
          const uint32_t row = i * St::kRows + t / St::kRowLanes, chunk = 2 * (t % St::kRowLanes);
          if (kKeys < St::kRows && row >= kKeys) break;
          const uint8_t* of = lv + at + row * D * 2;
          bad |= w.nonfinite(*(const u32x4*)(of + (chunk ^ WideSwizzle<D>::v(row)) * 16)) ||
                 w.nonfinite(*(const u32x4*)(of + ((chunk + 1) ^ WideSwizzle<D>::v(row)) * 16));
        }
      } else {
#pragma unroll
        for (int i = 0; i < St::kSteps; ++i) bad |= w.nonfinite(*(const u32x4*)(lv + at + i * WAVES * 1024 + t * 16));
      }
      if (__any(bad) && (t & 63) == 0) shared.bad[tile & 1][t >> 6] = 1;
      if (!__any(bad) && (t & 63) == 0) shared.bad[tile & 1][t >> 6] = 0;
    };
    if (n < it.walk.count) {
      look(n, now);
      meet();
    }
#pragma unroll 1
    for (; n < it.walk.count;) {
      const bool more = n + 1 < it.walk.count;
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) bad |= shared.bad[n & 1][i];
      if (more) fetch();
      const auto seen = seen_of<true>(a, row, walk_pos<kKeys>(it.walk, n), kKeys);
      if (__any(seen.bits != 0)) w.template tile<2, true>(a, lk + now, lv + now, seen, uniform(bad));
      if (!more) break;
      step();
      if (!E4M3) wait_copies<2 * St::kSteps>();
      look(n, now);
      meet();
    }
    wait_loads();  // the copies of tiles past the last
  } else {
#pragma unroll 1
    for (uint32_t pos = lo + full * kKeys; pos < hi; pos += kKeys) {  // hi + kKeys fits 32 bits
      const bool more = pos + kKeys < hi;
      if (more) fetch();
      if (pos < wave_hi) w.template tile<2, false>(a, lk + now, lv + now, seen_of<false>(a, row, pos, kKeys));
      if (!more) break;
      step();
      wait_loads();
      meet();
    }
  }
  // with a window, a split's part counts as seen where the row sees any key at all
  const bool sees = WIN ? row.limit > 0 : row.limit > lo && hi > lo;
  if (a.part_o) {
    meet();  // the tiles have been read
    constexpr uint32_t kRoom = 32 * D * 4;
    static_assert(WAVES / 2 * kRoom <= 4 * kTile, "");
    const uint32_t wave = uniform(t >> 6);
    w.template finish_part<WIN>(a, row, sees, prefix ? a.own_splits + split : split, a.own_splits + a.prefix_splits,
                  wave < WAVES / 2 ? lk + wave * kRoom : lv + (wave - WAVES / 2) * kRoom);
  } else {
    w.template finish<WIN>(a, row, sees);
  }
}

// ------------------------------------------------------------ few query rows
//
// QT x 16 query rows, as columns of 16 x 16 products, against a long axis of
// keys: the rows of one decoding sequence, or of many that share a prefix.
// Four waves hold the same rows and take every fourth group of KEYS keys
// through LDS of their own, so no wave waits for another until their parts
// are joined at the end.  K and V have two places each; the copy into one
// begins as soon as what it held has been multiplied, so that one to two
// groups are always on their way.  Bytes stay e4m3 in LDS and are widened on
// the way into the product.
//
// Bound by memory: 64 sequences of 8192 tokens, 8 KV heads of 128 for 4 query
// heads each, take 367 us, 5.9 TB/s of K and V, each read once.  16 columns, as
// that is the least that a matrix product takes; 32 where a sequence has more
// rows (33 to 64 as two tiles that read the keys twice, from L2 the second time).
//
// A lane holds column lane % 16; of scores it has keys 4 (lane / 16) + r of
// each 16, which is P^T's operand of a 16 x 16 x 16 product, and of a 16 x 16 x
// 32 one over two groups of 16 if V^T's operand takes its keys in that order.

template <int D, bool E4M3, int QT, int KEYS, bool WIN>
struct Narrow {
  static constexpr int kBytes = D * (E4M3 ? 1 : 2), kSub = KEYS / 16;
  static_assert(KEYS == 32 || (KEYS == 16 && !E4M3), "");
  bf16x8 q[QT][D / 32];
  f32x4 o[QT][D / 16];
  float m[QT], l[QT];  // the maximum is the row's; the sum this lane's share
  float e[WIN ? QT : 1];  // the sum before rounding, for its logarithm
  uint32_t k_lane, v_lane;

  __device__ __forceinline__ void start(const Args& a, const Row (&row)[QT]) {
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, x = lane & 15;
#pragma unroll
    for (int c = 0; c < QT; ++c) {
      const uint16_t* src = a.q + row[c].row * a.q_row + row[c].head * a.q_head + 8 * g;
#pragma unroll
      for (int t = 0; t < D / 32; ++t) {
        u32x4 w = {0, 0, 0, 0};
        if (row[c].valid) w = *(const u32x4*)(src + 32 * t);
        q[c][t] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o[c][j] = f32x4{};
      m[c] = kNoMax;
      l[c] = 0;
      if (WIN) e[c] = 0;
    }
    using S = NarrowSwizzle<kBytes>;
    if (E4M3) {
      k_lane = x * kBytes + (((g >> 1) ^ S::k(x)) << 4) + (g & 1) * 8;
      // rows of eight keys: 4 g .. 4 g + 3 and the same 16 on
      const uint32_t r = x >> 1, key = 4 * g + (r & 3) + (r >> 2) * 16;
      v_lane = key * kBytes + (S::v(key) << 4) + (x & 1) * 8;
    } else {
      k_lane = x * kBytes + ((g ^ S::k(x)) << 4);
      const uint32_t key = 4 * g + (x >> 2);
      v_lane = key * kBytes + ((((x & 3) >> 1) ^ S::v(key)) << 4) + (x & 1) * 8;
    }
  }

  __device__ __forceinline__ void scores(const uint8_t* lk, f32x4 (&s)[QT][kSub]) const {
    uint32_t at = lds_address(lk) + k_lane;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int c = 0; c < QT; ++c)
#pragma unroll
      for (int n = 0; n < kSub; ++n) s[c][n] = f32x4{};
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int n = 0; n < kSub; ++n) {
        const uint32_t x = (at ^ (t << (E4M3 ? 5 : 6))) + n * 16 * kBytes;
        u32x4 w;
        if (E4M3) {
          const u32x2 e = *(const lds_pair*)(uintptr_t)x;
          w = widen(e.x, e.y);
        } else {
          w = *(const lds_words*)(uintptr_t)x;
        }
#pragma unroll
        for (int c = 0; c < QT; ++c)
          s[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), q[c][t], s[c][n], 0, 0, 0);
      }
  }

  // Weights of a group, and the running maximum and sum (see Wave::weights).
  __device__ __forceinline__ void weights(const Args& a, f32x4 (&s)[QT][kSub], bool masked,
                                          const Seen<WIN> (&seen)[QT]) {
    const int g4 = ((threadIdx.x >> 4) & 3) * 4;
    float top[QT];
    bool up = false;
#pragma unroll
    for (int c = 0; c < QT; ++c) {
      float x = kNoMax;
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (masked) s[c][n][r] = seen[c].part(g4).key(16 * n + r) ? s[c][n][r] : kNoMax;
          x = fmaxf(x, s[c][n][r]);
        }
      const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      top[c] = across_halves_max(fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
      up |= top[c] > m[c] + a.margin || m[c] == kNoMax;
    }
    if (__any(up)) {
#pragma unroll
      for (int c = 0; c < QT; ++c) {
        const float to = fmaxf(m[c], top[c]), base = to == kNoMax ? 0.0f : to;
        const float f = __builtin_amdgcn_exp2f((m[c] - base) * a.c);
        l[c] *= f;
        if (WIN) e[c] *= f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[c][j] *= f;
        m[c] = to;
      }
    }
#pragma unroll
    for (int c = 0; c < QT; ++c) {
      const float mc = m[c] == kNoMax ? 0.0f : m[c] * a.c;
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // the weight that is summed is the rounded one that multiplies V:
          // what rounding does to a row's heaviest weights divides out again
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][n][r], a.c, -mc));
          if (WIN) e[c] += x;
          s[c][n][r] = (float)(__bf16)x;
          l[c] += s[c][n][r];
        }
    }
  }

  // P^T's operand: keys 4 (lane / 16) + r of each group of 16
  static __device__ __forceinline__ auto p_operand(const f32x4 (&s)[kSub]) {
    if constexpr (KEYS == 16) {
      s16x4 p;
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = __builtin_bit_cast(short, (__bf16)s[0][r]);
      return p;
    } else {
      bf16x8 p;
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = (__bf16)s[i / 4][i % 4];
      return p;
    }
  }

  // V^T's operand: 16 values of D from 16 j
  static __device__ __forceinline__ auto v_operand(uint32_t at, int j) {
    typedef __attribute__((address_space(3))) s16x4* p4;
    if constexpr (E4M3) {
      typedef int i32x2 __attribute__((ext_vector_type(2)));
      typedef __attribute__((address_space(3))) i32x2* p2;
      const i32x2 e = __builtin_amdgcn_ds_read_tr8_b64_v2i32((p2)(uintptr_t)(at ^ (j << 4)));
      return __builtin_bit_cast(bf16x8, widen((uint32_t)e.x, (uint32_t)e.y));
    } else if constexpr (KEYS == 16) {
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(at ^ (j << 5)));
    } else {
      const uint32_t x = at ^ (j << 5);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)x);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(x + 16 * kBytes));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }

  static __device__ __forceinline__ f32x4 multiply(s16x4 v, s16x4 p, f32x4 o) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, p, o, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 multiply(bf16x8 v, bf16x8 p, f32x4 o) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0);
  }

  __device__ __forceinline__ void values(const uint8_t* lv, const f32x4 (&s)[QT][kSub], bool masked,
                                         const Seen<WIN> (&seen)[QT]) {
    uint32_t at = lds_address(lv) + v_lane;
    asm volatile("" : "+v"(at));
    if (masked && nonfinite(lv)) {
      values_seen(at, s, seen);
      return;
    }
    decltype(p_operand(s[0])) p[QT];
#pragma unroll
    for (int c = 0; c < QT; ++c) p[c] = p_operand(s[c]);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const auto v = v_operand(at, j);
#pragma unroll
      for (int c = 0; c < QT; ++c) o[c][j] = multiply(v, p[c], o[c][j]);
    }
  }

  // Whether the tile of V holds an infinity or a NaN (e4m3 has only NaN).
  __device__ __forceinline__ bool nonfinite(const uint8_t* lv) const {
    bool bad = false;
#pragma unroll 1
    for (uint32_t at = (threadIdx.x & 63) * 16; at < KEYS * kBytes; at += 1024) {
      const u32x4 w = *(const u32x4*)(lv + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (E4M3) {
#pragma unroll
          for (int y = 0; y < 32; y += 8) bad |= (w[i] >> y & 0x7Fu) == 0x7Fu;
        } else {
          bad |= (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
        }
      }
    }
    return __any(bad);
  }

  // values() where V holds infinities or NaN that some rows do not see: one
  // key's product at a time, kept by the rows that see the key.
  __device__ __forceinline__ void values_seen(uint32_t at, const f32x4 (&s)[QT][kSub],
                                              const Seen<WIN> (&seen)[QT]) {
    const uint32_t g = (threadIdx.x >> 4) & 3;
    constexpr int kWords = KEYS / 8;
    typedef uint32_t words __attribute__((ext_vector_type(kWords)));
#pragma unroll 1
    for (uint32_t key = 0; key < KEYS; ++key) {
      // the key's element of an operand: lanes of group key / 4 % 4, place key / 16 * 4 + key % 4
      const uint32_t place = key / 16 * 4 + key % 4;
      const uint32_t half = (key / 4 & 3) == g ? 0xFFFFu << (place & 1) * 16 : 0;
      words only;
#pragma unroll
      for (int i = 0; i < kWords; ++i) only[i] = place / 2 == (uint32_t)i ? half : 0;
#pragma unroll
      for (int c = 0; c < QT; ++c) {
        const auto p = p_operand(s[c]);
        using V = decltype(v_operand(at, 0));
        const V weight = __builtin_bit_cast(V, __builtin_bit_cast(words, p) & only);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          const V v = __builtin_bit_cast(V, __builtin_bit_cast(words, v_operand(at, j)) & only);
          const f32x4 with = multiply(v, weight, o[c][j]);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[c][j][r] = seen[c].key((int)key) ? with[r] : o[c][j][r];
        }
      }
    }
  }
};

template <int D, bool E4M3, int WAVES>
struct Few {
  static constexpr int kWaves = WAVES, kBytes = D * (E4M3 ? 1 : 2);
  static constexpr int kKeys = kBytes == 256 ? 16 : 32;  // LDS for two workgroups on a CU
  static constexpr int kTile = kKeys * kBytes;
  static constexpr int kRing = kWaves * 4 * kTile;
  static constexpr int kRows = 32;  // at most
  struct Lds {
    __align__(1024) uint8_t ring[kRing];
    float tops[kWaves][kRows], sums[kWaves][kRows];
  };
  struct WithSums : Lds {
    float exact[kWaves][kRows];
  };
};

template <int D, bool E4M3, int WAVES, Within WITHIN, int QT, bool WIN = false>
__device__ __forceinline__ void few_rows(
    const ArgsOf<WIN>& a, bool prefix, uint32_t b,
    std::conditional_t<WIN, typename Few<D, E4M3, WAVES>::WithSums, typename Few<D, E4M3, WAVES>::Lds>& shared) {
  using F = Few<D, E4M3, WAVES>;
  constexpr int M = 16 * QT, kKeys = F::kKeys, kTile = F::kTile, kWaves = F::kWaves;
  using St = Stage<F::kBytes, false, kKeys, 64, WITHIN, NarrowSwizzle<F::kBytes>>;
  uint8_t* const lds = shared.ring;
  auto& tops = shared.tops;
  auto& sums = shared.sums;
  const uint32_t wave = uniform(threadIdx.x >> 6), t = threadIdx.x & 63;
  const uint32_t kv_head = b % a.heads;
  b /= a.heads;
  const uint32_t splits = prefix ? a.prefix_splits : a.own_splits;
  const uint32_t split = b % splits, tile = b / splits;
  const Tile it = make_tile<M, false, kKeys, WIN>(a, prefix, tile, split, splits, kv_head, kKeys);
  if (!it.any) return;
  const uint64_t head_bytes = (uint64_t)kv_head * F::kBytes;
  const uint8_t *k = a.k + head_bytes, *v = a.v + head_bytes;
  // groups wave, wave + 4, ... of the range
  constexpr uint32_t kStep = kWaves * kKeys;
  // (with windows, `pos` and `hi` count groups, and a step is one for each wave)
  const uint32_t hi = WIN ? it.walk.count : it.range.hi;
  uint32_t pos = WIN ? wave : it.range.lo + wave * kKeys;
  constexpr uint32_t kMore = WIN ? kWaves : kStep;
  uint8_t* const lk = lds + wave * 4 * kTile;
  uint8_t* const lv = lk + 2 * kTile;
  Narrow<D, E4M3, QT, kKeys, WIN> w;
  const St st(a, t);
  const uint32_t add_blocks = kStep / a.bs, add_tokens = kStep % a.bs;
  const auto rest = [&](uint32_t from) {
    if constexpr (WIN) {
      const uint32_t x = walk_pos<kKeys>(it.walk, from);
      return from < hi && x < it.walk.end ? it.walk.end - x : 0;
    }
    return from < hi ? hi - from : 0;
  };
  const auto next = [&](uint32_t to, typename St::Rows& r) {
    if (WIN)
      st.first(a, walk_pos<kKeys>(it.walk, to), r);
    else
      st.next(a, add_blocks, add_tokens, r);
  };
  typename St::Rows rows;
  typename St::Places at;
  typename St::Held none;
  if (pos < hi) {  // copies begin before anything else
    typename St::Rows second;
    st.first(a, WIN ? walk_pos<kKeys>(it.walk, pos) : pos, rows);
    second = rows;
    next(pos + kMore, second);
    st.look(it.range, rows);
    st.look(it.range, second);
    at = st.place(a, rows, WIN ? rest(pos) : hi - pos);
    st.template issue<true>(k, at, lk, none);
    st.template issue<false>(v, at, lv, none);
    at = st.place(a, second, rest(pos + kMore));
    st.template issue<true>(k, at, lk + kTile, none);
    st.template issue<false>(v, at, lv + kTile, none);
    rows = second;
    next(pos + 2 * kMore, rows);
    st.look(it.range, rows);
  }
  Row row[QT];
  uint32_t least = ~0u;
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    row[c] = row_at(a, it, 16 * c + (t & 15));
    uint32_t hi, lo;
    seen_by_wave(row[c], 16, &hi, &lo);
    least = lo < least ? lo : least;
  }
  w.start(a, row);
  if (pos < hi) {
    uint32_t x = 0;
    constexpr int kLater = 3 * St::kSteps;  // copies begun after the one that is waited for
    const auto group = [&](auto masked) {
      f32x4 s[QT][kKeys / 16];
      Seen<WIN> seen[QT];
#pragma unroll
      for (int c = 0; c < QT; ++c) {
        if constexpr (WIN)
          seen[c] = {Seen<true>::first(kKeys)};
        else
          seen[c] = {kKeys};
        if (masked) seen[c] = seen_of<WIN>(a, row[c], WIN ? walk_pos<kKeys>(it.walk, pos) : pos, kKeys);
      }
      at = st.place(a, rows, rest(pos + 2 * kMore));
      wait_copies<kLater>();
      w.scores(lk + x, s);
      wait_lds();
      st.template issue<true>(k, at, lk + x, none);
      w.weights(a, s, masked, seen);
      wait_copies<kLater>();
      w.values(lv + x, s, masked, seen);
      // table entries are read where the products of V hide it: scalar loads
      // and LDS reads share a counter
      __builtin_amdgcn_sched_barrier(0);
      next(pos + 3 * kMore, rows);
      st.look(it.range, rows);
      wait_lds();
      st.template issue<false>(v, at, lv + x, none);
    };
    // groups that all rows see, then the others; hi + 2 kStep fits 32 bits
    const uint32_t whole = WIN ? it.walk.full : least < hi ? least : hi;
#pragma unroll 1
    for (; WIN ? pos < whole : pos + kKeys <= whole; pos += kMore, x ^= kTile) group(std::false_type{});
#pragma unroll 1
    for (; pos < hi; pos += kMore, x ^= kTile) group(std::true_type{});
    wait_loads();
  }
  // join the waves: each row's common maximum first, then two and two
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    if (t < 16) tops[wave][16 * c + t] = w.m[c];
    w.l[c] += __shfl_xor(w.l[c], 16);
    w.l[c] += __shfl_xor(w.l[c], 32);
    if (WIN) {
      w.e[c] += __shfl_xor(w.e[c], 16);
      w.e[c] += __shfl_xor(w.e[c], 32);
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    float m = kNoMax;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = fmaxf(m, tops[i][16 * c + (t & 15)]);
    const float f = w.m[c] == kNoMax ? 0.0f : __builtin_amdgcn_exp2f((w.m[c] - m) * a.c);
    w.m[c] = m;
    if (t < 16) sums[wave][16 * c + t] = w.l[c] * f;  // a wave that saw nothing adds zeros
    if constexpr (WIN)
      if (t < 16) shared.exact[wave][16 * c + t] = w.e[c] * f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) w.o[c][j] *= f;
  }
  constexpr uint32_t kPart = M * D;  // floats of one wave
  static_assert(kPart * 4 * kWaves / 2 <= F::kRing, "two waves' parts fit");
  float* const parts = (float*)lds;
#pragma unroll
  for (uint32_t half = kWaves / 2; half > 0; half /= 2) {
    float* mine = parts + (wave % half) * kPart;
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int c = 0; c < QT; ++c)
#pragma unroll
        for (int j = 0; j < D / 16; ++j) *(f32x4*)(mine + ((c * (D / 16) + j) * 64 + t) * 4) = w.o[c][j];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int c = 0; c < QT; ++c)
#pragma unroll
        for (int j = 0; j < D / 16; ++j) w.o[c][j] += *(const f32x4*)(mine + ((c * (D / 16) + j) * 64 + t) * 4);
    }
    __syncthreads();
  }
  if (wave != 0) return;
  const uint32_t all = a.own_splits + a.prefix_splits, g4 = (t >> 4) * 4;
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    if (!row[c].valid) continue;
    w.l[c] = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) w.l[c] += sums[i][16 * c + (t & 15)];
    const bool sees = WIN ? row[c].limit > 0 : row[c].limit > it.range.lo && hi > it.range.lo;
    float exact = 0;
    if constexpr (WIN)
#pragma unroll
      for (int i = 0; i < kWaves; ++i) exact += shared.exact[i][16 * c + (t & 15)];
    if (a.part_o) {
      const uint64_t to = ((uint64_t)row[c].row * a.heads * a.group + row[c].head) * all +
                          (prefix ? a.own_splits + split : split);
      if (t < 16) a.part_ml[to] = float2{sees ? fmaxf(w.m[c], kLeast) : w.m[c], w.l[c]};
      if constexpr (WIN)
        if (t < 16) a.part_sum[to] = exact;
      if (w.l[c] == 0.0f) continue;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) *(f32x4*)(a.part_o + to * D + 16 * j + g4) = w.o[c][j];
    } else {
      if constexpr (WIN)
        if (t < 16) write_lse(a, row[c].row, row[c].head, w.m[c], exact);
      const float f = over_sum(a.v_scale, w.l[c], sees);
      uint16_t* dst = a.out + row[c].row * a.out_row + row[c].head * a.out_head + g4;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 e;
#pragma unroll
        for (int r = 0; r < 4; ++r) e[r] = (__bf16)(w.o[c][j][r] * f);
        *(bf16x4*)(dst + 16 * j) = e;
      }
    }
  }
}

// ------------------------------------------------------------------ joining

constexpr uint32_t kMostSplits = 64;  // of either kind: two parts to a lane of the joining wave

// A wave joins the parts of one row and query head, by the rule at the top: 16
// bytes a lane, 64 / (D / 4) parts at a time, four such loads in flight.  Bound by
// memory and by its beginning: 17 parts of 64 rows and 32 heads of 128, 17.9 MB,
// take 6.0 us.
template <int D, bool WIN = false>
__global__ void __launch_bounds__(256) k_join(ArgsOf<WIN> a) {
  constexpr uint32_t kLanes = D / 4, kSide = 64 / kLanes;
  const uint32_t heads = a.heads * a.group, splits = a.own_splits + a.prefix_splits;
  const uint32_t x = blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63;
  if (x >= a.rows * heads) return;
  if constexpr (WIN)  // rows before the first sequence and behind the last have no parts
    if (a.offsets && (x / heads < a.offsets[0] || x / heads >= a.offsets[a.num_seqs])) return;
  const float2* ml = a.part_ml + (uint64_t)x * splits;
  float2 p[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) p[i] = lane + 64 * i < splits ? ml[lane + 64 * i] : float2{kNoMax, 0.0f};
  float m = fmaxf(p[0].x, p[1].x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  float f[2], l = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // a part that saw nothing has sum 0 (a NaN sum is not 0)
    f[i] = p[i].y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((p[i].x - m) * a.c);
    l += p[i].y * f[i];
    if (p[i].y == 0.0f) f[i] = -1.0f;  // nothing to read
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  if constexpr (WIN) {
    if (a.lse) {
      float sum = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (f[i] >= 0) sum += a.part_sum[(uint64_t)x * splits + lane + 64 * i] * f[i];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
      if (l != l) sum = l;  // the part of a NaN has no factor
      if (lane == 0) write_lse(a, x / heads, x % heads, m, sum);
    }
  }
  const float* src = a.part_o + (uint64_t)x * splits * D + lane % kLanes * 4;
  f32x4 o = {};
  for (uint32_t s0 = 0; s0 < splits; s0 += 4 * kSide) {
    f32x4 v[4];
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t s = s0 + i * kSide + lane / kLanes;
      const float w0 = __shfl(f[0], s & 63), w1 = __shfl(f[1], s & 63);
      w[i] = s >= splits ? -1.0f : s < 64 ? w0 : w1;
      v[i] = f32x4{};
      if (!(w[i] < 0)) v[i] = *(const f32x4*)(src + (uint64_t)s * D);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!(w[i] < 0)) o += v[i] * w[i];
  }
#pragma unroll
  for (uint32_t d = kLanes; d < 64; d <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
  if (lane >= kLanes) return;
  const float y = over_sum(a.v_scale, l, m != kNoMax);
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = (__bf16)(o[i] * y);
  *(bf16x4*)(a.out + x / heads * a.out_row + x % heads * a.out_head + lane * 4) = e;
}

constexpr uint32_t kRowsTile = 256;  // rows of k_attend_rows' tile

// Splits of `keys` for `groups` workgroups where `slots` run at a time: all of
// them in one round, no share shorter than `least` keys.
uint32_t splits_for(uint64_t groups, uint64_t slots, uint64_t keys, uint64_t least) {
  const uint64_t s = groups ? slots / groups : 1, most = keys / least;
  const uint64_t got = s < most ? s : most;
  return (uint32_t)(got < 1 ? 1 : got > kMostSplits ? kMostSplits : got);
}

// Whether the rows of one load instruction of a wave lie in one block (see Stage).
bool one_block_loads(const PoolView& p) { return p.bs % (1024 / (p.dim * p.elem)) == 0; }

int check_attend(const PoolView& p, const claim_seqs* s, const claim_attend_desc* d) {
  const int rc = check_kv(p, s, &d->kv);
  if (rc != CLAIM_OK) return rc;
  if (d->reserved != 0 || (p.dim != 64 && p.dim != 128) || p.chunk_bytes > 0xFFFFFFFFull)
    return CLAIM_EINVAL;
  if (d->num_heads == 0 || d->num_heads % p.heads || d->num_heads / p.heads > 64) return CLAIM_EINVAL;
  if (!finite_positive(d->scale)) return CLAIM_EINVAL;
  if ((uint64_t)d->prefix_blocks * p.bs > 0x7FFFFFFFull || (d->prefix_blocks && !d->prefix))
    return CLAIM_EINVAL;
  // a wave of the joining kernel for each row and query head, a workgroup of 512
  // threads for each sequence and KV head: fewer than 2^32 threads
  if ((uint64_t)d->kv.num_rows * d->num_heads >= 1u << 26 || (uint64_t)d->kv.num_seqs * p.heads > 1u << 22)
    return CLAIM_EINVAL;
  return CLAIM_OK;
}

// The arguments that a description gives, but for the plan's; false where the scores'
// factor leaves 32 bits.
bool fill_args(const PoolView& p, const claim_seqs* s, const claim_attend_desc* d, Args* a) {
  a->q = (const uint16_t*)d->q.data;
  a->out = (uint16_t*)d->out.data;
  a->q_row = d->q.row_stride;
  a->q_head = d->q.head_stride;
  a->out_row = d->out.row_stride;
  a->out_head = d->out.head_stride;
  a->rows = d->kv.num_rows;
  a->num_seqs = d->kv.num_seqs;
  a->group = d->num_heads / p.heads;
  a->heads = p.heads;
  a->ids = d->kv.ids;
  a->offsets = d->kv.offsets;
  a->max_seqs = s->max_seqs;
  a->max_blocks = s->max_blocks;
  a->tables = s->tables;
  a->lengths = s->lengths;
  a->prefix = d->prefix;
  a->prefix_tokens = d->prefix_blocks * p.bs;
  a->bs = p.bs;
  a->bs_magic = 0xFFFFFFFFu / p.bs;
  a->nb = p.nb;
  a->chunk_bytes = (uint32_t)p.chunk_bytes;
  a->token_bytes = p.heads * p.dim * p.elem;
  const uint64_t plane = (uint64_t)p.nb * p.chunk_bytes;
  a->k = p.kv + 2ull * d->kv.layer * plane;
  a->v = a->k + plane;
  const float log2e = 1.44269504088896340736f;
  a->c = d->scale * d->kv.k_scale * log2e;
  a->margin = 8.0f / a->c;
  a->v_scale = d->kv.v_scale;
  return finite_positive(a->c);
}

}  // namespace

#endif
