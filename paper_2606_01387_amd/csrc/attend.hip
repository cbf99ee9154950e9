// attend.hip -- attention over a pool's blocks (gfx950): rows of queries that
// follow or end their sequences' tokens, single tokens of a decoding batch, and
// batches that share a prefix.
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

#include <type_traits>

#include "pool_view.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNoMax = -__builtin_inff();

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
  uint32_t own_splits, prefix_splits, tiles, prefix_tiles;
  float* part_o;   // [row][query head][split][dim]
  float2* part_ml;  // [row][query head][split]: maximum, sum
};

// One tile's query row of this lane.
struct Row {
  bool valid;
  uint32_t row, head;  // packed row, query head
  uint32_t limit;      // positions below it are seen
};

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
// A tile is 32 or 64 rows of D bf16 values, whole rows one after another, the
// 16-byte chunks of a row exchanged by an exclusive or with bits of the row's
// number, so that both ways of reading it touch every bank equally: K by 32
// rows x one chunk, V by 8 rows x 64 bytes.

template <int D>
__device__ __forceinline__ uint32_t k_swizzle(uint32_t row) {
  return D == 128 ? row & 15 : (row >> 1) & 7;
}

template <int D>
__device__ __forceinline__ uint32_t v_swizzle(uint32_t row) {
  return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

typedef const __attribute__((address_space(3))) u32x4 lds_words;

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

// Moves KEYS rows of one plane into a tile with THREADS threads.  bf16 rows go
// straight to LDS; e4m3 rows are loaded into registers by issue() and widened
// into LDS by land().
//
// ONE: the rows that a wave loads with one instruction (4 of 256 bytes to 16
// of 64) lie in one block, as they do wherever their number divides the block
// size.  Block, token and address are then the wave's, on the scalar unit;
// otherwise each lane has its own.  16384 causal tokens, 32 heads over 8 of
// 128, blocks of 16: FIGURE-ONE.
template <int D, bool E4M3, int KEYS, int THREADS, bool ONE>
struct Stage {
  static constexpr int kRowLanes = D * (E4M3 ? 1 : 2) / 16;  // lanes of one row
  static constexpr int kWaveRows = 64 / kRowLanes;
  static constexpr int kRows = THREADS / kRowLanes;  // rows of one step
  static constexpr int kSteps = KEYS / kRows ? KEYS / kRows : 1;
  static_assert(E4M3 || KEYS % kRows == 0, "bf16 tiles are filled by whole steps");

  struct Held {  // e4m3 bytes on their way
    u32x4 r[E4M3 ? kSteps : 1];
  };

  // The rows of one tile, a wave's first of each step (ONE) or a lane's own:
  // where they are in the list of blocks, and its entries once they are read.
  struct Rows {
    uint32_t at[kSteps], token[kSteps], entry[kSteps];
  };

  // Where they are in a plane.
  struct Places {
    uint64_t byte[kSteps];
    uint32_t entry[kSteps];
    uint32_t left;  // rows of the tile that the range has
  };

  uint32_t t, wave, k_off, v_off;  // a lane's place in its wave's rows (ONE) or in its row

  __device__ __forceinline__ Stage(const Args& a, uint32_t thread) : t(thread) {
    wave = THREADS == 64 ? 0 : uniform(thread >> 6);
    const uint32_t row = thread / kRowLanes, chunk = thread % kRowLanes;
    // swizzles repeat every 16 rows: they are the same in every step
    static_assert(kRows % 16 == 0 || kSteps == 1 || THREADS == 64, "");
    k_off = (E4M3 ? chunk : chunk ^ k_swizzle<D>(row)) * 16;
    v_off = (E4M3 ? chunk : chunk ^ v_swizzle<D>(row)) * 16;
    if (ONE) {
      k_off += row % kWaveRows * a.token_bytes;
      v_off += row % kWaveRows * a.token_bytes;
    }
  }

  __device__ __forceinline__ uint32_t row(int i) const {
    return i * kRows + (ONE ? wave * kWaveRows : t / kRowLanes);
  }

  __device__ __forceinline__ void first(const Args& a, uint32_t pos, Rows& r) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      split_pos(a, pos + row(i), &r.at[i], &r.token[i]);
      if (ONE) {
        r.at[i] = uniform(r.at[i]);
        r.token[i] = uniform(r.token[i]);
      }
    }
  }

  // The rows `keys` positions on: add_blocks = keys / bs, add_tokens = keys % bs.
  __device__ __forceinline__ void next(const Args& a, uint32_t add_blocks, uint32_t add_tokens,
                                       Rows& r) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      r.token[i] += add_tokens;
      const bool over = r.token[i] >= a.bs;
      r.token[i] = over ? r.token[i] - a.bs : r.token[i];
      r.at[i] += add_blocks + over;
    }
  }

  __device__ __forceinline__ void look(const Range& g, Rows& r) const {
    typedef const __attribute__((address_space(4))) uint32_t* scalar_list;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      r.entry[i] = CLAIM_NONE;
      if (ONE) {
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
    for (int i = 0; i < kSteps; ++i) {
      p.entry[i] = r.entry[i] < a.nb ? r.entry[i] : CLAIM_NONE;
      p.byte[i] = (uint64_t)r.entry[i] * a.chunk_bytes + (uint64_t)r.token[i] * a.token_bytes;
    }
    return p;
  }

  template <bool KEY>
  __device__ __forceinline__ void issue(const uint8_t* plane, const Places& p, uint8_t* tile,
                                        Held& held) const {
    const uint32_t off = KEY ? k_off : v_off;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (E4M3 && KEYS < kRows && i * kRows + t / kRowLanes >= KEYS) break;
      const uint32_t to = lds_address(tile) + i * THREADS * 16 + wave * 1024;
      // swizzles of a step of 4 or 8 rows are its own
      const uint32_t mine = THREADS == 64 && !E4M3 ? off ^ step_swizzle<KEY>(i) : off;
      const uint8_t* base = ONE ? uniform(plane + p.byte[i]) : plane + p.byte[i];
      const bool fine = p.entry[i] != CLAIM_NONE && row(i) + (ONE ? kWaveRows : 1) <= p.left;
      if (ONE ? fine : __all(fine)) {
        if constexpr (E4M3)
          held.r[i] = *(const u32x4*)(base + mine);
        else if constexpr (ONE)
          copy_to_lds(base, mine, to);
        else
          copy_to_lds(base + mine, to);
      } else {
        const bool there = i * kRows + t / kRowLanes < p.left;
        const uint8_t* from = there && p.entry[i] != CLAIM_NONE
                                  ? base + mine
                                  : (const uint8_t*)kFill + (KEY && there ? 16 : 0);
        if constexpr (E4M3)
          held.r[i] = *(const u32x4*)from;
        else
          copy_to_lds(from, to);
      }
    }
  }

  // What step i's swizzle adds to step 0's (a wave alone: a step is kWaveRows
  // rows, and the swizzles repeat every 16).
  template <bool KEY>
  static __device__ __forceinline__ constexpr uint32_t step_swizzle(int i) {
    return (KEY ? (D == 128 ? i * kWaveRows & 15 : (i * kWaveRows >> 1) & 7)
                : (D == 128 ? (i * kWaveRows & 3) << 2 : ((i * kWaveRows >> 1) & 1) << 2)) * 16;
  }

  template <bool KEY>
  __device__ __forceinline__ void land(const Held& held, uint8_t* tile) const {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const uint32_t row = i * kRows + t / kRowLanes, chunk = 2 * (t % kRowLanes);
        if (KEYS < kRows && row >= KEYS) break;
        const uint32_t x = KEY ? k_swizzle<D>(row) : v_swizzle<D>(row);
        uint8_t* to = tile + row * D * 2;
        *(u32x4*)(to + (chunk ^ x) * 16) = widen(held.r[i].x, held.r[i].y);
        *(u32x4*)(to + ((chunk + 1) ^ x) * 16) = widen(held.r[i].z, held.r[i].w);
      }
    }
  }
};

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
    k_lane = row * D * 2 + ((h ^ k_swizzle<D>(row)) << 4);
    const uint32_t key = 4 * h + ((lane & 15) >> 2);
    v_lane = key * D * 2 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swizzle<D>(key)) << 4) +
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

  // Takes out the keys past the first `seen` of the tile.
  template <int U>
  __device__ __forceinline__ void mask(f32x16 (&s)[U], int seen) const {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[u][r] = 32 * u + 8 * (r / 4) + r % 4 < seen - 4 * h ? s[u][r] : kNoMax;
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
  // read from LDS two groups of four products ahead of their use.
  __device__ __forceinline__ void multiply(const uint8_t* lv, const bf16x8 (&p)[2][2], const uint8_t* lk,
                                           f32x16 (&s)[2]) {
    values<2>(lv, p);
    scores<2>(lk, s);
    constexpr int kV = D / 32, kK = D / 32;  // products of a group; groups of K operands
    constexpr int kRead = 0x100, kMul = 0x8;
    __builtin_amdgcn_sched_group_barrier(kRead, 4 * kV, 0);
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        __builtin_amdgcn_sched_group_barrier(kMul, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
      }
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        __builtin_amdgcn_sched_group_barrier(kMul, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kRead, 4 / kV, 0);
      }
#pragma unroll
    for (int g = 0; g < 4 * (kK - 2); ++g) {
      __builtin_amdgcn_sched_group_barrier(kMul, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMul, 8, 0);
  }

  // A whole tile of which the lane's row sees the first `seen` keys.
  template <int U>
  __device__ __forceinline__ void tile(const Args& a, const uint8_t* lk, const uint8_t* lv, int seen) {
    f32x16 s[U];
    bf16x8 p[U][2];
    scores<U>(lk, s);
    const bool masked = __any(seen < 32 * U);
    if (masked) mask<U>(s, seen);
    weights<U>(a, s, p);
    if (masked && nonfinite<U>(lv))
      values_seen<U>(lv, p, seen);
    else
      values<U>(lv, p);
  }

  // Whether the tile of V holds an infinity or a NaN: a weight of 0 does not
  // take it out of the product.
  template <int U>
  __device__ __forceinline__ bool nonfinite(const uint8_t* lv) const {
    bool bad = false;
#pragma unroll 1
    for (uint32_t at = (threadIdx.x & 63) * 16; at < 32 * U * D * 2; at += 1024) {
      const u32x4 w = *(const u32x4*)(lv + at);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        bad |= (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
    }
    return __any(bad);
  }

  // values() where V holds infinities or NaN that some rows do not see: the
  // product over finite values, then for each place whether a row sees an
  // infinity of either sign or a NaN there (products of ones and zeros).
  template <int U>
  __device__ __forceinline__ void values_seen(const uint8_t* lv, const bf16x8 (&p)[U][2], int seen) {
    const int h = (threadIdx.x >> 5) & 1;
    const uint32_t at = lds_address(lv) + v_lane;
    const __bf16 zero = (__bf16)0.0f, one = (__bf16)1.0f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      f32x16 up = {}, down = {};  // infinities seen; a NaN counts as both
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bf16x8 v = v_operand(at, u, t, j);
          bf16x8 fine, high, low, sees;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint16_t w = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
            fine[i] = (w & 0x7F80) == 0x7F80 ? zero : v[i];
            high[i] = (w & 0x7F80) == 0x7F80 && w != 0xFF80 ? one : zero;
            low[i] = (w & 0x7F80) == 0x7F80 && w != 0x7F80 ? one : zero;
            sees[i] = 32 * u + 16 * t + 8 * (i / 4) + i % 4 < seen - 4 * h ? one : zero;
          }
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fine, p[u][t], o[j], 0, 0, 0);
          up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(high, sees, up, 0, 0, 0);
          down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(low, sees, down, 0, 0, 0);
        }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (up[r] > 0) o[j][r] += __builtin_inff();
        if (down[r] > 0) o[j][r] -= __builtin_inff();
      }
    }
  }

  // The rows' results, or their parts for the joining kernel.
  __device__ __forceinline__ void finish(const Args& a, const Row& r, bool parts, uint32_t split,
                                         uint32_t splits) {
    const uint32_t h = (threadIdx.x >> 5) & 1;
    const float sum = across_halves_add(l);
    if (!r.valid) return;
    if (parts) {
      const uint64_t at = ((uint64_t)r.row * a.heads * a.group + r.head) * splits + split;
      if (h == 0) a.part_ml[at] = float2{m, sum};
      if (sum == 0.0f) return;
      float* dst = a.part_o + at * D + 4 * h;
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f32x4*)(dst + 32 * j + 8 * g) =
              f32x4{o[j][4 * g], o[j][4 * g + 1], o[j][4 * g + 2], o[j][4 * g + 3]};
      return;
    }
    const float f = sum == 0.0f ? 0.0f : a.v_scale / sum;
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

// The sequence whose tile `tile` (of M packed query rows) is.  Sequence s
// starts at tile floor(first row x group / M) + s: an ascending bound that
// leaves every sequence the tiles it needs.
__device__ __forceinline__ uint64_t first_tile(const Args& a, uint32_t s, uint32_t M) {
  const uint64_t first = a.offsets ? a.offsets[s] : s;
  return first * a.group / M + s;
}

__device__ __forceinline__ uint32_t find_tile(const Args& a, uint32_t tile, uint32_t M) {
  uint32_t lo = 0, hi = a.num_seqs;
  const uint32_t lane = threadIdx.x & 63;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64, s = lo + lane * step;
    const uint64_t m = __ballot(s < hi && first_tile(a, s, M) <= tile);
    lo += (m ? 63u - (uint32_t)__builtin_clzll(m) : 0u) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return lo;
}

struct Item {
  Row row;
  Range range;
  uint32_t wave_hi;  // positions at or past it are seen by no row of the wave
  uint32_t all_below;  // every valid row of the wave sees the positions below it
  uint32_t split;
  bool any;          // the item has rows
};

// The rows of a tile of M, `r` this lane's among them, and the keys of one
// split.
template <int M>
__device__ __forceinline__ Item make_item(const Args& a, bool prefix, uint32_t tile, uint32_t split,
                                          uint32_t kv_head, uint32_t r, uint32_t align) {
  Item it;
  it.row.valid = false;
  it.row.row = it.row.head = 0;
  it.row.limit = 0;
  it.any = false;
  uint32_t splits;
  int64_t top;  // limit of the tile's last row
  if (prefix) {
    const uint64_t x = (uint64_t)tile * M + r, all = (uint64_t)a.rows * a.group;
    it.any = (uint64_t)tile * M < all;
    if (x < all) {
      const uint32_t row = (uint32_t)(x / a.group);
      uint32_t s = row, n = 1, i = 0;
      if (a.offsets) {
        uint32_t lo = 0, hi = a.num_seqs;
        while (hi - lo > 1) {
          const uint32_t mid = (lo + hi) / 2;
          if (a.offsets[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
        n = a.offsets[s + 1] - a.offsets[s];
        i = row - a.offsets[s];
      }
      const uint32_t id = a.ids ? a.ids[s] : s;
      it.row.valid = true;
      it.row.row = row;
      it.row.head = kv_head * a.group + (uint32_t)(x % a.group);
      const int64_t limit = id < a.max_seqs ? (int64_t)a.lengths[id] - n + i + 1 : 0;
      it.row.limit = (uint32_t)(limit < 0 ? 0 : limit < a.prefix_tokens ? limit : a.prefix_tokens);
    }
    it.range = Range{a.prefix, a.prefix_tokens / a.bs, 0, a.prefix_tokens};
    splits = a.prefix_splits;
    top = a.prefix_tokens;
    it.split = a.own_splits + split;
  } else {
    const uint32_t s = find_tile(a, tile, M);
    const uint32_t first = a.offsets ? a.offsets[s] : s;
    const uint32_t n = a.offsets ? a.offsets[s + 1] - first : 1;
    const uint64_t x0 = ((uint64_t)tile - first_tile(a, s, M)) * M, x = x0 + r;
    const uint64_t all = (uint64_t)n * a.group;
    const uint32_t id = a.ids ? a.ids[s] : s;
    // offsets that run backwards or past the rows give the sequence none
    it.any = tile >= first_tile(a, s, M) && x0 < all && first <= a.rows && n <= a.rows - first;
    const int64_t len = id < a.max_seqs ? a.lengths[id] : 0;
    if (it.any && x < all) {
      const uint32_t i = (uint32_t)(x / a.group);
      it.row.valid = true;
      it.row.row = first + i;
      it.row.head = kv_head * a.group + (uint32_t)(x % a.group);
      it.row.limit = len - n + i + 1 > 0 ? (uint32_t)(len - n + i + 1) : 0;
    }
    const uint64_t last = x0 + M < all ? x0 + M : all;
    top = it.any ? len - n + (int64_t)((last + a.group - 1) / a.group) : 0;
    it.range = Range{a.tables + (uint64_t)(id < a.max_seqs ? id : 0) * a.max_blocks, a.max_blocks,
                     a.prefix_tokens, 0};
    splits = a.own_splits;
    it.split = split;
  }
  // a row that sees a position past the table is NaN whatever else it sees:
  // one such position is enough, and a wrong length cannot hold the GPU
  uint64_t end = (uint64_t)a.max_blocks * a.bs;
  end = end > a.prefix_tokens ? end : a.prefix_tokens;
  end = end < 0xFFFFF000u ? end : 0xFFFFF000u;
  if (top > (int64_t)end + 1) top = (int64_t)end + 1;
  // this split's share of the keys from lo to the last row's limit
  const uint32_t lo = it.range.lo;
  const uint64_t keys = top > (int64_t)lo ? (uint64_t)top - lo : 0;
  const uint64_t share = ((keys + splits - 1) / splits + align - 1) / align * align;
  const uint64_t from = share * split < keys ? share * split : keys;
  const uint64_t to = from + share < keys ? from + share : keys;
  it.range.lo = uniform((uint32_t)(lo + from));
  it.range.hi = uniform((uint32_t)(lo + to));
  it.range.list = uniform(it.range.list);
  it.range.entries = uniform(it.range.entries);
  // per wave: the most and the least that a row sees
  uint32_t most = it.row.valid ? it.row.limit : 0, least = it.row.valid ? it.row.limit : ~0u;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t x = __shfl_xor(most, d), y = __shfl_xor(least, d);
    most = x > most ? x : most;
    least = y < least ? y : least;
  }
  it.wave_hi = uniform(most);
  it.all_below = uniform(least);
  return it;
}

// How many of the `keys` positions from `pos` on the row sees.
__device__ __forceinline__ int seen_of(const Row& r, uint32_t pos, uint32_t keys) {
  return r.limit <= pos ? 0 : r.limit - pos < keys ? (int)(r.limit - pos) : (int)keys;
}

// Everything that this wave has asked memory for has arrived.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);  // no work of one phase moves into the other
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // this wave's LDS reads and writes are done
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
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
// tile n and copies tile n + A of K and n + A - 1 of V (A = 2; e4m3 3, since
// its bytes stop in registers and land in W(n + 1)).  A ring of A + 1 tiles: the
// one that W(n) fills was last read in M(n - 1), by every wave before any is in
// W(n).  bf16 copies are waited for at the end of M(n + 1), one barrier before
// the first wave is in M(n + 2).

template <int D, bool E4M3, int WAVES, bool ONE>
__global__ void __launch_bounds__(WAVES * 64, 2) k_attend_rows(Args a, uint32_t prefix) {
  constexpr int M = WAVES * 32, kKeys = 64, kTile = kKeys * D * 2, kAhead = E4M3 ? 3 : 2;
  using St = Stage<D, E4M3, kKeys, WAVES * 64, ONE>;
  __shared__ __align__(1024) uint8_t lk[(kAhead + 1) * kTile];
  __shared__ __align__(1024) uint8_t lv[(kAhead + 1) * kTile];
  __shared__ uint32_t least[WAVES];
  const uint32_t t = threadIdx.x;
  uint32_t b = blockIdx.x;
  const uint32_t kv_head = b % a.heads;  // one head's keys stay in one die's cache where heads = 8
  b /= a.heads;
  const uint32_t splits = prefix ? a.prefix_splits : a.own_splits;
  const uint32_t split = b % splits, tiles = prefix ? a.prefix_tiles : a.tiles;
  const uint32_t tile = tiles - 1 - b / splits;  // late rows see the most: they start first
  const uint32_t r = (t >> 6) * 32 + (t & 31);
  const Item it = make_item<M>(a, prefix, tile, split, kv_head, r, kKeys);
  if (!it.any) return;
  const uint64_t head_bytes = (uint64_t)kv_head * D * (E4M3 ? 1 : 2);
  const uint8_t *k = a.k + head_bytes, *v = a.v + head_bytes;
  const uint32_t lo = it.range.lo, hi = it.range.hi;
  // whole tiles that every row of the workgroup sees
  if ((t & 63) == 0) least[t >> 6] = it.all_below;
  __syncthreads();
  uint32_t below = hi;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) below = least[w] < below ? least[w] : below;
  const uint32_t full = uniform(below > lo ? (below - lo) / kKeys : 0);

  Wave<D> w;
  w.start(a, it.row);
  const St st(a, t);
  typename St::Held kh, vh;
  typename St::Rows rows;
  if (full) {
    const uint32_t add_blocks = kKeys / a.bs, add_tokens = kKeys % a.bs;
    typename St::Places kp, vp;
    // tiles 0 and 1 of K and 0 of V, then what W(-1) would have asked for;
    // tiles past the full ones are copied too, and nothing reads them
    st.first(a, lo, rows);
    st.look(it.range, rows);
    vp = st.place(a, rows, kKeys);
    st.template issue<true>(k, vp, lk, kh);
    st.template issue<false>(v, vp, lv, vh);
    st.template land<true>(kh, lk);
    st.template land<false>(vh, lv);
    st.next(a, add_blocks, add_tokens, rows);
    st.look(it.range, rows);
    kp = st.place(a, rows, kKeys);
    st.template issue<true>(k, kp, lk + kTile, kh);
    st.template land<true>(kh, lk + kTile);
    st.next(a, add_blocks, add_tokens, rows);
    st.look(it.range, rows);
    if (E4M3) {
      vp = kp;
      kp = st.place(a, rows, kKeys);
      st.template issue<true>(k, kp, lk, kh);
      st.template issue<false>(v, vp, lv, vh);
      st.next(a, add_blocks, add_tokens, rows);
      st.look(it.range, rows);
    }
    wait_loads();
    meet();
    if (uniform(t >> 6) >= WAVES / 2) meet();  // these waves are a phase behind
    f32x16 s[2];
    bf16x8 p[2][2];
    uint32_t now = 0;                                  // where tile n is in the ring
    const auto before = [&](uint32_t x) { return x ? x - kTile : kAhead * kTile; };
    const auto weigh = [&] {
      const uint32_t to = before(now);  // tile n + A of K takes the place of n - 1
      if (E4M3) {  // what W(n - 1) asked for: tile n + A - 1 of K, n + A - 2 of V
        st.template land<true>(kh, lk + before(to));
        st.template land<false>(vh, lv + before(before(to)));
      }
      vp = kp;
      kp = st.place(a, rows, kKeys);
      st.template issue<true>(k, kp, lk + to, kh);
      st.template issue<false>(v, vp, lv + before(to), vh);
      st.next(a, add_blocks, add_tokens, rows);
      st.look(it.range, rows);
      w.template weights<2>(a, s, p);
      now = now == kAhead * kTile ? 0 : now + kTile;
      meet();
    };
    w.template scores<2>(lk, s);
    meet();
    weigh();
#pragma unroll 1
    for (uint32_t n = 1; n < full; ++n) {
      __builtin_amdgcn_s_setprio(1);
      w.multiply(lv + before(now), p, lk + now, s);
      __builtin_amdgcn_s_setprio(0);
      if (!E4M3) wait_loads();
      meet();
      weigh();
    }
    w.template values<2>(lv + before(now), p);
    wait_loads();
    if (uniform(t >> 6) < WAVES / 2) meet();
    meet();
  }
  uint32_t pos = lo + full * kKeys;
  if (pos < hi) {
    const auto fetch = [&](uint32_t from, uint32_t buffer) {
      st.first(a, from, rows);
      st.look(it.range, rows);
      const typename St::Places at = st.place(a, rows, hi - from);
      st.template issue<true>(k, at, lk + buffer, kh);
      st.template issue<false>(v, at, lv + buffer, vh);
    };
    fetch(pos, 0);
    st.template land<true>(kh, lk);
    st.template land<false>(vh, lv);
    wait_loads();
    meet();
    uint32_t at = 0;
#pragma unroll 1
    for (; pos < hi; pos += kKeys, at ^= kTile) {  // hi + kKeys fits 32 bits
      const bool more = pos + kKeys < hi;
      if (more) fetch(pos + kKeys, at ^ kTile);
      if (pos < it.wave_hi) w.template tile<2>(a, lk + at, lv + at, seen_of(it.row, pos, kKeys));
      if (more) {
        st.template land<true>(kh, lk + (at ^ kTile));
        st.template land<false>(vh, lv + (at ^ kTile));
      }
      wait_loads();
      meet();
    }
  }
  w.finish(a, it.row, a.part_o != nullptr, it.split, a.own_splits + a.prefix_splits);
}

// ------------------------------------------------------------ few query rows
//
// Four waves of one workgroup hold the same (up to 32) rows and take a quarter
// of the keys each, 32 at a time through LDS of their own: no wave waits for
// another until their parts are joined at the end.

template <int D, bool E4M3, bool ONE>
__global__ void __launch_bounds__(256, 1) k_attend_few(Args a) {
  constexpr int M = 32, kKeys = 32, kTile = kKeys * D * 2, kWaves = 4;
  using St = Stage<D, E4M3, kKeys, 64, ONE>;
  __shared__ __align__(1024) uint8_t lds[kWaves][2][2][kTile];
  const uint32_t wave = uniform(threadIdx.x >> 6), t = threadIdx.x & 63;
  uint32_t b = blockIdx.x;
  const uint32_t kv_head = b % a.heads;
  b /= a.heads;
  const uint32_t split = b % a.own_splits, tile = b / a.own_splits;
  const Item it = make_item<M>(a, false, tile, split, kv_head, t & 31, kKeys);
  if (!it.any) return;
  const uint64_t head_bytes = (uint64_t)kv_head * D * (E4M3 ? 1 : 2);
  const uint8_t *k = a.k + head_bytes, *v = a.v + head_bytes;
  Wave<D> w;
  w.start(a, it.row);
  // tiles wave, wave + 4, ... of the range
  constexpr uint32_t kStep = kWaves * kKeys;
  const uint32_t hi = it.range.hi;
  uint32_t pos = it.range.lo + wave * kKeys;
  uint8_t(*mine)[2][kTile] = lds[wave];
  const St st(a, t);
  typename St::Held kh, vh;
  if (pos < hi) {
    const uint32_t add_blocks = kStep / a.bs, add_tokens = kStep % a.bs;
    typename St::Rows rows;
    const auto fetch = [&](uint32_t from, int x) {
      const typename St::Places at = st.place(a, rows, hi - from);
      st.template issue<true>(k, at, mine[x][0], kh);
      st.template issue<false>(v, at, mine[x][1], vh);
      st.next(a, add_blocks, add_tokens, rows);
      st.look(it.range, rows);
    };
    st.first(a, pos, rows);
    st.look(it.range, rows);
    fetch(pos, 0);
    st.template land<true>(kh, mine[0][0]);
    st.template land<false>(vh, mine[0][1]);
    wait_loads();
    int x = 0;
#pragma unroll 1
    for (; pos < hi; pos += kStep, x ^= 1) {  // hi + kStep fits 32 bits
      const bool more = pos + kStep < hi;
      if (more) fetch(pos + kStep, x ^ 1);
      if (pos < it.wave_hi) w.template tile<1>(a, mine[x][0], mine[x][1], seen_of(it.row, pos, kKeys));
      if (more) {
        st.template land<true>(kh, mine[x ^ 1][0]);
        st.template land<false>(vh, mine[x ^ 1][1]);
      }
      wait_loads();
    }
  }
  // join the four waves: each row's common maximum first
  __shared__ float top[kWaves][32];
  if (t < 32) top[wave][t] = w.m;
  __syncthreads();
  float m = kNoMax;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) m = fmaxf(m, top[i][t & 31]);
  const float f = w.m == kNoMax ? 0.0f : __builtin_amdgcn_exp2f((w.m - m) * a.c);
  // a wave that saw nothing adds zeros
  float* sums = (float*)&lds[0][0][0][0];  // [wave][D / 32 + 1][16][64]
  float* part = sums + wave * (D / 32 * 16 + 1) * 64;
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) part[(j * 16 + r) * 64 + t] = w.o[j][r] * f;
  part[D / 32 * 16 * 64 + t] = w.l * f;
  __syncthreads();
  if (wave != 0) return;
  w.m = m;
#pragma unroll
  for (int i = 1; i < kWaves; ++i) {
    const float* p = sums + i * (D / 32 * 16 + 1) * 64;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[j][r] = (i == 1 ? w.o[j][r] * f : w.o[j][r]) + p[(j * 16 + r) * 64 + t];
    w.l = (i == 1 ? w.l * f : w.l) + p[D / 32 * 16 * 64 + t];
  }
  w.finish(a, it.row, a.part_o != nullptr, it.split, a.own_splits + a.prefix_splits);
}

// ------------------------------------------------------------------ joining

// A wave joins the parts of one row and query head: D / 64 values a lane.
template <int D>
__global__ void __launch_bounds__(256) k_join(Args a) {
  const uint32_t heads = a.heads * a.group, splits = a.own_splits + a.prefix_splits;
  const uint64_t x = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63;
  if (x >= (uint64_t)a.rows * heads) return;
  const float2* ml = a.part_ml + x * splits;
  float m = kNoMax;
  for (uint32_t s = lane; s < splits; s += 64) m = fmaxf(m, ml[s].x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  float o[D / 64] = {}, l = 0;
  for (uint32_t s = 0; s < splits; ++s) {
    const float2 p = ml[s];
    if (p.y == 0.0f) continue;  // this part saw nothing (a NaN sum is not 0)
    const float f = __builtin_amdgcn_exp2f((p.x - m) * a.c);
    l += p.y * f;
    const float* src = a.part_o + (x * splits + s) * D + lane * (D / 64);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] += src[i] * f;
  }
  const float f = l == 0.0f ? 0.0f : a.v_scale / l;
  uint16_t* dst = a.out + x / heads * a.out_row + x % heads * a.out_head + lane * (D / 64);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) ((__bf16*)dst)[i] = (__bf16)(o[i] * f);
}

// --------------------------------------------------------------------- host

struct Plan {
  bool few;  // own keys by k_attend_few
  uint32_t own_splits, prefix_splits, tiles, prefix_tiles;
  uint64_t parts;  // parts of all rows and heads; 0: none are kept
};

constexpr uint32_t kRowsTile = 256;

uint32_t splits_for(uint64_t groups, uint64_t want, uint64_t keys, uint64_t least) {
  // enough workgroups for the GPU, no share shorter than `least` keys
  const uint64_t s = groups ? (want + groups - 1) / groups : 1;
  const uint64_t most = keys / least;
  const uint64_t got = s < most ? s : most;
  return (uint32_t)(got < 1 ? 1 : got > 256 ? 256 : got);
}

Plan make_plan(const PoolView& p, const claim_seqs* s, const claim_attend_desc* d) {
  Plan r{};
  const uint64_t group = d->num_heads / p.heads, rows = d->kv.num_rows;
  const uint64_t prefix = (uint64_t)d->prefix_blocks * p.bs;
  const uint64_t table = (uint64_t)s->max_blocks * p.bs;
  const uint64_t own = table > prefix ? table - prefix : 0;
  r.few = rows * group <= 32ull * d->kv.num_seqs;
  const uint32_t M = r.few ? 32 : kRowsTile;
  r.tiles = (uint32_t)(rows * group / M + d->kv.num_seqs);
  r.own_splits = splits_for((uint64_t)r.tiles * p.heads, r.few ? 2 * p.cus : p.cus, own, r.few ? 256 : 512);
  if (prefix) {
    r.prefix_tiles = (uint32_t)((rows * group + kRowsTile - 1) / kRowsTile);
    r.prefix_splits = splits_for((uint64_t)r.prefix_tiles * p.heads, p.cus, prefix, 256);
  }
  const uint64_t splits = (uint64_t)r.own_splits + r.prefix_splits;
  r.parts = splits > 1 ? rows * d->num_heads * splits : 0;
  return r;
}

uint64_t plan_bytes(const Plan& r, uint32_t dim) {
  return r.parts ? ((r.parts * sizeof(float2) + 255) & ~255ull) + r.parts * dim * sizeof(float) : 0;
}

int check_attend(const PoolView& p, const claim_seqs* s, const claim_attend_desc* d) {
  const int rc = check_kv(p, s, &d->kv);
  if (rc != CLAIM_OK) return rc;
  if (d->reserved != 0 || (p.dim != 64 && p.dim != 128) || p.chunk_bytes > 0xFFFFFFFFull)
    return CLAIM_EINVAL;
  if (d->num_heads == 0 || d->num_heads % p.heads || d->num_heads / p.heads > 64) return CLAIM_EINVAL;
  if (!finite_positive(d->scale)) return CLAIM_EINVAL;
  if ((uint64_t)d->prefix_blocks * p.bs > 0x7FFFFFFFull || (d->prefix_blocks && !d->prefix))
    return CLAIM_EINVAL;
  if ((uint64_t)d->kv.num_rows * d->num_heads > 0x7FFFFFFFull) return CLAIM_EINVAL;
  return CLAIM_OK;
}

template <int D, bool E4M3, bool ONE>
int launch_one(const PoolView& p, const Plan& plan, const Args& a) {
  constexpr int kWaves = kRowsTile / 32;
  if (plan.few)
    hipLaunchKernelGGL((k_attend_few<D, E4M3, ONE>), dim3(plan.tiles * a.heads * a.own_splits),
                       dim3(256), 0, p.stream, a);
  else
    hipLaunchKernelGGL((k_attend_rows<D, E4M3, kWaves, ONE>),
                       dim3(plan.tiles * a.heads * a.own_splits), dim3(kWaves * 64), 0, p.stream, a, 0u);
  if (plan.prefix_tiles)
    hipLaunchKernelGGL((k_attend_rows<D, E4M3, kWaves, ONE>),
                       dim3(plan.prefix_tiles * a.heads * a.prefix_splits), dim3(kWaves * 64), 0,
                       p.stream, a, 1u);
  if (plan.parts)
    hipLaunchKernelGGL((k_join<D>), dim3((uint32_t)(((uint64_t)a.rows * a.heads * a.group + 3) / 4)),
                       dim3(256), 0, p.stream, a);
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
}

template <int D, bool E4M3>
int launch(const PoolView& p, const Plan& plan, const Args& a) {
  // the rows of one load instruction in one block: see Stage
  return p.bs % (64 * 16 / (D * (E4M3 ? 1 : 2))) == 0 ? launch_one<D, E4M3, true>(p, plan, a)
                                                       : launch_one<D, E4M3, false>(p, plan, a);
}

}  // namespace

extern "C" {

int claim_attend_work(const claim_pool* P, const claim_seqs* s, const claim_attend_desc* d,
                      uint64_t* bytes) {
  if (!P || !d || !bytes) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_attend(p, s, d);
  if (rc != CLAIM_OK) return rc;
  *bytes = d->kv.num_rows ? plan_bytes(make_plan(p, s, d), p.dim) : 0;
  return CLAIM_OK;
}

int claim_attend(claim_pool* P, const claim_seqs* s, const claim_attend_desc* d) {
  if (!P || !d) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_attend(p, s, d);
  if (rc != CLAIM_OK) return rc;
  if (d->kv.num_rows == 0) return CLAIM_OK;
  if (!rows_ok(d->q) || !rows_ok(d->out)) return CLAIM_EINVAL;
  const Plan plan = make_plan(p, s, d);
  const uint64_t need = plan_bytes(plan, p.dim);
  if (need && ((uintptr_t)d->work & 255)) return CLAIM_EINVAL;
  if (need && (!d->work || d->work_bytes < need)) return CLAIM_ENOSPC;
  SEQ_HIP(hipSetDevice(p.device));
  Args a{};
  a.q = (const uint16_t*)d->q.data;
  a.out = (uint16_t*)d->out.data;
  a.q_row = d->q.row_stride;
  a.q_head = d->q.head_stride;
  a.out_row = d->out.row_stride;
  a.out_head = d->out.head_stride;
  a.rows = d->kv.num_rows;
  a.num_seqs = d->kv.num_seqs;
  a.group = d->num_heads / p.heads;
  a.heads = p.heads;
  a.ids = d->kv.ids;
  a.offsets = d->kv.offsets;
  a.max_seqs = s->max_seqs;
  a.max_blocks = s->max_blocks;
  a.tables = s->tables;
  a.lengths = s->lengths;
  a.prefix = d->prefix;
  a.prefix_tokens = d->prefix_blocks * p.bs;
  a.bs = p.bs;
  a.bs_magic = 0xFFFFFFFFu / p.bs;
  a.nb = p.nb;
  a.chunk_bytes = (uint32_t)p.chunk_bytes;
  a.token_bytes = p.heads * p.dim * p.elem;
  const uint64_t plane = (uint64_t)p.nb * p.chunk_bytes;
  a.k = p.kv + 2ull * d->kv.layer * plane;
  a.v = a.k + plane;
  const float log2e = 1.44269504088896340736f;
  a.c = d->scale * d->kv.k_scale * log2e;
  if (!finite_positive(a.c)) return CLAIM_EINVAL;
  a.margin = 8.0f / a.c;
  a.v_scale = d->kv.v_scale;
  a.own_splits = plan.own_splits;
  a.prefix_splits = plan.prefix_splits;
  a.tiles = plan.tiles;
  a.prefix_tiles = plan.prefix_tiles;
  if (plan.parts) {
    a.part_ml = (float2*)d->work;
    a.part_o = (float*)((uint8_t*)d->work + ((plan.parts * sizeof(float2) + 255) & ~255ull));
  }
  if (p.dim == 128)
    return p.elem == 1 ? launch<128, true>(p, plan, a) : launch<128, false>(p, plan, a);
  return p.elem == 1 ? launch<64, true>(p, plan, a) : launch<64, false>(p, plan, a);
}

}  // extern "C"
