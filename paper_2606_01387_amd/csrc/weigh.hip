// weigh.hip -- the weight that each cached token got from a batch of query rows
// (gfx950): for position p, the sum over rows and query heads of exp(scale q.k_p -
// lse), lse being the logarithm of the row's sum that attention gave.
//
// Keys stay and queries pass by: a wave holds 64 keys of one KV head in registers
// as rows of its products, S = K Q^T, and adds the weights of one column of queries
// after another to one sum a key and lane.  Sums leave the lanes once, at the end.
// Nothing depends on the order in which workgroups run: each position has one
// workgroup, or parts that are joined in order.

#include "attend_rows.h"

namespace {

struct WeighArgs {
  const uint16_t* q;
  uint64_t q_row, q_head;
  uint32_t rows, num_seqs, group, heads;  // heads: KV heads
  uint32_t group_magic;                   // as bs_magic
  const uint32_t *ids, *offsets;
  uint32_t max_seqs, max_blocks;
  const uint32_t *tables, *lengths;
  uint32_t bs, bs_magic, nb;
  uint32_t chunk_bytes, token_bytes;
  const uint8_t* k;
  float c;  // scale * k_scale * log2(e)
  uint32_t window, sinks;
  uint32_t room;  // positions of a table
  const float* lse;
  float* weights;
  uint64_t weights_row;
  uint32_t tiles, chunks;  // workgroups along a sequence's keys; along its columns
  float* parts;            // [kv head][chunk][sequence][room]
};

constexpr float kLog2e = 1.44269504088896340736f;

// A sequence of the batch.
struct Item {
  uint32_t first, n, id;  // rows
  int64_t len;
  uint32_t keys;  // positions that any row sees and a table has
};

__device__ __forceinline__ Item item_at(const WeighArgs& a, uint32_t s) {
  Item it{s, 1, 0, 0, 0};
  if (a.offsets) {
    it.first = a.offsets[s];
    it.n = a.offsets[s + 1] - it.first;
    // offsets that run backwards or past the rows give the sequence none
    if (it.first > a.rows || it.n > a.rows - it.first) it.n = 0;
  }
  it.id = a.ids ? a.ids[s] : s;
  if (it.id >= a.max_seqs) return it;
  it.len = a.lengths[it.id];
  if (it.n) it.keys = it.len < (int64_t)a.room ? (uint32_t)it.len : a.room;
  return it;
}

__device__ __forceinline__ uint32_t quotient(uint32_t x, uint32_t by, uint32_t magic) {
  const uint32_t q = __umulhi(x, magic);  // rounded down: right, or one too small
  return x - q * by >= by ? q + 1 : q;
}

// A column: query head `head` of row i of the sequence, which sees positions below
// `limit`, from `low` on or below the sinks.
struct Column {
  uint32_t limit, low;
  float lse;  // in powers of two; infinity for one that adds nothing
};

__device__ __forceinline__ Column column_at(const WeighArgs& a, const Item& it, uint32_t kv_head, uint32_t x) {
  Column c{0, 0, __builtin_inff()};
  const uint32_t i = quotient(x, a.group, a.group_magic);
  if (i >= it.n) return c;
  const uint64_t heads = (uint64_t)a.heads * a.group;
  const float lse = a.lse[(it.first + i) * heads + kv_head * a.group + (x - i * a.group)];
  // a row whose logarithm is not a number, or infinite, adds nothing
  if (!(fabsf(lse) < __builtin_inff())) return c;
  const int64_t limit = it.len - it.n + i + 1;
  c.limit = limit > 0 ? (uint32_t)(limit < 0xFFFFFFFF ? limit : 0xFFFFFFFF) : 0;
  c.low = c.limit > a.window ? c.limit - a.window : 0;
  c.lse = lse * kLog2e;
  return c;
}

__device__ __forceinline__ bool sees(const Column& c, uint32_t pos, uint32_t sinks) {
  return pos < c.limit && (pos >= c.low || pos < sinks);
}

// Whether the sequence's rows i .. j all see positions first .. last, or any of them
// does one of them.
__device__ __forceinline__ bool all_see(const WeighArgs& a, const Item& it, int64_t i, int64_t j, int64_t first,
                                        int64_t last) {
  const int64_t base = it.len - it.n;
  return last <= base + i && (first > base + j - a.window || last < (int64_t)a.sinks);
}

__device__ __forceinline__ bool some_see(const WeighArgs& a, const Item& it, int64_t i, int64_t j, int64_t first,
                                         int64_t last) {
  const int64_t base = it.len - it.n;
  return first <= base + j && (last > base + i - a.window || first < (int64_t)a.sinks);
}

// A position's row in a plane; those without a block read the first one, and what
// they got is left out at the end.
__device__ __forceinline__ const uint8_t* key_row(const WeighArgs& a, const uint32_t* table, uint32_t pos,
                                                  bool* there) {
  const uint32_t at = quotient(pos, a.bs, a.bs_magic), token = pos - at * a.bs;
  const uint32_t entry = pos < a.room ? table[at] : CLAIM_NONE;
  *there = entry < a.nb;
  return a.k + (uint64_t)(*there ? entry : 0) * a.chunk_bytes + (uint64_t)(*there ? token : 0) * a.token_bytes;
}

// A value's sum over 16 neighbouring lanes, on all of them: pairs, fours, then halves
// mirrored, within the vector unit (by shuffles through LDS, a workgroup of
// k_weigh_rows took 6 us for its beginning and end).
__device__ __forceinline__ float sum16(float x) {
  const auto add = [](float v, auto how) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), decltype(how)::value, 15, 15, true));
  };
  x = add(x, std::integral_constant<int, 0xB1>{});   // lane ^ 1
  x = add(x, std::integral_constant<int, 0x4E>{});   // lane ^ 2
  x = add(x, std::integral_constant<int, 0x141>{});  // 7 - lane of eight
  return add(x, std::integral_constant<int, 0x140>{});  // 15 - lane of sixteen
}

// -------------------------------------------------------------- few columns
//
// Four waves share the KV heads of 64 keys (of 128 or 256, where there are two heads
// or one); their sums meet in LDS.  Bound by memory: each key is read once, for
// all heads of its group.  A lane has key lane % 16 of 16 and, of each 32
// elements, eight; keys and queries take them in the same order.  64 sequences of up
// to 8192 tokens, 8 KV heads of 128 for 4 query heads each, in 126 us, 4.9 TB/s.  Half
// of the keys on their way while the other half is weighed takes more registers and
// 134 us; what is left is the order of the loads, 64 bytes of 16 keys each: whole keys
// one after another would take 118 us, but not lie as the products need them.  The same
// in e4m3 takes 85 us, 3.6 TB/s.

template <int D, bool E4M3>
__global__ void __launch_bounds__(256) k_weigh_few(WeighArgs a) {
  constexpr int kBytes = D * (E4M3 ? 1 : 2), kSteps = D / 32, kLoads = kBytes / 64;
  __shared__ float sums[256];
  const uint32_t s = blockIdx.x / a.tiles, lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint32_t x = lane & 15, g = lane >> 4;
  const Item it = item_at(a, s);
  const uint32_t together = a.heads >= 4 ? 4 : a.heads >= 2 ? 2 : 1;  // waves of the same keys
  const uint32_t span = 256 / together;
  const uint32_t* table = a.tables + (uint64_t)(it.id < a.max_seqs ? it.id : 0) * a.max_blocks;
  const uint32_t columns = it.n * a.group;
  for (uint32_t tile = blockIdx.x - s * a.tiles; (uint64_t)tile * span < it.keys; tile += a.tiles) {
    if (!some_see(a, it, 0, it.n - 1, tile * span, (int64_t)tile * span + span - 1)) continue;
    const uint32_t pos = tile * span + wave / together * 64;  // this wave's 64 keys
    float acc[4][4] = {};
    const bool work = pos < it.keys && some_see(a, it, 0, it.n - 1, pos, (int64_t)pos + 63);
    const bool full = all_see(a, it, 0, it.n - 1, pos, (int64_t)pos + 63);
    if (work) {
      const uint8_t* at[4];
      bool there;
#pragma unroll
      for (int n = 0; n < 4; ++n) at[n] = key_row(a, table, pos + 16 * n + x, &there) + 16 * g;
      for (uint32_t h = wave % together; h < a.heads; h += together) {
        u32x4 key[4][kLoads];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int t = 0; t < kLoads; ++t) key[n][t] = *(const u32x4*)(at[n] + (uint64_t)h * kBytes + 64 * t);
        for (uint32_t x0 = 0; x0 < columns; x0 += 16) {
          const Column col = column_at(a, it, h, x0 + x);
          const uint32_t i = quotient(x0 + x, a.group, a.group_magic);
          const uint16_t* q = a.q + (it.first + (uint64_t)i) * a.q_row +
                              (h * a.group + (x0 + x - i * a.group)) * a.q_head;
          u32x4 query[kSteps];
#pragma unroll
          for (int t = 0; t < kSteps; ++t) {
            // bf16: elements 32 t + 8 g on; e4m3: 64 (t / 2) + 16 g + 8 (t % 2) on
            const uint32_t e = E4M3 ? t / 2 * 64 + 16 * g + t % 2 * 8 : 32 * t + 8 * g;
            query[t] = i < it.n ? *(const u32x4*)(q + e) : u32x4{0, 0, 0, 0};
          }
          f32x4 score[4];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            score[n] = f32x4{};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
              u32x4 w;
              if (E4M3)
                w = t % 2 ? widen(key[n][t / 2].z, key[n][t / 2].w) : widen(key[n][t / 2].x, key[n][t / 2].y);
              else
                w = key[n][t];
              score[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w),
                                                                 __builtin_bit_cast(bf16x8, query[t]),
                                                                 score[n], 0, 0, 0);
            }
          }
          const bool counts = col.lse < __builtin_inff();
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(score[n][r], a.c, -col.lse));
              const bool in = counts && (full || sees(col, pos + 16 * n + 4 * g + r, a.sinks));
              acc[n][r] += in ? w : 0.0f;
            }
        }
      }
    }
    // over the 16 columns, then the waves of the same keys
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[n][r] = sum16(acc[n][r]);
    if (x == 0)
#pragma unroll
      for (int n = 0; n < 4; ++n)
        *(f32x4*)(sums + wave * 64 + 16 * n + 4 * g) = f32x4{acc[n][0], acc[n][1], acc[n][2], acc[n][3]};
    __syncthreads();
    const uint32_t t = threadIdx.x;
    if (t < span && tile * span + t < it.keys) {
      float sum = 0;
      for (uint32_t w = 0; w < together; ++w) sum += sums[(t / 64 * together + w) * 64 + t % 64];
      bool there;
      key_row(a, table, tile * span + t, &there);
      // one workgroup adds to a position, unless its sequence is named twice
      if (there && sum != 0.0f) unsafeAtomicAdd(a.weights + it.id * a.weights_row + tile * span + t, sum);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------- many columns
//
// Four waves of 64 keys each of one KV head take a chunk of the sequence's columns,
// 64 at a time through LDS, in two halves: while one half's scores become weights on
// the vector unit, the matrix cores make those of the next.  A ring of four tiles:
// two are on their way while one is read and one is there.  A tile is as many whole
// rows as 64 columns hold (63 columns of a group of 7), so that a lane's place in it
// is the same in every tile.
//
// Bound by both units at once: 16 products and 96 vector operations of a wave take
// 0.38 us together on a SIMD, 0.28 and 0.25 us alone.  8192 causal rows of 32 query
// heads over 8 of 128 take 312 to 338 us on several cards (0.81 to 0.88 PFLOP/s of the
// pairs that are seen), of which reading operands from LDS is some 50, copies to LDS 35, the masks on the
// diagonal 15 and the beginnings of 2048 workgroups 20.  Eight waves to a workgroup:
// 361 us; half or twice the chunks: 404 and 343 us; one phase after the other: 478 us.
// The same in e4m3 takes 317 to 326 us.  In a window two compares a pair and nine words
// of a lane that do not stay in registers (of 256, heads of 128) set the pace: the same
// rows in a window of 4096 take 287 to 293 us and in one of 512 191 to 194.

constexpr uint32_t kManyWaves = 4, kManyKeys = 64 * kManyWaves, kManyColumns = 64;

template <int D>
struct WeighMany {
  static constexpr int kTile = kManyColumns * D * 2, kRing = 4;
  static constexpr int kCopies = kTile / (1024 * kManyWaves) + 1;  // of a wave, for a tile
};

// 64 lanes copy 4 bytes each to LDS from `to` on (see copy_to_lds).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_words_to_lds(const uint8_t* base, uint32_t lane_offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(lane_offset), "s"(base), "s"(to)
               : "memory", "m0");
}
#pragma clang diagnostic pop

template <int D, bool E4M3>
__global__ void __launch_bounds__(64 * kManyWaves, 2) k_weigh_rows(WeighArgs a) {
  using F = WeighMany<D>;
  constexpr int kBytes = D * (E4M3 ? 1 : 2), kSteps = D / 16;
  __shared__ __align__(1024) uint8_t ring[F::kRing * F::kTile];
  __shared__ float sums[F::kRing][kManyColumns];  // the columns' logarithms
  const uint32_t t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6), half = lane >> 5;
  uint32_t b = blockIdx.x;
  const uint32_t h = b % a.heads;
  b /= a.heads;
  const uint32_t chunk = b % a.chunks;
  b /= a.chunks;
  const uint32_t tile = b % a.tiles, s = b / a.tiles;
  const Item it = item_at(a, s);
  if ((uint64_t)tile * kManyKeys >= it.keys) return;
  float* part = a.parts + (((uint64_t)h * a.chunks + chunk) * a.num_seqs + s) * a.room;
  const uint32_t base = tile * kManyKeys, pos = base + wave * 64;  // this wave's keys
  const int64_t before = it.len - it.n;
  // the tiles of rows that see any of the workgroup's keys, and this chunk's of them
  const uint32_t rows = kManyColumns / a.group;  // of a tile
  int64_t from = (int64_t)base - before, to = it.n;
  if (base >= a.sinks) {
    const int64_t last = (int64_t)base + kManyKeys - 1 - before + a.window;  // the first row past all of them
    to = last < to ? last : to;
  }
  from = from > 0 ? from : 0;
  const uint32_t first = from < to ? (uint32_t)from / rows : 0;
  const uint32_t past = from < to ? ((uint32_t)to + rows - 1) / rows : 0;
  const uint32_t share = (past - first + a.chunks - 1) / a.chunks;
  uint32_t n = uniform(first + share * chunk < past ? first + share * chunk : past);
  const uint32_t end = uniform(past - n < share ? past : n + share);
  f32x16 acc[2] = {};
  if (n < end) {
    const uint32_t* table = a.tables + (uint64_t)(it.id < a.max_seqs ? it.id : 0) * a.max_blocks;
    // a tile's columns to LDS: whole rows, 16-byte chunks exchanged as keys' are.  Columns
    // past the tile's rows, or in the last tile past the sequence's, read the first
    // one's, and add nothing.
    constexpr uint32_t kRowLanes = D / 8, kRows = 64 * kManyWaves / kRowLanes, kLooks = kManyColumns / kRows;
    const uint64_t all_heads = (uint64_t)a.heads * a.group;
    const uint32_t last = (it.n - 1) / rows, left = it.n - last * rows;  // of the last tile
    uint32_t look[kLooks], log;
    bool has[kLooks], has_log;  // in the last tile
    const uint32_t chunk_at = ((t % kRowLanes) ^ WideSwizzle<D>::k(t / kRowLanes)) * 16;  // kRows on: the same
#pragma unroll
    for (uint32_t i = 0; i < kLooks; ++i) {
      const uint32_t r = i * kRows + t / kRowLanes, row = quotient(r, a.group, a.group_magic);
      const uint32_t at = (row * (uint32_t)a.q_row + (r - row * a.group) * (uint32_t)a.q_head) * 2;
      static_assert(WideSwizzle<D>::k(kRows) == 0, "");
      look[i] = chunk_at + (row < rows ? at : 0);
      has[i] = row < left;
    }
    const uint32_t lane_row = quotient(lane, a.group, a.group_magic);
    log = lane_row < rows ? (lane_row * (uint32_t)all_heads + lane - lane_row * a.group) * 4 : 0;
    has_log = lane_row < left;
    const uint8_t* q = (const uint8_t*)(a.q + it.first * a.q_row + h * a.group * a.q_head);
    const uint8_t* lse = (const uint8_t*)(a.lse + it.first * all_heads + h * a.group);
    const auto fetch = [&](uint32_t m, uint32_t slot) {
      const bool ends = m >= last;
      const uint64_t row = (uint64_t)(ends ? last : m) * rows;
      const uint8_t *from = uniform(q + row * a.q_row * 2), *sums_from = uniform(lse + row * all_heads * 4);
#pragma unroll
      for (uint32_t i = 0; i < kLooks; ++i)
        copy_to_lds(from, ends && !has[i] ? chunk_at : look[i],
                    lds_address(ring) + slot * F::kTile + (i * kManyWaves + wave) * 1024);
      copy_words_to_lds(sums_from, ends && !has_log ? 0 : log,
                        lds_address((const uint8_t*)sums) + slot * kManyColumns * 4);
    };
    fetch(n, 0);
    fetch(n + 1, 1);
    fetch(n + 2, 2);
    bf16x8 key[2][kSteps];
    bool there;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* at = key_row(a, table, pos + 32 * u + (lane & 31), &there) + (uint64_t)h * kBytes;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        u32x4 w;
        if (E4M3) {
          const u32x2 e = *(const u32x2*)(at + 16 * i + 8 * half);
          w = widen(e.x, e.y);
        } else {
          w = *(const u32x4*)(at + 32 * i + 16 * half);
        }
        key[u][i] = __builtin_bit_cast(bf16x8, w);
      }
    }
    const uint32_t lane_at = lds_address(ring) + (lane & 31) * D * 2 + ((half ^ WideSwizzle<D>::k(lane & 31)) << 4);
    // a half's operands; the first two are read before the half before it is done
    u32x4 w[kSteps];
    const auto read = [&](uint32_t at, int i) { w[i] = *(const lds_words*)(uintptr_t)(at ^ (i << 5)); };
    const auto place = [&](uint32_t slot, int c) { return slot * F::kTile + 32 * c * D * 2 + lane_at; };
    // The scores of a half at `at`, while the last half's (half c of tile m, with the
    // columns' logarithms `lse`) become weights: of keys that all see, of keys up to the
    // columns' own, or of any.  Two products, then what the vector unit does
    // meanwhile; operands are read two steps ahead, `after`'s in the end.
    const uint32_t half_row[2] = {quotient(lane & 31, a.group, a.group_magic),
                                  quotient(32 + (lane & 31), a.group, a.group_magic)};
    const bool causal = a.window == ~0u;
    const auto step = [&](auto mode, uint32_t at, uint32_t after, f32x16 (&score)[2], float l, uint32_t limit,
                          const f32x16 (&last)[2]) {
      constexpr int kMode = decltype(mode)::value;
      // keys 0 .. upto - 1 of this lane's are seen: its keys are at steps of 1 and 8 from 4 half on
      const int upto = limit <= pos ? 0 : limit - pos < 64 ? (int)(limit - pos) - 4 * (int)half : 64;
      const Column col{limit, limit > a.window ? limit - a.window : 0, 0};
      score[0] = score[1] = f32x16{};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          score[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key[u][i], __builtin_bit_cast(bf16x8, w[i]),
                                                             score[u], 0, 0, 0);
        if (i + 2 < kSteps) read(at, i + 2); else read(after, i + 2 - kSteps);
#pragma unroll
        for (int e = 32 / kSteps * i; e < 32 / kSteps * (i + 1); ++e) {
          const int u = e / 16, r = e % 16, k = 32 * u + 8 * (r / 4) + r % 4;
          const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(last[u][r], a.c, -l));
          const bool in = kMode == 0 || (kMode == 1 ? k < upto : sees(col, pos + 4 * half + k, a.sinks));
          acc[u][r] += in ? weight : 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const auto both = [&](uint32_t at, uint32_t after, f32x16 (&score)[2], uint32_t m, int c, float lse, bool full,
                          const f32x16 (&last)[2]) {
      asm volatile("" : "+v"(at), "+v"(after));
      const bool counts = fabsf(lse) < __builtin_inff();
      const float l = half_row[c] < rows ? lse * kLog2e : __builtin_inff();
      if (full && __all(counts)) {
        step(std::integral_constant<int, 0>{}, at, after, score, l, 0, last);
        return;
      }
      const int64_t i = (int64_t)m * rows + half_row[c], limit = before + i + 1;
      uint32_t sees_to = limit < 0xFFFFFFFF ? (uint32_t)limit : 0xFFFFFFFFu;
      if (!counts || half_row[c] >= rows || i >= it.n || limit <= 0) sees_to = 0;
      if (causal)
        step(std::integral_constant<int, 1>{}, at, after, score, l, sees_to, last);
      else
        step(std::integral_constant<int, 2>{}, at, after, score, l, sees_to, last);
    };
    // this wave's tiles: some row sees some key in seen_from .. seen_to - 1, every row
    // every key in full_from .. full_to - 1
    const auto down = [&](int64_t x) { return x > 0 ? (x < 0xFFFFFFFF ? (uint32_t)x : 0xFFFFFFFFu) / rows : 0; };
    const auto up = [&](int64_t x) { return down(x + rows - 1); };
    uint32_t seen_from = down(pos - before), seen_to = ~0u;
    uint32_t full_from = up(pos + 63ll - before), full_to = it.n / rows;
    if (pos >= a.sinks) seen_to = up(pos + 63ll - before + a.window);
    if (pos + 63 >= a.sinks) {
      const uint32_t x = down((int64_t)pos - before + a.window);
      full_to = x < full_to ? x : full_to;
    }
    seen_from = uniform(seen_from);
    full_from = uniform(full_from);
    seen_to = uniform(seen_to);
    full_to = uniform(full_to);
    const auto seen = [&](uint32_t m) { return m >= seen_from && m < seen_to; };
    // Half by half: (n - 1, 1) is weighed with the products of (n, 0), (n, 0) with those
    // of (n, 1).  All waves meet before (n, 0) when the copies of tile n + 1 have arrived
    // and tile n - 1 has been read, whose place tile n + 3 takes.
    uint32_t slot = 0;  // tile n's
    f32x16 one[2] = {}, two[2] = {};
    float l1 = __builtin_inff();  // of the half before the first: it adds nothing
    wait_copies<2 * F::kCopies>();
    meet();
    read(place(0, 0), 0);
    read(place(0, 0), 1);
    for (uint32_t m = n; m <= end; ++m) {
      const uint32_t next = (slot + 1) % F::kRing;
      wait_copies<F::kCopies>();
      meet();
      fetch(m + 3, (slot + 3) % F::kRing);
      const float l0 = sums[slot][lane & 31];
      // (past the last: of columns that nobody weighs)
      if (seen(m) || (m > n && seen(m - 1)))
        both(place(slot, 0), place(slot, 1), one, m - 1, 1, l1, m > n && m - 1 >= full_from && m - 1 < full_to, two);
      if (m < end && seen(m)) {
        both(place(slot, 1), place(next, 0), two, m, 0, l0, m >= full_from && m < full_to, one);
      } else {
        read(place(next, 0), 0);
        read(place(next, 0), 1);
      }
      l1 = sums[slot][32 + (lane & 31)];
      slot = next;
    }
    wait_loads();  // no copy outlives the workgroup
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = sum16(acc[u][r]);
      const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      acc[u][r] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
  if ((lane & 31) == 0)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t p = pos + 32 * u + 8 * (r / 4) + 4 * half + r % 4;
        if (p < it.keys) part[p] = acc[u][r];
      }
}

// Parts of a position, in order: eight loads on their way at a time.
__global__ void __launch_bounds__(64) k_weigh_join(WeighArgs a, uint32_t groups) {
  const uint32_t s = blockIdx.x / groups;
  const Item it = item_at(a, s);
  const uint32_t* table = a.tables + (uint64_t)(it.id < a.max_seqs ? it.id : 0) * a.max_blocks;
  const uint32_t parts = a.heads * a.chunks;
  const uint64_t stride = (uint64_t)a.num_seqs * a.room;
  for (uint64_t p = (uint64_t)(blockIdx.x - s * groups) * 64 + threadIdx.x; p < it.keys; p += (uint64_t)groups * 64) {
    const float* part = a.parts + (uint64_t)s * a.room + p;
    bool there;
    key_row(a, table, (uint32_t)p, &there);
    float sum = 0;
    for (uint32_t i = 0; i < parts; i += 8) {
      float x[8];
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) x[j] = i + j < parts ? part[(i + j) * stride] : 0.0f;
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) sum += x[j];
    }
    if (there && sum != 0.0f) unsafeAtomicAdd(a.weights + it.id * a.weights_row + p, sum);
  }
}

// --------------------------------------------------------------------- host

struct WeighPlan {
  bool many;
  uint32_t tiles, chunks;
};

// One kernel for a call, by the mean of its sequences' columns, as the host knows no
// more of them: k_weigh_few where a tile of 64 columns holds a sequence's.  Where
// sequences differ much, some of them get the wrong one.  8 KV heads of 128 for 4 query
// heads each, all behind 4000 tokens: 63 single tokens take 103 to 107 us, a chunk of 512
// rows 50 and of 4096 rows 241 to 250; the tokens with the chunk of 512, by k_weigh_few,
// 500 us, with the one of 4096, by k_weigh_rows, 677.
//
// Tiles and chunks go by what a table can hold, so that work of one size does for any
// lengths: the prompt of 8192 above takes 654 us in a table of 131072 positions, where
// its empty tiles leave it one chunk, and the 64 single tokens 145 us in such tables.
WeighPlan make_weigh_plan(const PoolView& p, const claim_seqs* s, const claim_weigh_desc* d) {
  WeighPlan r{};
  const uint64_t group = d->num_heads / p.heads, rows = d->kv.num_rows, seqs = d->kv.num_seqs;
  const uint64_t room = (uint64_t)s->max_blocks * p.bs;
  // k_weigh_rows keeps places within 64 rows in 32 bits
  const bool near = d->q.row_stride < 1u << 24 && d->q.head_stride < 1u << 24;
  r.many = (rows * group + seqs - 1) / seqs > 64 && near;
  r.chunks = 1;
  if (!r.many) {
    const uint64_t span = p.heads >= 4 ? 64 : p.heads >= 2 ? 128 : 256;
    const uint64_t tiles = (room + span - 1) / span, most = 65536 / seqs + 1;
    r.tiles = (uint32_t)(tiles < most ? tiles : most);
    return r;
  }
  r.tiles = (uint32_t)((room + kManyKeys - 1) / kManyKeys);
  const uint64_t groups = (uint64_t)r.tiles * seqs * p.heads, columns = rows * group / seqs;
  while (r.chunks < 32 && groups * r.chunks < 8ull * p.cus && columns / r.chunks > 512) r.chunks *= 2;
  return r;
}

uint64_t plan_bytes(const PoolView& p, const claim_seqs* s, const claim_weigh_desc* d, const WeighPlan& r) {
  return r.many ? 4ull * p.heads * r.chunks * d->kv.num_seqs * s->max_blocks * p.bs : 0;
}

int check_weigh(const PoolView& p, const claim_seqs* s, const claim_weigh_desc* d) {
  const int rc = check_kv(p, s, &d->kv);
  if (rc != CLAIM_OK) return rc;
  if ((p.dim != 64 && p.dim != 128) || p.chunk_bytes > 0xFFFFFFFFull) return CLAIM_EINVAL;
  if (d->num_heads == 0 || d->num_heads % p.heads || d->num_heads / p.heads > 64) return CLAIM_EINVAL;
  if (!finite_positive(d->scale) || !finite_positive(d->scale * d->kv.k_scale * kLog2e) || d->window == 0)
    return CLAIM_EINVAL;
  if ((uint64_t)d->kv.num_rows * d->num_heads >= 1u << 26 || (uint64_t)d->kv.num_seqs * p.heads > 1u << 22)
    return CLAIM_EINVAL;
  const uint64_t room = (uint64_t)s->max_blocks * p.bs;
  if (room > 0x7FFFFFFFull || d->weights_stride < room || ((uintptr_t)d->weights & 3) || ((uintptr_t)d->lse & 3))
    return CLAIM_EINVAL;
  if (d->kv.num_rows == 0) return CLAIM_OK;
  const WeighPlan plan = make_weigh_plan(p, s, d);
  const uint64_t groups = (uint64_t)plan.tiles * plan.chunks * d->kv.num_seqs * p.heads;
  return plan.many && groups >= 1u << 24 ? CLAIM_EINVAL : CLAIM_OK;  // 2^32 threads
}

template <int D, bool E4M3>
int launch(const PoolView& p, const WeighPlan& plan, const WeighArgs& a) {
  if (!plan.many) {
    hipLaunchKernelGGL((k_weigh_few<D, E4M3>), dim3(a.num_seqs * a.tiles), dim3(256), 0, p.stream, a);
  } else {
    hipLaunchKernelGGL((k_weigh_rows<D, E4M3>), dim3(a.num_seqs * a.tiles * a.chunks * a.heads),
                       dim3(64 * kManyWaves), 0, p.stream, a);
    const uint32_t most = 32 * p.cus / a.num_seqs + 1, need = (a.room + 63) / 64;
    const uint32_t groups = need < most ? need : most;
    hipLaunchKernelGGL(k_weigh_join, dim3(a.num_seqs * groups), dim3(64), 0, p.stream, a, groups);
  }
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
}

}  // namespace

extern "C" {

int claim_weigh_work(const claim_pool* P, const claim_seqs* s, const claim_weigh_desc* d, uint64_t* bytes) {
  if (!P || !d || !bytes) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_weigh(p, s, d);
  if (rc != CLAIM_OK) return rc;
  *bytes = d->kv.num_rows ? plan_bytes(p, s, d, make_weigh_plan(p, s, d)) : 0;
  return CLAIM_OK;
}

int claim_weigh(claim_pool* P, const claim_seqs* s, const claim_weigh_desc* d) {
  if (!P || !d) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_weigh(p, s, d);
  if (rc != CLAIM_OK) return rc;
  if (d->kv.num_rows == 0) return CLAIM_OK;
  if (!rows_ok(d->q) || !d->lse || !d->weights) return CLAIM_EINVAL;
  const WeighPlan plan = make_weigh_plan(p, s, d);
  const uint64_t need = plan_bytes(p, s, d, plan);
  if (need && ((uintptr_t)d->work & 255)) return CLAIM_EINVAL;
  if (need && (!d->work || d->work_bytes < need)) return CLAIM_ENOSPC;
  WeighArgs a{};
  a.q = (const uint16_t*)d->q.data;
  a.q_row = d->q.row_stride;
  a.q_head = d->q.head_stride;
  a.rows = d->kv.num_rows;
  a.num_seqs = d->kv.num_seqs;
  a.group = d->num_heads / p.heads;
  a.group_magic = 0xFFFFFFFFu / a.group;
  a.heads = p.heads;
  a.ids = d->kv.ids;
  a.offsets = d->kv.offsets;
  a.max_seqs = s->max_seqs;
  a.max_blocks = s->max_blocks;
  a.tables = s->tables;
  a.lengths = s->lengths;
  a.bs = p.bs;
  a.bs_magic = 0xFFFFFFFFu / p.bs;
  a.nb = p.nb;
  a.chunk_bytes = (uint32_t)p.chunk_bytes;
  a.token_bytes = p.heads * p.dim * p.elem;
  a.k = p.kv + 2ull * d->kv.layer * p.nb * p.chunk_bytes;
  a.c = d->scale * d->kv.k_scale * kLog2e;
  a.window = d->window;
  a.sinks = d->sinks;
  a.room = (uint32_t)((uint64_t)s->max_blocks * p.bs);
  a.lse = d->lse;
  a.weights = d->weights;
  a.weights_row = d->weights_stride;
  a.tiles = plan.tiles;
  a.chunks = plan.chunks;
  a.parts = (float*)d->work;
  SEQ_HIP(hipSetDevice(p.device));
  if (p.dim == 128) return p.elem == 1 ? launch<128, true>(p, plan, a) : launch<128, false>(p, plan, a);
  return p.elem == 1 ? launch<64, true>(p, plan, a) : launch<64, false>(p, plan, a);
}

}  // extern "C"
