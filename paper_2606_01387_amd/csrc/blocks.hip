// blocks.hip -- sequences' blocks: growing, forking, freeing, compacting and
// copying them, and writing keys and values into them (gfx950).
//
// The plans (which blocks go where) are whole numbers made by one workgroup:
// every rank is a prefix sum, so results do not depend on the order in which
// lanes or atomics run.  The bytes are moved by a second kernel over the
// whole GPU that reads the plan from device memory; nothing comes back to the
// host.

#include "pool_view.h"

namespace {

constexpr uint32_t kNone = CLAIM_NONE;
constexpr int kPlan = 1024;  // threads of a planning workgroup
constexpr int kCopy = 256;   // threads of a copying workgroup

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Seqs {
  uint32_t max_seqs, max_blocks;
  uint32_t *tables, *lengths, *refs;
  // scratch: header (16 words), then three lists of num_blocks, then four of max_seqs
  uint32_t *head, *list_a, *list_b, *map, *rank, *len, *owner, *need;
};

// header words
enum : int { kPairs = 0, kUsed = 1 };

Seqs seqs_dev(const claim_seqs* s, uint32_t nb) {
  uint32_t* w = s->work;
  uint32_t* q = w + 16 + 3 * (uint64_t)nb;
  return Seqs{s->max_seqs, s->max_blocks, s->tables, s->lengths, s->refs, w,
              w + 16, w + 16 + nb, w + 16 + 2 * (uint64_t)nb,
              q, q + s->max_seqs, q + 2 * (uint64_t)s->max_seqs, q + 3 * (uint64_t)s->max_seqs};
}

// Exclusive prefix sum of one 64-bit value a thread over a planning
// workgroup; *total is the sum.  Counts are summed in 64 bits: a request may
// ask for far more blocks than there are.
__device__ uint64_t block_scan(uint64_t v, uint64_t* total) {
  __shared__ uint64_t wave_sum[kPlan / 64];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t y = __shfl_up(x, d);
    if (lane >= (uint32_t)d) x += y;
  }
  __syncthreads();
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    const uint64_t s = wave_sum[w];
    all += s;
    if (w < (int)wave) before += s;
  }
  *total = all;
  return before + x - v;
}

// This thread's contiguous share of the blocks: whole groups of 4.
__device__ __forceinline__ void my_blocks(uint32_t nb, uint32_t* first, uint32_t* last) {
  const uint32_t per = (nb / 4 / kPlan + 1) * 4;
  const uint64_t f = (uint64_t)per * threadIdx.x;
  *first = f < nb ? (uint32_t)f : nb;
  *last = f + per < nb ? (uint32_t)(f + per) : nb;
}

// A thread's share of the blocks, with those in use: their number, and a bit
// for each of the first 32, so that shares of up to 32 blocks (pools of up to
// 32768) are read once, all of it on its way while an entry's lengths are read.
constexpr uint32_t kBits = 32;

struct Share {
  uint32_t first, last, used, bits;
};

__device__ __forceinline__ Share my_share(const uint32_t* refs, uint32_t nb) {
  Share s;
  my_blocks(nb, &s.first, &s.last);
  s.used = s.bits = 0;
  uint32_t b = s.first;
  if (((uintptr_t)refs & 15) == 0) {
#pragma unroll 8
    for (; b + 4 <= s.last; b += 4) {
      const u32x4 r = *(const u32x4*)(refs + b);
      const uint32_t in = (r.x != 0) | (r.y != 0) << 1 | (r.z != 0) << 2 | (r.w != 0) << 3;
      s.used += __popc(in);
      if (b - s.first < kBits) s.bits |= in << (b - s.first);
    }
  }
  for (; b < s.last; ++b) {
    const uint32_t in = refs[b] != 0;
    s.used += in;
    if (b - s.first < kBits) s.bits |= in << (b - s.first);
  }
  return s;
}

__device__ __forceinline__ bool in_use(const Share& s, const uint32_t* refs, uint32_t b) {
  return b - s.first < kBits ? s.bits >> (b - s.first) & 1 : refs[b] != 0;
}

__device__ __forceinline__ uint32_t row_of(const uint32_t* ids, uint32_t i) { return ids ? ids[i] : i; }

// owner[row] = the first i that names row (rows out of range have none).
__device__ void first_owner(const Seqs& s, const uint32_t* ids, uint32_t n) {
  for (uint32_t i = threadIdx.x; i < n; i += kPlan) {
    const uint32_t r = row_of(ids, i);
    if (r < s.max_seqs) s.owner[r] = kNone;
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kPlan) {
    const uint32_t r = row_of(ids, i);
    if (r < s.max_seqs) atomicMin(&s.owner[r], i);
  }
  __syncthreads();
}

// Which of the rows named by `row` (one a thread, kNone: none) name a row first:
// in LDS where all of it fits, the lowest thread wins.
constexpr uint32_t kOwners = 8192;

__device__ bool first_to_name(uint32_t row, uint32_t max_seqs) {
  __shared__ uint32_t owner[kOwners];
  const bool in = row < max_seqs;
  if (in) owner[row] = kNone;
  __syncthreads();
  if (in) atomicMin(&owner[row], threadIdx.x);
  __syncthreads();
  return in && owner[row] == threadIdx.x;
}

// The first `want` free blocks, ascending, into list (the first kPlan of them
// into `near` too, if there is one); returns how many there are free in all.
__device__ uint64_t list_free(const Share& s, const uint32_t* refs, uint64_t want, uint32_t* list,
                              uint32_t* near = nullptr) {
  uint64_t total;
  uint64_t at = block_scan(s.last - s.first - s.used, &total);
  for (uint32_t b = s.first; b < s.last && at < want; ++b) {
    if (in_use(s, refs, b)) continue;
    if (near && at < kPlan) near[at] = b;
    list[at++] = b;
  }
  return total;
}

// The plans come in two forms.  Up to as many entries as the workgroup has
// threads, and rows enough for LDS, each entry is a thread's, in registers;
// beyond either, the entries' ranks are kept in scratch.  64 entries over 1200
// blocks: grow 5.5 us in registers and 7.9 us in scratch, fork 5.1 and 6.6 us.
__host__ __device__ inline bool plan_in_registers(uint32_t n, uint32_t max_seqs) {
  return n <= kPlan && max_seqs <= kOwners;
}

// ---------------------------------------------------------------------- grow

// Blocks that a row of `len` tokens needs for `more`: kNone if it may not.
__device__ __forceinline__ uint64_t blocks_for(uint64_t len, uint32_t more, uint32_t max_blocks, uint32_t bs) {
  const uint64_t to = len + more;
  if (to > (uint64_t)max_blocks * bs || to > 0xFFFFFFFFull) return kNone;
  return (to + bs - 1) / bs - (len + bs - 1) / bs;
}

// Rank of an entry's blocks: the prefix sum of what entries before it need.  Bound
// by dependent reads (numbers, lengths, then tables are written): 64 entries over
// 1200 blocks in 5.9 us.
__global__ void __launch_bounds__(kPlan) k_grow_few(Seqs s, const uint32_t* ids, const uint32_t* tokens,
                                                    uint32_t n, uint32_t bs, uint32_t nb,
                                                    uint64_t* holder, uint32_t* status) {
  __shared__ uint32_t ranks[kPlan], rows[kPlan], ats[kPlan], list[kPlan], blocks;
  const uint32_t i = threadIdx.x;
  if (i == 0) blocks = 0;
  const uint32_t r = i < n ? row_of(ids, i) : kNone;
  const uint32_t more = i < n ? tokens[i] : 0;
  const uint32_t len = r < s.max_seqs ? s.lengths[r] : 0;
  const Share share = my_share(s.refs, nb);
  const bool mine = first_to_name(r, s.max_seqs);
  uint64_t need = mine ? blocks_for(len, more, s.max_blocks, bs) : kNone;
  const bool fine = need != kNone;
  if (!fine) need = 0;
  uint64_t all;
  const uint64_t rank = block_scan(need, &all);
  const uint64_t free_all = list_free(share, s.refs, all, s.list_a, list);
  const bool given = fine && rank + need <= free_all;
  if (given && need) atomicMax(&blocks, (uint32_t)(rank + need));  // up to the last that got all of its own
  if (i < n) {
    if (status) status[i] = given ? CLAIM_SEQ_OK : fine ? CLAIM_SEQ_NO_BLOCKS : CLAIM_SEQ_REFUSED;
    if (given && more) s.lengths[r] = len + more;
  }
  ranks[i] = rank < nb ? (uint32_t)rank : nb;
  rows[i] = r;
  ats[i] = (uint32_t)(((uint64_t)len + bs - 1) / bs);
  __syncthreads();
  for (uint32_t k = i; k < blocks; k += kPlan) {
    uint32_t lo = 0, hi = n;  // the last entry with rank <= k: one that needs none has the rank of the next
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (ranks[mid] <= k) lo = mid; else hi = mid;
    }
    const uint32_t b = k < kPlan ? list[k] : s.list_a[k];
    s.tables[(uint64_t)rows[lo] * s.max_blocks + ats[lo] + (k - ranks[lo])] = b;
    s.refs[b] = 1;
    holder[b] = 0;
  }
}

__global__ void __launch_bounds__(kPlan) k_grow(Seqs s, const uint32_t* ids, const uint32_t* tokens,
                                                uint32_t n, uint32_t bs, uint32_t nb,
                                                uint64_t* holder, uint32_t* status) {
  first_owner(s, ids, n);
  uint64_t run = 0;  // blocks that earlier entries need
  for (uint32_t i0 = 0; i0 < n; i0 += kPlan) {
    const uint32_t i = i0 + threadIdx.x;
    uint64_t need = kNone;
    if (i < n) {
      const uint32_t r = row_of(ids, i);
      if (r < s.max_seqs && s.owner[r] == i) need = blocks_for(s.lengths[r], tokens[i], s.max_blocks, bs);
    }
    const bool fine = need != kNone;
    uint64_t total;
    const uint64_t at = run + block_scan(fine ? need : 0, &total);
    if (i < n) {
      // ranks past the blocks there are stay past them in 32 bits, also where an
      // entry needs none
      s.rank[i] = at <= nb ? (uint32_t)at : nb + 1;
      s.need[i] = (uint32_t)need;
    }
    run += total;
  }
  const uint64_t free_all = list_free(my_share(s.refs, nb), s.refs, run, s.list_a);
  __syncthreads();
  // entries whose blocks are all there: a leading part of those that need any
  uint64_t mine = 0;
  for (uint32_t i = threadIdx.x; i < n; i += kPlan) {
    const uint32_t need = s.need[i];
    uint32_t st = CLAIM_SEQ_REFUSED;
    if (need != kNone) {
      const uint64_t end = (uint64_t)s.rank[i] + need;
      st = end <= free_all ? CLAIM_SEQ_OK : CLAIM_SEQ_NO_BLOCKS;
      if (st == CLAIM_SEQ_OK && need && end > mine) mine = end;
      const uint32_t r = row_of(ids, i);
      s.len[i] = s.lengths[r];
      if (st == CLAIM_SEQ_OK) s.lengths[r] += tokens[i];
    }
    if (status) status[i] = st;
  }
  __shared__ uint32_t given_all;
  if (threadIdx.x == 0) given_all = 0;
  __syncthreads();
  if (mine) atomicMax(&given_all, (uint32_t)mine);
  __syncthreads();
  const uint32_t given = given_all;
  for (uint32_t k = threadIdx.x; k < given; k += kPlan) {
    uint32_t lo = 0, hi = n;  // as in k_grow_few
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (s.rank[mid] <= k) lo = mid; else hi = mid;
    }
    const uint32_t r = row_of(ids, lo), b = s.list_a[k];
    const uint32_t at = (s.len[lo] + bs - 1) / bs + (k - s.rank[lo]);
    s.tables[(uint64_t)r * s.max_blocks + at] = b;
    s.refs[b] = 1;
    holder[b] = 0;
  }
}

// ---------------------------------------------------------------------- fork

// Entry i's copy of a partly filled last block, with its place in the list.
__device__ __forceinline__ void fork_last(const Seqs& s, uint32_t c, uint32_t len, uint32_t rank,
                                          uint32_t from, uint32_t to, uint32_t bs, uint32_t nb,
                                          uint64_t* holder) {
  s.list_b[rank] = from;  // a missing one is passed over by the copy
  if (from < nb) {
    s.tables[(uint64_t)c * s.max_blocks + len / bs] = to;
    s.refs[to] = 1;
    holder[to] = 0;
  }
}

struct CopyShape {
  uint32_t planes, nb, pieces, piece_words, words;  // words of a chunk
};

// Child i, of `len` shared tokens, takes the full blocks of its parent's row.
__device__ __forceinline__ void share_full(const Seqs& s, uint32_t p, uint32_t c, uint32_t len, uint32_t bs,
                                           uint32_t nb, uint32_t thread, uint32_t threads) {
  const uint32_t full = len / bs < s.max_blocks ? len / bs : s.max_blocks;
  const uint32_t* from = s.tables + (uint64_t)p * s.max_blocks;
  uint32_t* to = s.tables + (uint64_t)c * s.max_blocks;
  for (uint32_t j = thread; j < full; j += threads) {
    const uint32_t b = from[j];
    to[j] = b;
    if (b < nb) atomicAdd(&s.refs[b], 1u);
  }
}

// A fork whose copies and table entries are four rounds of a workgroup at most
// is done by the planning workgroup to its end: 3 children of 2 layers of 4 KiB
// chunks, freed, forked and grown, take 15.6 us so and 18.1 us with a
// launch of its own for the copies.
constexpr uint32_t kForkAlone = 4 * kPlan;

__host__ __device__ inline bool fork_alone(const CopyShape& c, uint32_t n, uint32_t max_blocks) {
  return (uint64_t)n * c.planes * c.words <= kForkAlone && (uint64_t)n * max_blocks <= kForkAlone;
}

__global__ void __launch_bounds__(kPlan) k_fork_few(Seqs s, const uint32_t* parents, const uint32_t* children,
                                                    uint32_t n, uint32_t bs, uint32_t nb, uint64_t* holder,
                                                    uint32_t* status, CopyShape shape, u32x4* kv) {
  __shared__ uint32_t list[kPlan], sources[kPlan];
  const uint32_t i = threadIdx.x;
  const uint32_t p = i < n ? parents[i] : kNone, c = i < n ? children[i] : kNone;
  const uint32_t len = p < s.max_seqs ? s.lengths[p] : 0;
  const uint32_t there = c < s.max_seqs ? s.lengths[c] : 1;
  const Share share = my_share(s.refs, nb);
  const bool fine = first_to_name(c, s.max_seqs) && p < s.max_seqs && p != c && there == 0;
  const bool part = fine && len % bs != 0 && (uint64_t)len <= (uint64_t)s.max_blocks * bs;
  const uint32_t from = part ? s.tables[(uint64_t)p * s.max_blocks + len / bs] : kNone;
  uint64_t all;
  const uint64_t rank = block_scan(part, &all);
  const uint64_t free_all = list_free(share, s.refs, all, s.list_a, list);
  const uint32_t pairs = (uint32_t)(all < free_all ? all : free_all);
  if (i == 0) s.head[kPairs] = pairs;
  if (part) sources[rank] = from;
  __syncthreads();  // the lists are whole
  const bool given = fine && rank + part <= free_all;
  if (i < n) {
    if (status) status[i] = given ? CLAIM_SEQ_OK : fine ? CLAIM_SEQ_NO_BLOCKS : CLAIM_SEQ_REFUSED;
    s.len[i] = given ? len : 0;  // what the children share
    if (given) {
      s.lengths[c] = len;
      if (part) fork_last(s, c, len, (uint32_t)rank, from, list[rank], bs, nb, holder);
    }
  }
  if (!fork_alone(shape, n, s.max_blocks)) return;
  // copies first: their loads are on their way while tables are written
  const uint32_t per = shape.planes * shape.words, words = pairs * per;
  u32x4 r[kForkAlone / kPlan];
  uint64_t to[kForkAlone / kPlan];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t v = i + j * kPlan, pair = v / per, rest = v - pair * per;
    const uint32_t plane = rest / shape.words, word = rest - plane * shape.words;
    to[j] = ~0ull;
    if (v >= words || sources[pair] >= nb) continue;
    const uint64_t row = (uint64_t)plane * nb;
    r[j] = kv[(row + sources[pair]) * shape.words + word];
    to[j] = (row + list[pair]) * shape.words + word;
  }
  __syncthreads();  // s.len is whole
  for (uint32_t k = i / 64; k < n; k += kPlan / 64)
    share_full(s, parents[k], children[k], s.len[k], bs, nb, i % 64, 64);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (to[j] != ~0ull) kv[to[j]] = r[j];
}

__global__ void __launch_bounds__(kPlan) k_fork_plan(Seqs s, const uint32_t* parents,
                                                     const uint32_t* children, uint32_t n,
                                                     uint32_t bs, uint32_t nb, uint64_t* holder,
                                                     uint32_t* status) {
  first_owner(s, children, n);
  uint64_t run = 0;
  for (uint32_t i0 = 0; i0 < n; i0 += kPlan) {
    const uint32_t i = i0 + threadIdx.x;
    uint64_t need = 0;
    if (i < n) {
      const uint32_t p = parents[i], c = children[i];
      const bool fine = p < s.max_seqs && c < s.max_seqs && p != c && s.owner[c] == i &&
                        s.lengths[c] == 0;
      const uint32_t len = fine ? s.lengths[p] : 0;
      need = len % bs != 0 && (uint64_t)len <= (uint64_t)s.max_blocks * bs;
      s.len[i] = len;
      s.need[i] = fine ? (uint32_t)need : kNone;
    }
    uint64_t total;
    const uint64_t at = run + block_scan(need, &total);
    if (i < n) s.rank[i] = (uint32_t)at;
    run += total;
  }
  const uint64_t free_all = list_free(my_share(s.refs, nb), s.refs, run, s.list_a);
  if (threadIdx.x == 0) s.head[kPairs] = (uint32_t)(run < free_all ? run : free_all);
  __syncthreads();  // parents' lengths are in s.len: children's may change now
  for (uint32_t i = threadIdx.x; i < n; i += kPlan) {
    const uint32_t need = s.need[i], len = s.len[i], rank = s.rank[i];
    uint32_t st = CLAIM_SEQ_REFUSED;
    if (need != kNone) st = (uint64_t)rank + need <= free_all ? CLAIM_SEQ_OK : CLAIM_SEQ_NO_BLOCKS;
    if (status) status[i] = st;
    if (st != CLAIM_SEQ_OK) {
      s.len[i] = 0;  // shares nothing
      continue;
    }
    const uint32_t p = parents[i], c = children[i];
    s.lengths[c] = len;
    if (need)
      fork_last(s, c, len, rank, s.tables[(uint64_t)p * s.max_blocks + len / bs], s.list_a[rank], bs, nb,
                holder);
  }
}

// One contiguous piece of a block's chunk in one plane, `n` 16-byte words:
// eight loads of a thread are in flight before its first store.
__device__ __forceinline__ void copy_words(const u32x4* __restrict__ src, u32x4* __restrict__ dst,
                                           uint32_t n) {
  uint32_t v = threadIdx.x;
  for (; v + 7 * kCopy < n; v += 8 * kCopy) {
    u32x4 r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = src[v + j * kCopy];
#pragma unroll
    for (int j = 0; j < 8; ++j) dst[v + j * kCopy] = r[j];
  }
  u32x4 r[7];
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (v + j * kCopy < n) r[j] = src[v + j * kCopy];
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (v + j * kCopy < n) dst[v + j * kCopy] = r[j];
}

__device__ void copy_pairs(u32x4* kv, const CopyShape& c, const uint32_t* src, const uint32_t* dst,
                           uint32_t pairs, uint32_t first, uint32_t stride) {
  const uint64_t items = (uint64_t)pairs * c.planes * c.pieces;
  for (uint64_t it = first; it < items; it += stride) {
    const uint32_t piece = (uint32_t)(it % c.pieces);
    const uint64_t rest = it / c.pieces;
    const uint32_t pair = (uint32_t)(rest % pairs), plane = (uint32_t)(rest / pairs);
    const uint32_t a = src[pair], b = dst[pair];
    if (a >= c.nb || b >= c.nb) continue;
    const uint32_t w0 = piece * c.piece_words;
    const uint32_t n = c.words - w0 < c.piece_words ? c.words - w0 : c.piece_words;
    const uint64_t row = (uint64_t)plane * c.nb;
    copy_words(kv + (row + a) * c.words + w0, kv + (row + b) * c.words + w0, n);
  }
}

// The first n workgroups share the full blocks of one child each; all of them
// copy.  Bound by memory: 64 children of 16 parents, last blocks of 64 planes of 32
// KiB each (256 MB read and written), take 36.8 us: what several children copy
// is read from memory once.
__global__ void __launch_bounds__(kCopy) k_fork_apply(Seqs s, const uint32_t* parents,
                                                      const uint32_t* children, uint32_t n,
                                                      uint32_t bs, CopyShape c, u32x4* kv) {
  for (uint32_t i = blockIdx.x; i < n; i += gridDim.x)
    share_full(s, parents[i], children[i], s.len[i], bs, c.nb, threadIdx.x, kCopy);
  copy_pairs(kv, c, s.list_b, s.list_a, s.head[kPairs], blockIdx.x, gridDim.x);
}

// Bound by memory: 500 blocks of 64 planes of 32 KiB, 2.1 GB read and written, in
// 421 us, 5.0 TB/s.
__global__ void __launch_bounds__(kCopy) k_copy(const uint32_t* src, const uint32_t* dst,
                                                uint32_t n, CopyShape c, u32x4* kv,
                                                uint64_t* holder) {
  if (blockIdx.x == 0)
    for (uint32_t i = threadIdx.x; i < n; i += kCopy)
      if (src[i] < c.nb && dst[i] < c.nb) holder[dst[i]] = 0;
  copy_pairs(kv, c, src, dst, n, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------- free

// One count of block b.  A count that is 0 already stays 0: a step below it is
// taken back, and while steps are below no other finds a count to give up (counts
// are below 2^31, so that a count below 0 has the top bit).
__device__ __forceinline__ void give_up(uint32_t* count) {
  if ((int32_t)atomicSub(count, 1u) <= 0) atomicAdd(count, 1u);
}

// A workgroup frees a row.  All of it is waiting: for the row's number, then its
// length and entries, then the counts.  64 rows of 4 to 44 blocks, each shared by
// four rows: 4.4 us, where a read, compare and
// swap for each count took 6.7 us.
__global__ void __launch_bounds__(kCopy) k_free(Seqs s, const uint32_t* ids, uint32_t bs,
                                                uint32_t nb) {
  const uint32_t r = row_of(ids, blockIdx.x);
  if (r >= s.max_seqs) return;
  __shared__ uint32_t len;
  uint32_t* row = s.tables + (uint64_t)r * s.max_blocks;
  if (threadIdx.x == 0) len = atomicExch(&s.lengths[r], 0u);  // a row named twice is freed once
  uint32_t j = threadIdx.x;
  uint32_t b = j < s.max_blocks ? row[j] : kNone;
  __syncthreads();
  if (len == 0) return;
  const uint64_t blocks = ((uint64_t)len + bs - 1) / bs;
  while (j < s.max_blocks) {
    if (j < blocks && b < nb) give_up(&s.refs[b]);
    row[j] = kNone;
    j += kCopy;
    b = j < s.max_blocks ? row[j] : kNone;
  }
}

// ------------------------------------------------------------------- compact

// How many table entries name each block, as a block with more counts than that is
// held by the program and stays where it is: a claim's or a prefix list's blocks are
// named from outside the tables.  The plan counts in LDS where the pool and the
// tables are small, else two launches ahead of it count in scratch.  A compaction that
// moves nothing, with no count / one in the plan / one in launches: 64 blocks and
// entries 5.0 / 5.6 / 8.3 us, 2000 blocks and 3120 entries 5.0 / 6.2 / 8.8, 8000 and
// 8192 6.2 / 8.2 / 10.1, 16000 and 16384 8.5 / 11.5 / 11.6.
constexpr uint32_t kCounted = 8192;  // blocks, and table entries, that the plan counts itself

__host__ __device__ inline bool plan_counts(uint32_t nb, uint32_t max_seqs, uint32_t max_blocks) {
  return nb <= kCounted && (uint64_t)max_seqs * max_blocks <= kCounted;
}

__global__ void __launch_bounds__(kCopy) k_count_none(uint32_t* counts, uint32_t nb) {
  for (uint64_t b = (uint64_t)blockIdx.x * kCopy + threadIdx.x; b < nb; b += (uint64_t)gridDim.x * kCopy)
    counts[b] = 0;
}

__global__ void __launch_bounds__(kCopy) k_count_entries(Seqs s, uint32_t nb) {
  const uint64_t entries = (uint64_t)s.max_seqs * s.max_blocks;
  for (uint64_t i = (uint64_t)blockIdx.x * kCopy + threadIdx.x; i < entries;
       i += (uint64_t)gridDim.x * kCopy) {
    const uint32_t b = s.tables[i];
    if (b < nb) atomicAdd(&s.map[b], 1u);
  }
}

// Which blocks move, as the header defines it: U blocks in use, those of them at
// or past U that are not held in `list_b`, the first free ones below U in `list_a`,
// pair by pair.  COUNT: entries are counted here, else `map` has their numbers.
// Bound by dependent reads: 2000 blocks and 3120 entries in 7.8 us.
template <bool COUNT>
__global__ void __launch_bounds__(kPlan) k_compact_plan(Seqs s, uint32_t nb, uint64_t* holder,
                                                        uint32_t* moved) {
  __shared__ uint32_t counts[COUNT ? kCounted : 1];
  const Share share = my_share(s.refs, nb);
  if (COUNT) {
    for (uint32_t b = threadIdx.x; b < nb; b += kPlan) counts[b] = 0;
    __syncthreads();
    const uint32_t entries = s.max_seqs * s.max_blocks;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < entries; i += kPlan) {
      const uint32_t b = s.tables[i];
      if (b < nb) atomicAdd(&counts[b], 1u);
    }
    __syncthreads();
  }
  const auto movable = [&](uint32_t b) { return s.refs[b] <= (COUNT ? counts[b] : s.map[b]); };
  uint64_t total;
  const uint32_t before = (uint32_t)block_scan(share.used, &total);
  const uint32_t U = (uint32_t)total;
  // blocks that move, in order
  uint32_t mine = 0;
  for (uint32_t b = share.first > U ? share.first : U; b < share.last; ++b)
    mine += in_use(share, s.refs, b) && movable(b);
  uint64_t pairs_all;
  uint32_t at = (uint32_t)block_scan(mine, &pairs_all);
  const uint32_t pairs = (uint32_t)pairs_all;
  uint32_t used = before;
  for (uint32_t b = share.first; b < share.last; ++b) {
    const bool taken = in_use(share, s.refs, b);
    if (b < U) {
      if (!taken) s.list_a[b - used] = b;  // at least `pairs` of them: U less those in use below U
    } else {
      const bool moves = taken && movable(b);
      // an entry that names a block with no count names nothing
      s.map[b] = taken ? b : kNone;
      if (moves) s.list_b[at++] = b;
    }
    used += taken;
  }
  if (threadIdx.x == 0) {
    s.head[kPairs] = pairs;
    s.head[kUsed] = U;
    if (moved) *moved = pairs;
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < pairs; i += kPlan) {
    const uint32_t to = s.list_a[i], from = s.list_b[i];
    s.map[from] = to;
    s.refs[to] = s.refs[from];
    s.refs[from] = 0;
    holder[to] = 0;
  }
}

// Tables follow and bytes move.  Bound by memory: 1.1 GB of blocks of 61 planes of
// 36 KiB, read and written, in 476 us, 4.6 TB/s.
__global__ void __launch_bounds__(kCopy) k_compact_apply(Seqs s, CopyShape c, u32x4* kv) {
  const uint32_t pairs = s.head[kPairs], U = s.head[kUsed];
  if (pairs == 0) return;
  const uint64_t entries = (uint64_t)s.max_seqs * s.max_blocks;
  for (uint64_t i = (uint64_t)blockIdx.x * kCopy + threadIdx.x; i < entries;
       i += (uint64_t)gridDim.x * kCopy) {
    const uint32_t b = s.tables[i];
    if (b >= U && b < c.nb) s.tables[i] = s.map[b];
  }
  copy_pairs(kv, c, s.list_b, s.list_a, pairs, blockIdx.x, gridDim.x);
}

// --------------------------------------------------------------------- write

struct WriteArgs {
  uint32_t num_seqs, rows, vecs, head_vecs;  // 8-element vectors of a row, of a head
  const uint32_t *ids, *offsets;
  const uint16_t *k, *v;
  uint64_t k_row, k_head, v_row, v_head;  // strides in elements
  bool apart;  // some head does not begin where the one before ends
  float k_scale, v_scale, k_inverse, v_inverse;
  uint32_t bs, nb;
  uint64_t chunk_bytes;
  uint32_t token_bytes;
  uint8_t *k_plane, *v_plane;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// x / scale, rounded as a division is, limited to the largest e4m3 value; NaN
// passes through.  q = x (1 / scale) is off by an ulp or two at most; the
// remainder x - q scale is exact in one fused step, and so corrects it to the
// nearest value (Markstein's division; inverse is 1 / scale rounded to nearest).
// q is kept finite so that the remainder of an overflow is no NaN: it is past
// the limit anyway.  24 prompts of 100 to 1500 rows of 4 heads of 128: 18.8 us
// with the compiler's division, 15.3 us so.
__device__ __forceinline__ float limit_e4m3(float x, float scale, float inverse) {
  const float q = __builtin_amdgcn_fmed3f(x * inverse, -1000.0f, 1000.0f);
  const float y = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
  const float z = __builtin_amdgcn_fmed3f(y, -448.0f, 448.0f);
  return x != x ? x : z;
}

// Four bf16 values (two words) to four e4m3 bytes, to nearest even.
__device__ __forceinline__ uint32_t to_e4m3(uint32_t w0, uint32_t w1, float scale, float inverse) {
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(limit_e4m3(bf16_lo(w0), scale, inverse),
                                          limit_e4m3(bf16_hi(w0), scale, inverse), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(limit_e4m3(bf16_lo(w1), scale, inverse),
                                                   limit_e4m3(bf16_hi(w1), scale, inverse), p, true);
}

// Where a packed row goes: the byte of its token in a plane, or false.
__device__ __forceinline__ bool find_row(const WriteArgs& a, const Seqs& s, uint32_t row, uint64_t* token_at) {
  uint32_t q = row, i = 0, n = 1;
  if (a.offsets) {
    q = wave_find_seq(a.offsets, a.num_seqs, row);
    const uint32_t o = a.offsets[q], e = a.offsets[q + 1];
    if (o > row || e <= row) return false;  // offsets that do not hold the row
    i = row - o;
    n = e - o;
  }
  const uint32_t r = a.ids ? a.ids[q] : q;
  if (r >= s.max_seqs) return false;
  const int64_t pos = (int64_t)s.lengths[r] - n + i;
  if (pos < 0) return false;
  const uint32_t at = (uint32_t)pos / a.bs, token = (uint32_t)pos % a.bs;
  if (at >= s.max_blocks) return false;
  const uint32_t b = s.tables[(uint64_t)r * s.max_blocks + at];
  *token_at = (uint64_t)b * a.chunk_bytes + (uint64_t)token * a.token_bytes;
  return b < a.nb;
}

// A wave takes one row; its lanes take the row's 16-byte vectors, first K's,
// then V's, four each at a time.  The first of them are asked for before the
// row's place is looked up (three to five dependent reads), which does not
// depend on them.  Bound by memory: 24 prompts of 100 to 1500 rows of 4 heads of
// 128 to e4m3 take 15.3 us, 3.7 TB/s read and written.
template <bool E4M3>
__global__ void __launch_bounds__(256) k_write(WriteArgs a, Seqs s) {
  constexpr uint32_t kMany = 4;
  const uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  bool found = false;
  uint64_t base = 0;
  for (uint32_t x0 = 0; x0 < 2 * a.vecs; x0 += 64 * kMany) {
    u32x4 w[kMany];
#pragma unroll
    for (uint32_t j = 0; j < kMany; ++j) {
      const uint32_t x = x0 + 64 * j + lane;
      if (x >= 2 * a.vecs) continue;
      const bool is_v = x >= a.vecs;
      const uint32_t v = is_v ? x - a.vecs : x;
      uint64_t at = 8 * v;  // heads one after another, unless a stride says otherwise
      const uint64_t head_stride = is_v ? a.v_head : a.k_head;
      if (a.apart) {
        const uint32_t head = v / a.head_vecs;
        at = head * head_stride + 8 * (v - head * a.head_vecs);
      }
      w[j] = *(const u32x4*)((is_v ? a.v + row * a.v_row : a.k + row * a.k_row) + at);
    }
    if (x0 == 0) found = find_row(a, s, row, &base);
    if (!found) return;
#pragma unroll
    for (uint32_t j = 0; j < kMany; ++j) {
      const uint32_t x = x0 + 64 * j + lane;
      if (x >= 2 * a.vecs) continue;
      const bool is_v = x >= a.vecs;
      const uint32_t v = is_v ? x - a.vecs : x;
      uint8_t* dst = (is_v ? a.v_plane : a.k_plane) + base;
      if (E4M3) {
        const float scale = is_v ? a.v_scale : a.k_scale, inverse = is_v ? a.v_inverse : a.k_inverse;
        *(u32x2*)(dst + v * 8) = u32x2{to_e4m3(w[j].x, w[j].y, scale, inverse),
                                       to_e4m3(w[j].z, w[j].w, scale, inverse)};
      } else {
        *(u32x4*)(dst + v * 16) = w[j];
      }
    }
  }
}

// ---------------------------------------------------------------------- host

CopyShape copy_shape(const PoolView& p) {
  CopyShape c;
  c.planes = p.layers * p.planes_per_layer;
  c.nb = p.nb;
  c.words = (uint32_t)(p.chunk_bytes / 16);
  const uint32_t most = 8 * kCopy;  // 32 KiB: one round of eight loads a thread
  c.pieces = (c.words + most - 1) / most;
  c.piece_words = (c.words + c.pieces - 1) / c.pieces;
  return c;
}

// Workgroups for at most `items` pieces: eight to a CU read the plan's
// counts and share what there is.
uint32_t copy_grid(const PoolView& p, uint64_t items) {
  const uint64_t most = 8ull * p.cus;
  return (uint32_t)(items < 1 ? 1 : items < most ? items : most);
}

int launched() {
  if (hipGetLastError() != hipSuccess) return CLAIM_EHIP;
  return CLAIM_OK;
}

int check_planned(const claim_pool* P, const claim_seqs* s, uint32_t n) {
  if (!P) return CLAIM_EINVAL;
  const int rc = check_seqs(s);
  if (rc != CLAIM_OK) return rc;
  return !s->work || n > s->max_seqs ? CLAIM_EINVAL : CLAIM_OK;
}

}  // namespace

extern "C" {

int claim_seqs_grow(claim_pool* P, const claim_seqs* s, const uint32_t* ids, const uint32_t* tokens,
                    uint32_t n, uint32_t* status) {
  const int rc = check_planned(P, s, n);
  if (rc != CLAIM_OK || (n && !tokens)) return rc != CLAIM_OK ? rc : CLAIM_EINVAL;
  if (n == 0) return CLAIM_OK;
  const PoolView p = pool_view(P);
  SEQ_HIP(hipSetDevice(p.device));
  hipLaunchKernelGGL(plan_in_registers(n, s->max_seqs) ? k_grow_few : k_grow, dim3(1), dim3(kPlan), 0,
                     p.stream, seqs_dev(s, p.nb), ids, tokens, n, p.bs, p.nb, p.holder, status);
  return launched();
}

int claim_seqs_fork(claim_pool* P, const claim_seqs* s, const uint32_t* parents,
                    const uint32_t* children, uint32_t n, uint32_t* status) {
  const int rc = check_planned(P, s, n);
  if (rc != CLAIM_OK || (n && (!parents || !children))) return rc != CLAIM_OK ? rc : CLAIM_EINVAL;
  if (n == 0) return CLAIM_OK;
  const PoolView p = pool_view(P);
  SEQ_HIP(hipSetDevice(p.device));
  const Seqs d = seqs_dev(s, p.nb);
  const CopyShape c = copy_shape(p);
  if (plan_in_registers(n, s->max_seqs)) {
    hipLaunchKernelGGL(k_fork_few, dim3(1), dim3(kPlan), 0, p.stream, d, parents, children, n, p.bs, p.nb,
                       p.holder, status, c, (u32x4*)p.kv);
    if (fork_alone(c, n, s->max_blocks)) return launched();
  } else {
    hipLaunchKernelGGL(k_fork_plan, dim3(1), dim3(kPlan), 0, p.stream, d, parents, children, n, p.bs, p.nb,
                       p.holder, status);
  }
  hipLaunchKernelGGL(k_fork_apply, dim3(copy_grid(p, (uint64_t)n * c.planes * c.pieces)),
                     dim3(kCopy), 0, p.stream, d, parents, children, n, p.bs, c, (u32x4*)p.kv);
  return launched();
}

int claim_seqs_free(claim_pool* P, const claim_seqs* s, const uint32_t* ids, uint32_t n) {
  if (!P) return CLAIM_EINVAL;
  const int rc = check_seqs(s);
  if (rc != CLAIM_OK || n > s->max_seqs) return rc != CLAIM_OK ? rc : CLAIM_EINVAL;
  if (n == 0) return CLAIM_OK;
  const PoolView p = pool_view(P);
  SEQ_HIP(hipSetDevice(p.device));
  Seqs d{};
  d.max_seqs = s->max_seqs;
  d.max_blocks = s->max_blocks;
  d.tables = s->tables;
  d.lengths = s->lengths;
  d.refs = s->refs;
  hipLaunchKernelGGL(k_free, dim3(n), dim3(kCopy), 0, p.stream, d, ids, p.bs, p.nb);
  return launched();
}

int claim_seqs_compact(claim_pool* P, const claim_seqs* s, uint32_t* moved) {
  const int rc = check_planned(P, s, 0);
  if (rc != CLAIM_OK) return rc;
  const PoolView p = pool_view(P);
  SEQ_HIP(hipSetDevice(p.device));
  const Seqs d = seqs_dev(s, p.nb);
  if (plan_counts(p.nb, s->max_seqs, s->max_blocks)) {
    hipLaunchKernelGGL(k_compact_plan<true>, dim3(1), dim3(kPlan), 0, p.stream, d, p.nb, p.holder, moved);
  } else {
    const uint64_t blocks = ((uint64_t)p.nb + kCopy - 1) / kCopy;
    const uint64_t entries = ((uint64_t)s->max_seqs * s->max_blocks + kCopy - 1) / kCopy;
    hipLaunchKernelGGL(k_count_none, dim3(copy_grid(p, blocks)), dim3(kCopy), 0, p.stream, d.map, p.nb);
    hipLaunchKernelGGL(k_count_entries, dim3(copy_grid(p, entries)), dim3(kCopy), 0, p.stream, d, p.nb);
    hipLaunchKernelGGL(k_compact_plan<false>, dim3(1), dim3(kPlan), 0, p.stream, d, p.nb, p.holder, moved);
  }
  const CopyShape c = copy_shape(p);
  const uint64_t most = (uint64_t)(p.nb / 2 + 1) * c.planes * c.pieces;
  hipLaunchKernelGGL(k_compact_apply, dim3(copy_grid(p, most)), dim3(kCopy), 0, p.stream, d, c,
                     (u32x4*)p.kv);
  return launched();
}

int claim_blocks_copy(claim_pool* P, const uint32_t* src, const uint32_t* dst, uint32_t n) {
  if (!P || (n && (!src || !dst))) return CLAIM_EINVAL;
  const PoolView p = pool_view(P);
  if (n > p.nb) return CLAIM_EINVAL;  // some block would be written twice
  if (n == 0) return CLAIM_OK;
  SEQ_HIP(hipSetDevice(p.device));
  const CopyShape c = copy_shape(p);
  hipLaunchKernelGGL(k_copy, dim3(copy_grid(p, (uint64_t)n * c.planes * c.pieces)), dim3(kCopy), 0,
                     p.stream, src, dst, n, c, (u32x4*)p.kv, p.holder);
  return launched();
}

int claim_kv_write(claim_pool* P, const claim_seqs* s, const claim_kv_desc* kv, const claim_rows* k,
                   const claim_rows* v) {
  if (!P || !kv || !k || !v) return CLAIM_EINVAL;
  const PoolView p = pool_view(P);
  int rc = check_seqs(s);
  if (rc == CLAIM_OK) rc = check_kv(p, s, kv);
  if (rc != CLAIM_OK) return rc;
  if (p.dim % 8) return CLAIM_EINVAL;
  if (kv->num_rows == 0) return CLAIM_OK;
  if (!rows_ok(*k) || !rows_ok(*v)) return CLAIM_EINVAL;
  SEQ_HIP(hipSetDevice(p.device));
  WriteArgs a;
  a.num_seqs = kv->num_seqs;
  a.rows = kv->num_rows;
  a.head_vecs = p.dim / 8;
  a.vecs = p.heads * a.head_vecs;
  a.ids = kv->ids;
  a.offsets = kv->offsets;
  a.k = (const uint16_t*)k->data;
  a.v = (const uint16_t*)v->data;
  a.k_row = k->row_stride;
  a.k_head = k->head_stride;
  a.v_row = v->row_stride;
  a.v_head = v->head_stride;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.k_inverse = 1.0f / kv->k_scale;
  a.v_inverse = 1.0f / kv->v_scale;
  a.apart = p.heads > 1 && (k->head_stride != p.dim || v->head_stride != p.dim);
  a.bs = p.bs;
  a.nb = p.nb;
  a.chunk_bytes = p.chunk_bytes;
  a.token_bytes = (uint32_t)(p.chunk_bytes / p.bs);
  const uint64_t plane = (uint64_t)p.nb * p.chunk_bytes;
  a.k_plane = p.kv + 2ull * kv->layer * plane;
  a.v_plane = a.k_plane + plane;
  Seqs d{};
  d.max_seqs = s->max_seqs;
  d.max_blocks = s->max_blocks;
  d.tables = s->tables;
  d.lengths = s->lengths;
  const dim3 grid((kv->num_rows + 3) / 4);
  if (p.elem == 1)
    hipLaunchKernelGGL(k_write<true>, grid, dim3(256), 0, p.stream, a, d);
  else
    hipLaunchKernelGGL(k_write<false>, grid, dim3(256), 0, p.stream, a, d);
  return launched();
}

}  // extern "C"
