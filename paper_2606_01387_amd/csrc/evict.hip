// evict.hip -- sequences cut to their first tokens, their last ones, and of the
// others those of the most weight (gfx950).
//
// Three launches: each sequence's choice (a workgroup a sequence), the plan of the
// blocks that shared ones need in their place (one workgroup), and the move of the
// bytes, tables, counts and weights.  Every rank is a count or a prefix sum, so
// results do not depend on the order in which lanes or atomics run; nothing comes
// back to the host.

#include "block_plan.h"

namespace {

enum : uint32_t { kCut = 0, kShort = 1, kNoRoom = 2, kRefused = 3 };

// What is known of an entry.
struct Entry {
  uint32_t state;  // one of the above
  uint32_t len;    // tokens before
  uint32_t first;  // the first block that changes
  uint32_t stay;   // tokens at the front that stay where they are
  uint32_t need;   // blocks needed in place of shared ones
  uint32_t rank;   // where those begin in the list of free ones
  uint32_t unused[2];
};

struct EvictArgs {
  Seqs s;
  const uint32_t* ids;
  uint32_t n, tokens, sinks, recent;
  float* weights;
  uint64_t weights_row;
  uint32_t *kept, *status;
  Entry* entries;   // [n]
  uint32_t* from;   // [n][max_blocks]: the rows of tables before
  uint32_t* place;  // [n][blocks]: 0: where it is; else the how-manieth needed block, from 1
  uint32_t blocks;  // blocks of `tokens`
  uint32_t bs, nb;
  uint64_t* holder;
  // bytes
  uint8_t* kv;
  uint64_t plane_bytes, chunk_bytes;
  uint32_t planes, token_bytes, token_units, width, slices;
};

// A weight as a number of the same order: NaN lowest, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0;
  const uint32_t b = w == 0.0f ? 0 : __float_as_uint(w);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A thread's weights as numbers: wave w has a run of positions, its lanes the run's
// 64 at a time.  The first of them stay in registers from one look to the next.
constexpr uint32_t kNear = 8;

struct Numbers {
  const float* w;
  uint32_t begin, end, run;  // the wave's positions; run: a multiple of 64
  uint32_t near[kNear];

  __device__ __forceinline__ void start(const float* weights, uint32_t len) {
    w = weights;
    run = (len / kPlan + 1) * 64;
    begin = threadIdx.x / 64 * run;
    begin = begin < len ? begin : len;
    end = len - begin < run ? len : begin + run;
    float x[kNear];  // all of them on their way at once
#pragma unroll
    for (uint32_t k = 0; k < kNear; ++k) {
      const uint32_t p = begin + 64 * k + threadIdx.x % 64;
      x[k] = p < end && 64 * k < run ? w[p] : 0.0f;
    }
#pragma unroll
    for (uint32_t k = 0; k < kNear; ++k) near[k] = order_of(x[k]);
  }

  // f(position, number) for each 64 positions of the wave, all lanes together.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    const uint32_t lane = threadIdx.x % 64;
#pragma unroll
    for (uint32_t k = 0; k < kNear; ++k)
      if (begin + 64 * k < end) f(begin + 64 * k + lane, near[k]);
    for (uint32_t p = begin + 64 * kNear; p < end; p += 64) f(p + lane, p + lane < end ? order_of(w[p + lane]) : 0);
  }
};

// The k-th largest (k >= 1) of the numbers at lo .. hi - 1, by their digits from the
// highest on; *equal is how many of that very number are among the k.
__device__ uint32_t kth_largest(const Numbers& numbers, uint32_t lo, uint32_t hi, uint32_t k, uint32_t* equal) {
  __shared__ uint32_t count[2048];
  __shared__ uint32_t found, left;
  const uint32_t t = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  for (int digit = 0; digit < 3; ++digit) {
    const uint32_t shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : 2048;
    count[t] = count[t + kPlan] = 0;
    __syncthreads();
    numbers.each([&](uint32_t p, uint32_t x) {
      if (p >= lo && p < hi && (x & mask) == prefix) atomicAdd(&count[x >> shift & (bins - 1)], 1u);
    });
    __syncthreads();
    // thread t has the bins bins - 1 - 2 t and the one below
    const uint32_t a = 2 * t < bins ? count[bins - 1 - 2 * t] : 0, b = 2 * t < bins ? count[bins - 2 - 2 * t] : 0;
    uint64_t total;
    const uint32_t before = (uint32_t)block_scan((uint64_t)a + b, &total);
    if (before < k && k <= before + a + b) {
      const bool upper = k <= before + a;
      found = upper ? bins - 1 - 2 * t : bins - 2 - 2 * t;
      left = k - before - (upper ? 0 : a);
    }
    __syncthreads();
    prefix |= found << shift;
    mask |= (bins - 1) << shift;
    k = left;
    __syncthreads();
  }
  *equal = k;
  return prefix;
}

// Whether an earlier entry names the same row: each workgroup looks through the
// entries before its own where they are few, else two launches have left the first
// entry of every row in `owner` (a look through n entries by n workgroups takes n^2).
constexpr uint32_t kLookThrough = 4096;

__global__ void __launch_bounds__(256) k_owner_none(uint32_t* owner, const uint32_t* ids, uint32_t n,
                                                    uint32_t max_seqs) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256)
    if (ids[i] < max_seqs) owner[ids[i]] = kNone;
}

__global__ void __launch_bounds__(256) k_owner_first(uint32_t* owner, const uint32_t* ids, uint32_t n,
                                                     uint32_t max_seqs) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256)
    if (ids[i] < max_seqs) atomicMin(&owner[ids[i]], i);
}

// A workgroup chooses what an entry keeps: the weights above the last that has a
// place, and of those equal to it the first ones.  Waves take runs of positions,
// count, and then write what they keep in order.  Bound by dependent reads (length,
// table and weights, counts) and the digits' barriers: 11 us for 200 tokens, 16 us
// for 4000, 32 for 16000; 61 us for 16000 of one weight, which are counted in one place.
__global__ void __launch_bounds__(kPlan) k_evict_select(EvictArgs a) {
  __shared__ uint32_t above[kPlan / 64], same[kPlan / 64], gone;
  const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
  for (uint32_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const uint32_t r = row_of(a.ids, i);
    bool bad = r >= a.s.max_seqs;
    if (a.ids && !bad) {
      if (a.n > kLookThrough)
        bad = a.s.owner[r] != i;
      else
        for (uint32_t k = t; k < i; k += kPlan) bad |= a.ids[k] == r;
    }
    const uint32_t len = r < a.s.max_seqs ? a.s.lengths[r] : 0;
    const uint32_t held = len / a.bs + (len % a.bs != 0);
    bad |= held > a.s.max_blocks;
    const bool cut = !bad && len > a.tokens;
    Numbers numbers;
    numbers.start(a.weights + (r < a.s.max_seqs ? r : 0) * a.weights_row, cut ? len : 0);
    uint32_t* from = a.from + (uint64_t)i * a.s.max_blocks;
    if (!bad)
      for (uint32_t j = t; j < held; j += kPlan) {
        const uint32_t b = a.s.tables[(uint64_t)r * a.s.max_blocks + j];
        from[j] = b;
        bad |= b >= a.nb;
      }
    bad = __syncthreads_or(bad);
    uint32_t* kept = a.kept + (uint64_t)i * a.tokens;
    if (bad || len <= a.tokens) {
      for (uint32_t j = t; j < a.tokens; j += kPlan) kept[j] = !bad && j < len ? j : kNone;
      if (t == 0) a.entries[i] = Entry{bad ? kRefused : kShort, len, 0, 0, 0, 0, {}};
      continue;
    }
    const uint32_t lo = a.sinks, hi = len - a.recent, m = a.tokens - a.sinks - a.recent;
    uint32_t least = ~0u, equal = 0;  // (no weight has the highest number)
    if (m) least = kth_largest(numbers, lo, hi, m, &equal);
    const auto kind = [&](uint32_t p, uint32_t x) {  // 0: goes, 1: equal to the least, 2: stays
      return p >= numbers.end ? 0 : p < lo || p >= hi || x > least ? 2 : x == least ? 1 : 0;
    };
    uint32_t more = 0, ties = 0;
    numbers.each([&](uint32_t p, uint32_t number) {
      const int x = kind(p, number);
      more += __popcll(__ballot(x == 2));
      ties += __popcll(__ballot(x == 1));
    });
    if (lane == 0) {
      above[wave] = more;
      same[wave] = ties;
    }
    if (t == 0) gone = len;
    __syncthreads();
    uint32_t at = 0, tied = 0;
    for (uint32_t k = 0; k < wave; ++k) {
      at += above[k];
      tied += same[k];
    }
    at += tied < equal ? tied : equal;
    const uint64_t below = (1ull << lane) - 1;
    uint32_t mine = len;  // the first position that goes
    numbers.each([&](uint32_t p, uint32_t number) {
      const int x = kind(p, number);
      const uint64_t t1 = __ballot(x == 1);
      const bool stays = x == 2 || (x == 1 && tied + __popcll(t1 & below) < equal);
      const uint64_t k1 = __ballot(stays);
      if (stays) kept[at + __popcll(k1 & below)] = p;
      if (!stays && p < numbers.end && p < mine) mine = p;
      at += __popcll(k1);
      tied += __popcll(t1);
    });
    if (mine < len) atomicMin(&gone, mine);
    __syncthreads();
    const uint32_t stay = gone < a.tokens ? gone : a.tokens;
    // a last block that is not full will be written: it must be the sequence's own
    const bool writes = stay < a.tokens || a.tokens % a.bs;
    const uint32_t first = writes ? (stay < a.tokens ? stay : a.tokens - 1) / a.bs : a.blocks;
    if (wave == 0) {
      uint32_t need = 0;
      for (uint32_t j = first; j < a.blocks; j += 64) {
        const bool shared = j + lane < a.blocks && a.s.refs[from[j + lane]] > 1;
        const uint64_t b = __ballot(shared);
        if (j + lane < a.blocks)
          a.place[(uint64_t)i * a.blocks + j + lane] = shared ? need + __popcll(b & below) + 1 : 0;
        need += __popcll(b);
      }
      if (lane == 0) a.entries[i] = Entry{kCut, len, first, stay, need, 0, {}};
    }
    __syncthreads();
  }
}

// Which entries get the blocks that they need: those that the free ones reach for, in
// order of the entries.
__global__ void __launch_bounds__(kPlan) k_evict_plan(EvictArgs a) {
  uint64_t run = 0;
  for (uint32_t i0 = 0; i0 < a.n; i0 += kPlan) {
    const uint32_t i = i0 + threadIdx.x;
    uint64_t total;
    const uint64_t at = run + block_scan(i < a.n ? a.entries[i].need : 0, &total);
    if (i < a.n) a.entries[i].rank = at < a.nb ? (uint32_t)at : a.nb;  // the free ones are fewer
    run += total;
  }
  const uint64_t free_all = run ? list_free(my_share(a.s.refs, a.nb), a.s.refs, run, a.s.list_a) : 0;
  for (uint32_t i = threadIdx.x; i < a.n; i += kPlan) {
    Entry& e = a.entries[i];
    if (e.state == kCut && e.need && (uint64_t)e.rank + e.need > free_all) e.state = kNoRoom;
    if (a.status)
      a.status[i] = e.state == kRefused ? CLAIM_SEQ_REFUSED : e.state == kNoRoom ? CLAIM_SEQ_NO_BLOCKS : CLAIM_SEQ_OK;
  }
}

constexpr int kMove = 256;     // threads of a moving workgroup
constexpr uint32_t kHeld = 8;  // what a thread holds at a time

// An entry's table, counts, length and weights.
__device__ void move_entry(const EvictArgs& a, uint32_t i, const Entry& e) {
  const uint32_t t = threadIdx.x, r = row_of(a.ids, i);
  const uint32_t* from = a.from + (uint64_t)i * a.s.max_blocks;
  uint32_t* table = a.s.tables + (uint64_t)r * a.s.max_blocks;
  const uint32_t held = e.len / a.bs + (e.len % a.bs != 0);
  for (uint32_t j = e.first + t; j < held; j += kMove) {
    const uint32_t place = j < a.blocks ? a.place[(uint64_t)i * a.blocks + j] : 0;
    if (j >= a.blocks) {
      table[j] = kNone;
      give_up(&a.s.refs[from[j]]);
    } else if (place) {
      const uint32_t b = a.s.list_a[e.rank + place - 1];
      table[j] = b;
      a.s.refs[b] = 1;
      a.holder[b] = 0;
      give_up(&a.s.refs[from[j]]);
    } else {
      a.holder[from[j]] = 0;  // other bytes than its identity's
    }
  }
  if (t == 0) a.s.lengths[r] = a.tokens;
  // weights go down, never up: what is read next is not written yet
  const uint32_t* kept = a.kept + (uint64_t)i * a.tokens;
  float* w = a.weights + r * a.weights_row;
  for (uint32_t j0 = e.stay; j0 < a.tokens; j0 += kMove * kHeld) {
    float x[kHeld];
#pragma unroll
    for (uint32_t k = 0; k < kHeld; ++k) {
      const uint32_t j = j0 + k * kMove + t;
      if (j < a.tokens) x[k] = w[kept[j]];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kHeld; ++k) {
      const uint32_t j = j0 + k * kMove + t;
      if (j < a.tokens) w[j] = x[k];
    }
  }
  __syncthreads();
  for (uint32_t j = a.tokens + t; j < e.len; j += kMove) w[j] = 0.0f;
}

// Workgroups move tokens down in their blocks: each one slice of a token's bytes in
// one plane, all of a sequence's tokens in order.  The j-th token kept comes from
// position j or later, so a token that is still to be read lies behind all that
// have been written, and a batch is safe to write once all of it has been read.
// Bound by memory: 8 sequences cut to 2048 tokens of 32 planes of 2 KiB, 2.1 GB read
// and written but for what stays, in 450 us (98 % of a copy's rate; 461 us with loads
// and stores that the caches keep, which hold a small part of it).
template <typename V>
__global__ void __launch_bounds__(kMove) k_evict_move(EvictArgs a) {
  constexpr uint32_t kBatch = kMove / 4 * kHeld;  // slices are 4 units wide at least
  __shared__ uint64_t source[kBatch], target[kBatch];
  const uint32_t t = threadIdx.x, units = a.planes * a.slices + 1;
  const uint64_t items = (uint64_t)a.n * units;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t i = (uint32_t)(item / units), unit = (uint32_t)(item - (uint64_t)i * units);
    const Entry e = a.entries[i];
    if (e.state == kNoRoom && unit == 0)
      for (uint32_t j = t; j < a.tokens; j += kMove) a.kept[(uint64_t)i * a.tokens + j] = kNone;
    if (e.state != kCut) continue;
    if (unit == 0) {
      move_entry(a, i, e);
      continue;
    }
    const uint32_t plane = (unit - 1) / a.slices, slice = (unit - 1) - plane * a.slices;
    uint8_t* base = a.kv + plane * a.plane_bytes;
    const uint32_t *from = a.from + (uint64_t)i * a.s.max_blocks, *place = a.place + (uint64_t)i * a.blocks;
    const uint32_t* kept = a.kept + (uint64_t)i * a.tokens;
    const uint32_t at_once = kMove / a.width, batch = at_once * kHeld;  // tokens
    const uint32_t column = slice * a.width + t % a.width, lane_token = t / a.width;
    const bool in = column < a.token_units;
    for (uint32_t j0 = e.first * a.bs; j0 < a.tokens; j0 += batch) {
      __syncthreads();
      for (uint32_t k = t; k < batch; k += kMove) {
        const uint32_t j = j0 + k;
        uint64_t src = 0, dst = ~0ull;
        if (j < a.tokens) {
          const uint32_t p = kept[j], to = j / a.bs, sb = p / a.bs, moved = place[to];
          if (p != j || moved) {
            src = from[sb] * a.chunk_bytes + (uint64_t)(p - sb * a.bs) * a.token_bytes;
            dst = (moved ? a.s.list_a[e.rank + moved - 1] : from[to]) * a.chunk_bytes +
                  (uint64_t)(j - to * a.bs) * a.token_bytes;
          }
        }
        source[k] = src;
        target[k] = dst;
      }
      __syncthreads();
      V held[kHeld];
      uint64_t dst[kHeld];
#pragma unroll
      for (uint32_t k = 0; k < kHeld; ++k) {
        dst[k] = in ? target[k * at_once + lane_token] : ~0ull;
        if (dst[k] != ~0ull)
          held[k] = __builtin_nontemporal_load((const V*)(base + source[k * at_once + lane_token] +
                                                          (uint64_t)column * sizeof(V)));
      }
#pragma unroll
      for (uint32_t k = 0; k < kHeld; ++k) asm volatile("" : "+v"(held[k]));  // all of them have arrived
      __syncthreads();
#pragma unroll
      for (uint32_t k = 0; k < kHeld; ++k)
        if (dst[k] != ~0ull)
          __builtin_nontemporal_store(held[k], (V*)(base + dst[k] + (uint64_t)column * sizeof(V)));
    }
  }
}

// --------------------------------------------------------------------- host

int check_evict(const PoolView& p, const claim_seqs* s, const claim_evict_desc* d) {
  const int rc = check_seqs(s);
  if (rc != CLAIM_OK) return rc;
  if (!s->work || d->n > s->max_seqs) return CLAIM_EINVAL;
  if (d->tokens == 0 || d->tokens > 0x7FFFFFFFu || (uint64_t)d->sinks + d->recent > d->tokens) return CLAIM_EINVAL;
  const uint64_t room = (uint64_t)s->max_blocks * p.bs;
  if (room > 0x7FFFFFFFull || d->weights_stride < room || ((uintptr_t)d->weights & 3)) return CLAIM_EINVAL;
  if ((p.chunk_bytes / p.bs) % 8) return CLAIM_EINVAL;
  return CLAIM_OK;
}

uint32_t blocks_of(const PoolView& p, const claim_seqs* s, const claim_evict_desc* d) {
  const uint32_t blocks = d->tokens / p.bs + (d->tokens % p.bs != 0);
  return blocks < s->max_blocks ? blocks : s->max_blocks;
}

}  // namespace

extern "C" {

int claim_seqs_evict_work(const claim_pool* P, const claim_seqs* s, const claim_evict_desc* d, uint64_t* bytes) {
  if (!P || !d || !bytes) return CLAIM_EINVAL;
  const PoolView p = pool_view(P);
  const int rc = check_evict(p, s, d);
  if (rc != CLAIM_OK) return rc;
  *bytes = (uint64_t)d->n * (sizeof(Entry) + 4ull * s->max_blocks + 4ull * blocks_of(p, s, d));
  return CLAIM_OK;
}

int claim_seqs_evict(claim_pool* P, const claim_seqs* s, const claim_evict_desc* d) {
  uint64_t need;
  const int rc = claim_seqs_evict_work(P, s, d, &need);
  if (rc != CLAIM_OK || d->n == 0) return rc;
  if (!d->weights || !d->kept || ((uintptr_t)d->kept & 3) || ((uintptr_t)d->work & 255)) return CLAIM_EINVAL;
  if (!d->work || d->work_bytes < need) return CLAIM_ENOSPC;
  const PoolView p = pool_view(P);
  EvictArgs a{};
  a.s = seqs_dev(s, p.nb);
  a.ids = d->ids;
  a.n = d->n;
  a.tokens = d->tokens;
  a.sinks = d->sinks;
  a.recent = d->recent;
  a.weights = d->weights;
  a.weights_row = d->weights_stride;
  a.kept = d->kept;
  a.status = d->status;
  a.blocks = blocks_of(p, s, d);
  a.entries = (Entry*)d->work;
  a.from = (uint32_t*)(a.entries + d->n);
  a.place = a.from + (uint64_t)d->n * s->max_blocks;
  a.bs = p.bs;
  a.nb = p.nb;
  a.holder = p.holder;
  a.kv = p.kv;
  a.chunk_bytes = p.chunk_bytes;
  a.plane_bytes = (uint64_t)p.nb * p.chunk_bytes;
  a.planes = p.layers * p.planes_per_layer;
  a.token_bytes = (uint32_t)(p.chunk_bytes / p.bs);
  const bool wide = a.token_bytes % 16 == 0;
  a.token_units = a.token_bytes / (wide ? 16 : 8);
  // slices as wide as a token, narrower where that leaves CUs idle
  a.width = 4;
  while (a.width < 64 && a.width < a.token_units) a.width *= 2;
  while (a.width > 16 && (uint64_t)d->n * a.planes * ((a.token_units + a.width - 1) / a.width) < 4ull * p.cus)
    a.width /= 2;
  a.slices = (a.token_units + a.width - 1) / a.width;
  SEQ_HIP(hipSetDevice(p.device));
  if (d->ids && d->n > kLookThrough) {
    const dim3 some(4 * p.cus);
    hipLaunchKernelGGL(k_owner_none, some, dim3(256), 0, p.stream, a.s.owner, d->ids, d->n, s->max_seqs);
    hipLaunchKernelGGL(k_owner_first, some, dim3(256), 0, p.stream, a.s.owner, d->ids, d->n, s->max_seqs);
  }
  hipLaunchKernelGGL(k_evict_select, dim3(d->n < 65536 ? d->n : 65536), dim3(kPlan), 0, p.stream, a);
  hipLaunchKernelGGL(k_evict_plan, dim3(1), dim3(kPlan), 0, p.stream, a);
  const uint64_t items = (uint64_t)d->n * (a.planes * (uint64_t)a.slices + 1), most = 16ull * p.cus;
  const dim3 grid((uint32_t)(items < most ? items : most));
  if (wide)
    hipLaunchKernelGGL(k_evict_move<u32x4>, grid, dim3(kMove), 0, p.stream, a);
  else
    hipLaunchKernelGGL(k_evict_move<u32x2>, grid, dim3(kMove), 0, p.stream, a);
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
}

}  // extern "C"
