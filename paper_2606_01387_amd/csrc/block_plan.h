// block_plan.h -- planning which blocks go where, by one workgroup (library-internal).
#ifndef CLAIMKV_BLOCK_PLAN_H
#define CLAIMKV_BLOCK_PLAN_H

#include "pool_view.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kNone = CLAIM_NONE;
constexpr int kPlan = 1024;  // threads of a planning workgroup

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

// One count of block b.  A count that is 0 already stays 0: a step below it is
// taken back, and while steps are below no other finds a count to give up (counts
// are below 2^31, so that a count below 0 has the top bit).
__device__ __forceinline__ void give_up(uint32_t* count) {
  if ((int32_t)atomicSub(count, 1u) <= 0) atomicAdd(count, 1u);
}

}  // namespace

#endif
