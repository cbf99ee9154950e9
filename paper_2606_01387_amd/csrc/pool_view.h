// pool_view.h -- what the sequence operators see of a pool (library-internal).
#ifndef CLAIMKV_POOL_VIEW_H
#define CLAIMKV_POOL_VIEW_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "claimkv.h"

struct PoolView {
  int device;
  hipStream_t stream;
  uint32_t cus;
  uint32_t layers, planes_per_layer, bs, heads, dim, elem, nb;
  uint64_t chunk_bytes;
  uint8_t* kv;       // [plane][block][chunk]
  uint64_t* holder;  // per block: the identity it holds (0: none)
};

__attribute__((visibility("hidden"))) PoolView pool_view(const claim_pool* P);

// Host-side checks shared by the sequence operators.  The counts are limited so
// that a launch of one workgroup a row, a sequence or a tile of theirs has fewer
// than 2^32 threads.
constexpr uint32_t kMostSeqs = 1u << 22, kMostRows = 1u << 25;

inline int check_seqs(const claim_seqs* s) {
  if (!s || s->max_seqs == 0 || s->max_blocks == 0 || !s->tables || !s->lengths || !s->refs)
    return CLAIM_EINVAL;
  if (s->max_seqs > kMostSeqs || (uint64_t)s->max_seqs * s->max_blocks > (1ull << 40))
    return CLAIM_EINVAL;
  return CLAIM_OK;
}

inline bool finite_positive(float x) { return x > 0.0f && x <= 3.4e38f; }

// A scale of e4m3 bytes: its inverse and its product with a byte are finite.
inline bool scale_ok(float x) { return x >= 1e-30f && x <= 1e30f; }

inline int check_kv(const PoolView& p, const claim_seqs* s, const claim_kv_desc* kv) {
  if (kv->reserved != 0 || p.planes_per_layer != 2 || kv->layer >= p.layers ||
      (p.elem != 1 && p.elem != 2) || kv->num_seqs > s->max_seqs || kv->num_rows > kMostRows)
    return CLAIM_EINVAL;
  if (!kv->offsets && kv->num_rows != kv->num_seqs) return CLAIM_EINVAL;
  if (kv->num_rows > 0 && kv->num_seqs == 0) return CLAIM_EINVAL;
  if (p.elem == 2 ? kv->k_scale != 1.0f || kv->v_scale != 1.0f
                  : !scale_ok(kv->k_scale) || !scale_ok(kv->v_scale))
    return CLAIM_EINVAL;
  return CLAIM_OK;
}

inline bool rows_ok(const claim_rows& r) {
  return r.data && ((uintptr_t)r.data & 15) == 0 && r.row_stride % 8 == 0 && r.head_stride % 8 == 0;
}

#define SEQ_HIP(expr)                                   \
  do {                                                  \
    if ((expr) != hipSuccess) {                         \
      (void)hipGetLastError();                          \
      return CLAIM_EHIP;                                \
    }                                                   \
  } while (0)

// The packed row that `row` is: its sequence among n (binary search of the
// first rows, 64 at a time: lane k tests one of 64 evenly spaced sequences,
// so 4096 sequences take two dependent loads).  `off` holds n + 1 first
// rows; all lanes of the wave call it with the same `row`.  The answer is in
// [0, n) whatever `off` holds.
__device__ __forceinline__ uint32_t wave_find_seq(const uint32_t* off, uint32_t n, uint32_t row) {
  uint32_t lo = 0, hi = n;  // the last s in [lo, hi) with off[s] <= row, else lo
  const uint32_t lane = threadIdx.x & 63;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64;
    const uint32_t s = lo + lane * step;
    const bool below = s < hi && off[s] <= row;
    const uint64_t m = __ballot(below);
    const uint32_t k = m ? 63u - (uint32_t)__builtin_clzll(m) : 0u;
    lo += k * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return lo;
}

#endif
