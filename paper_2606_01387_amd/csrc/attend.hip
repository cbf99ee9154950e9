// attend.hip -- attention over a pool's blocks (gfx950): rows of queries that
// follow or end their sequences' tokens, single tokens of a decoding batch, and
// batches that share a prefix.
//
// The rows' walk over their keys, with the products and the running softmax, is in
// attend_rows.h.

#include "attend_rows.h"

namespace {

template <int D, bool E4M3, int WAVES, Within WITHIN>
__global__ void __launch_bounds__(WAVES * 64, 2) k_attend_rows(Args a, uint32_t prefix) {
  __shared__ typename Many<D, WAVES>::Lds shared;
  many_rows<D, E4M3, WAVES, WITHIN>(a, prefix, blockIdx.x, shared);
}

// Items of a shared prefix (32 rows each) and of the sequences' own keys (16
// QT rows) in one launch, eight of the one kind and eight of the other in
// turn: the first are bound by products and weights, the second by memory, and
// two workgroups share a CU.
template <int D, bool E4M3, Within WITHIN, int QT>
__global__ void __launch_bounds__(256, 2) k_attend_few(Args a, uint32_t prefix_items, uint32_t own_items) {
  __shared__ typename Few<D, E4M3, 4>::Lds shared;
  const uint32_t b = blockIdx.x, of8 = b / 8;
  const uint32_t prefix8 = (prefix_items + 7) / 8, own8 = (own_items + 7) / 8;
  const uint32_t both = prefix8 < own8 ? prefix8 : own8;
  const bool prefix = of8 < 2 * both ? of8 % 2 == 0 : prefix8 > own8;
  const uint32_t item = (of8 < 2 * both ? of8 / 2 : of8 - both) * 8 + b % 8;
  if (item >= (prefix ? prefix_items : own_items)) return;
  if (prefix)
    few_rows<D, E4M3, 4, WITHIN, 2>(a, true, item, shared);
  else
    few_rows<D, E4M3, 4, WITHIN, QT>(a, false, item, shared);
}

// Items of a long prefix by many_rows and items of the sequences' own keys by
// few_rows with eight waves, in one launch: the first keep the matrix cores of
// some CUs busy and little memory, the second memory, and CUs that are done with
// the one kind take up the other.  The prefix's items, which are the longer ones,
// begin where they leave a quarter of the CUs to the others, else they come last:
// 128 of them and 512 of nothing 32 us first and 41 us last, 252 and 200 of up to
// 2000 e4m3 tokens 55 us first and 51 us last.  64 sequences of up to 1024 own tokens behind
// 8192, 8 KV heads of 128 for 4 query heads each: 60 us, where the two
// kinds one after another take 41 and 27 us.
template <int D, bool E4M3, Within WITHIN>
__global__ void __launch_bounds__(512, 2) k_attend_both(Args a, uint32_t prefix_items, bool prefix_first) {
  __shared__ union {
    typename Many<D, 8>::Lds many;
    typename Few<D, E4M3, 8>::Lds few;
  } shared;
  const uint32_t b = blockIdx.x, own_items = gridDim.x - prefix_items;
  const uint32_t prefix_from = prefix_first ? 0 : own_items, own_from = prefix_first ? prefix_items : 0;
  if (prefix_first ? b < prefix_items : b >= own_items)
    many_rows<D, E4M3, 8, kLoads>(a, true, b - prefix_from, shared.many);
  else
    few_rows<D, E4M3, 8, WITHIN, 1>(a, false, b - own_from, shared.few);
}

// --------------------------------------------------------------------- host

struct Plan {
  uint32_t columns;    // own keys by few_rows with 16 x columns rows a tile; 0: by many_rows
  bool prefix_narrow;  // the prefix by few_rows, in k_attend_few's launch; else by many_rows
  bool both;           // ... in k_attend_both's launch, with the own keys
  uint32_t own_splits, prefix_splits, tiles, prefix_tiles;
  uint64_t parts;  // parts of all rows and heads; 0: none are kept
};

constexpr uint32_t kPrefixTile = 32;  // of k_attend_few's, for a prefix

Plan make_plan(const PoolView& p, const claim_seqs* s, const claim_attend_desc* d) {
  Plan r{};
  const uint64_t group = d->num_heads / p.heads, rows = d->kv.num_rows, seqs = d->kv.num_seqs;
  const uint64_t prefix = (uint64_t)d->prefix_blocks * p.bs;
  const uint64_t table = (uint64_t)s->max_blocks * p.bs;
  const uint64_t own = table > prefix ? table - prefix : 0;
  const uint64_t each = (rows * group + seqs - 1) / seqs;  // query rows of a sequence
  r.columns = each <= 16 ? 1 : each <= 64 ? 2 : 0;
  const uint32_t M = r.columns ? 16 * r.columns : kRowsTile;
  r.tiles = (uint32_t)(d->kv.offsets ? rows * group / M + seqs : seqs * ((group + M - 1) / M));
  const uint64_t groups = (uint64_t)r.tiles * p.heads;
  if (prefix) {
    // The wide tile is slow to begin (its first keys, then 256 rows of parts to
    // store): half of the CUs with 512 keys each take the time that all take with
    // 256, and leave half the parts to join.  64 sequences of up to 1024 own tokens
    // behind 8192, 8 KV heads of 128 for 4 query heads each: 74.8 us with splits
    // from 256 keys on, 70.1 from 512, 76.7 from 1024 (in launches of their own).
    r.prefix_tiles = (uint32_t)((rows * group + kRowsTile - 1) / kRowsTile);
    r.prefix_splits = splits_for((uint64_t)r.prefix_tiles * p.heads, p.cus, prefix, 512);
    // One launch for both kinds of keys where a CU has two items of own keys at
    // most, as they have a CU to themselves there: the same 70.4 -> 64.2 us, but 256
    // sequences with nothing of their own 75 -> 94 us.
    r.both = r.columns == 1 && one_block_loads(p) && groups <= 2ull * p.cus;
    // Narrow tiles make 0.2 to 0.3 M (query row, key) pairs a microsecond, all CUs
    // together; a wide one, full or not, 32 keys, and 10 us more where it needs a
    // launch of its own.  8192 shared tokens, 8 KV heads for 4 query heads each, 8 /
    // 16 / 32 sequences: 21.6 / 30.2 / 37.7 us narrow and 25.6 / 25.6 / 27.2 us wide;
    // 30000 tokens, one KV head for 8, 12 sequences: 23.1 and 29.9 us.
    const uint64_t wide = 6144 * (prefix / r.prefix_splits) + (r.both ? 0 : 3u << 20);
    r.prefix_narrow = r.columns && rows * d->num_heads * prefix <= wide;
    if (r.prefix_narrow) {
      r.both = false;
      r.prefix_tiles = (uint32_t)((rows * group + kPrefixTile - 1) / kPrefixTile);
      r.prefix_splits = splits_for((uint64_t)r.prefix_tiles * p.heads, 2ull * p.cus, prefix, 256);
    }
  }
  // k_attend_few's workgroups run two to a CU
  r.own_splits = splits_for(groups, r.columns && !r.both ? 2ull * p.cus : p.cus, own, r.columns ? 256 : 512);
  const uint64_t splits = (uint64_t)r.own_splits + r.prefix_splits;
  r.parts = splits > 1 ? rows * d->num_heads * splits : 0;
  return r;
}

uint64_t plan_bytes(const Plan& r, uint32_t dim) {
  return r.parts ? ((r.parts * sizeof(float2) + 255) & ~255ull) + r.parts * dim * sizeof(float) : 0;
}

template <int D, bool E4M3, Within WITHIN>
void launch_few(const PoolView& p, const Plan& plan, const Args& a, uint32_t prefix, uint32_t own) {
  const dim3 both((own + 7) / 8 * 8 + (prefix + 7) / 8 * 8);
  if (plan.columns == 1)
    hipLaunchKernelGGL((k_attend_few<D, E4M3, WITHIN, 1>), both, dim3(256), 0, p.stream, a, prefix, own);
  else
    hipLaunchKernelGGL((k_attend_few<D, E4M3, WITHIN, 2>), both, dim3(256), 0, p.stream, a, prefix, own);
}

template <int D, bool E4M3, Within WITHIN>
void launch_rows(const PoolView& p, const Args& a, uint32_t items, uint32_t prefix) {
  constexpr int kWaves = kRowsTile / 32;
  hipLaunchKernelGGL((k_attend_rows<D, E4M3, kWaves, WITHIN>), dim3(items), dim3(kWaves * 64), 0, p.stream,
                     a, prefix);
}

template <int D, bool E4M3>
int launch(const PoolView& p, const Plan& plan, const Args& a) {
  const uint32_t own = plan.tiles * a.heads * a.own_splits;
  const uint32_t prefix = plan.prefix_tiles * a.heads * a.prefix_splits;
  const uint32_t narrow = plan.prefix_narrow ? prefix : 0;
  const bool loads = one_block_loads(p);
  if (plan.both) {
    const bool first = 4 * prefix <= 3 * p.cus;
    if (p.bs % Few<D, E4M3, 8>::kKeys == 0)
      hipLaunchKernelGGL((k_attend_both<D, E4M3, kTiles>), dim3(prefix + own), dim3(512), 0, p.stream, a, prefix,
                         first);
    else
      hipLaunchKernelGGL((k_attend_both<D, E4M3, kLoads>), dim3(prefix + own), dim3(512), 0, p.stream, a, prefix,
                         first);
  } else if (plan.columns) {
    if (p.bs % Few<D, E4M3, 4>::kKeys == 0)
      launch_few<D, E4M3, kTiles>(p, plan, a, narrow, own);
    else if (loads)
      launch_few<D, E4M3, kLoads>(p, plan, a, narrow, own);
    else
      launch_few<D, E4M3, kLanes>(p, plan, a, narrow, own);
  }
  const auto rows = loads ? launch_rows<D, E4M3, kLoads> : launch_rows<D, E4M3, kLanes>;
  if (!plan.columns) rows(p, a, own, 0);
  if (prefix > narrow && !plan.both) rows(p, a, prefix, 1);
  if (plan.parts)
    hipLaunchKernelGGL((k_join<D>), dim3((a.rows * a.heads * a.group + 3) / 4), dim3(256), 0, p.stream, a);
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
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
  Args a{};
  if (!fill_args(p, s, d, &a)) return CLAIM_EINVAL;
  SEQ_HIP(hipSetDevice(p.device));
  a.own_splits = plan.own_splits;
  a.prefix_splits = plan.prefix_splits;
  a.tiles = plan.tiles;
  if (plan.parts) {
    a.part_ml = (float2*)d->work;
    a.part_o = (float*)((uint8_t*)d->work + ((plan.parts * sizeof(float2) + 255) & ~255ull));
  }
  if (p.dim == 128)
    return p.elem == 1 ? launch<128, true>(p, plan, a) : launch<128, false>(p, plan, a);
  return p.elem == 1 ? launch<64, true>(p, plan, a) : launch<64, false>(p, plan, a);
}

}  // extern "C"
