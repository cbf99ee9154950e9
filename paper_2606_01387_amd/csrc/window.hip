// window.hip -- attention over a pool's blocks in a sliding window behind a few
// first tokens (gfx950).
//
// The row at position P sees positions P - window + 1 .. P and 0 .. sinks - 1.  A
// tile of rows walks over the groups of keys that some of its rows see, wherever
// they lie: those that all rows see whole first, at the pace of attention without
// a window, then the ones where windows begin and end and the first of the
// sequence, with a mask.  Work and bytes go by the window, not by the length.  The
// walk, the products and the running softmax are in attend_rows.h.

#include "attend_rows.h"

namespace {

// Bound by the matrix cores and the vector unit beside them: 16384 rows of 32 query
// heads over 8 of 128 in a window of 4096 behind 4 first tokens take 966 to 1028 us on
// several cards, 0.94 to 1.0 PFLOP/s of the pairs that are seen, the matrix cores 46 %
// busy.  Tiles with a mask cost a
// short window the most: 12 ragged e4m3 prompts in a window of 1000 behind 20 took 257 us
// when every wave looked through all of a masked tile's V for infinities and waited
// for copies just begun, 183 us with its own part and the copies of a tile before.
template <int D, bool E4M3, Within WITHIN>
__global__ void __launch_bounds__(512, 2) k_window_rows(WindowArgs a) {
  __shared__ typename Many<D, 8>::WithBad shared;
  many_rows<D, E4M3, 8, WITHIN, true>(a, false, blockIdx.x, shared);
}

// Bound by memory: 64 single tokens of 32 query heads over 8 of 128 in a window of 4096
// read 1.0 GB of keys and values in 183 us, 5.5 TB/s; twice as many workgroups, with
// their parts joined, take as long.  The same in e4m3 takes 112 us, 4.5 TB/s.
template <int D, bool E4M3, Within WITHIN, int QT>
__global__ void __launch_bounds__(256, 2) k_window_few(WindowArgs a) {
  __shared__ typename Few<D, E4M3, 4>::WithSums shared;
  few_rows<D, E4M3, 4, WITHIN, QT, true>(a, false, blockIdx.x, shared);
}

// --------------------------------------------------------------------- host

struct WindowPlan {
  uint32_t columns;  // by few_rows with 16 x columns rows a tile; 0: by many_rows
  uint32_t splits, tiles;
  uint64_t parts;  // parts of all rows and heads; 0: none are kept
};

// One kernel for a call, by the mean of its sequences' query rows, as the host knows no
// more of them: few_rows up to 64.  Where sequences differ much, some of them get the
// wrong one.  32 heads over 8 of 128 in a window of 4096 behind 4000 tokens: 63 single
// tokens take 221 us, a chunk of 512 rows 67 and of 4096 rows 288 to 300; the tokens with
// the chunk of 512, by few_rows, 319 us, with the one of 4096, by many_rows, 528 to 553.
WindowPlan make_window_plan(const PoolView& p, const claim_seqs* s, const claim_window_desc* w) {
  const claim_attend_desc* d = &w->attend;
  WindowPlan r{};
  const uint64_t group = d->num_heads / p.heads, rows = d->kv.num_rows, seqs = d->kv.num_seqs;
  const uint64_t table = (uint64_t)s->max_blocks * p.bs;
  const uint64_t each = (rows * group + seqs - 1) / seqs;  // query rows of a sequence
  r.columns = each <= 16 ? 1 : each <= 64 ? 2 : 0;
  const uint32_t M = r.columns ? 16 * r.columns : kRowsTile;
  r.tiles = (uint32_t)(d->kv.offsets ? rows * group / M + seqs : seqs * ((group + M - 1) / M));
  // what a tile reads at most: its rows' windows and the first keys
  const uint64_t seen = (uint64_t)w->window + w->sinks + M / group + 1;
  r.splits = splits_for((uint64_t)r.tiles * p.heads, r.columns ? 2ull * p.cus : p.cus, seen < table ? seen : table,
                        r.columns ? 256 : 512);
  r.parts = r.splits > 1 ? rows * d->num_heads * r.splits : 0;
  return r;
}

// Parts: maxima and sums, sums before rounding, then outputs.
uint64_t sums_at(const WindowPlan& r) { return (r.parts * sizeof(float2) + 255) & ~255ull; }
uint64_t outputs_at(const WindowPlan& r) { return (sums_at(r) + r.parts * sizeof(float) + 255) & ~255ull; }

uint64_t plan_bytes(const WindowPlan& r, uint32_t dim) {
  return r.parts ? outputs_at(r) + r.parts * dim * sizeof(float) : 0;
}

int check_window(const PoolView& p, const claim_seqs* s, const claim_window_desc* w) {
  if (w->window == 0 || w->attend.prefix_blocks || w->attend.prefix || ((uintptr_t)w->lse & 3)) return CLAIM_EINVAL;
  return check_attend(p, s, &w->attend);
}

template <int D, bool E4M3, Within WITHIN>
void launch_few(const PoolView& p, const WindowPlan& plan, const WindowArgs& a, uint32_t items) {
  if (plan.columns == 1)
    hipLaunchKernelGGL((k_window_few<D, E4M3, WITHIN, 1>), dim3(items), dim3(256), 0, p.stream, a);
  else
    hipLaunchKernelGGL((k_window_few<D, E4M3, WITHIN, 2>), dim3(items), dim3(256), 0, p.stream, a);
}

template <int D, bool E4M3>
int launch(const PoolView& p, const WindowPlan& plan, const WindowArgs& a) {
  const uint32_t items = plan.tiles * a.heads * a.own_splits;
  const bool loads = one_block_loads(p);
  if (plan.columns) {
    if (p.bs % Few<D, E4M3, 4>::kKeys == 0)
      launch_few<D, E4M3, kTiles>(p, plan, a, items);
    else if (loads)
      launch_few<D, E4M3, kLoads>(p, plan, a, items);
    else
      launch_few<D, E4M3, kLanes>(p, plan, a, items);
  } else if (loads) {
    hipLaunchKernelGGL((k_window_rows<D, E4M3, kLoads>), dim3(items), dim3(512), 0, p.stream, a);
  } else {
    hipLaunchKernelGGL((k_window_rows<D, E4M3, kLanes>), dim3(items), dim3(512), 0, p.stream, a);
  }
  if (plan.parts)
    hipLaunchKernelGGL((k_join<D, true>), dim3((a.rows * a.heads * a.group + 3) / 4), dim3(256), 0, p.stream, a);
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
}

}  // namespace

extern "C" {

int claim_attend_window_work(const claim_pool* P, const claim_seqs* s, const claim_window_desc* w,
                             uint64_t* bytes) {
  if (!P || !w || !bytes) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_window(p, s, w);
  if (rc != CLAIM_OK) return rc;
  *bytes = w->attend.kv.num_rows ? plan_bytes(make_window_plan(p, s, w), p.dim) : 0;
  return CLAIM_OK;
}

int claim_attend_window(claim_pool* P, const claim_seqs* s, const claim_window_desc* w) {
  if (!P || !w) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_window(p, s, w);
  if (rc != CLAIM_OK) return rc;
  const claim_attend_desc* d = &w->attend;
  if (d->kv.num_rows == 0) return CLAIM_OK;
  if (!rows_ok(d->q) || !rows_ok(d->out)) return CLAIM_EINVAL;
  const WindowPlan plan = make_window_plan(p, s, w);
  const uint64_t need = plan_bytes(plan, p.dim);
  if (need && ((uintptr_t)d->work & 255)) return CLAIM_EINVAL;
  if (need && (!d->work || d->work_bytes < need)) return CLAIM_ENOSPC;
  WindowArgs a{};
  if (!fill_args(p, s, d, &a)) return CLAIM_EINVAL;
  a.own_splits = plan.splits;
  a.tiles = plan.tiles;
  a.window = w->window;
  a.sinks = w->sinks;
  const uint64_t room = (uint64_t)s->max_blocks * p.bs;
  a.room = room < 0xFFFFF000u ? (uint32_t)room : 0xFFFFF000u;
  a.lse = w->lse;
  if (plan.parts) {
    a.part_ml = (float2*)d->work;
    a.part_sum = (float*)((uint8_t*)d->work + sums_at(plan));
    a.part_o = (float*)((uint8_t*)d->work + outputs_at(plan));
  }
  SEQ_HIP(hipSetDevice(p.device));
  if (p.dim == 128) return p.elem == 1 ? launch<128, true>(p, plan, a) : launch<128, false>(p, plan, a);
  return p.elem == 1 ? launch<64, true>(p, plan, a) : launch<64, false>(p, plan, a);
}

}  // extern "C"
