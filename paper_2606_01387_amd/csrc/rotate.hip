// rotate.hip -- new tokens' queries and keys, normed by head and turned by their
// positions, the keys and values on their way into a pool's blocks (gfx950).
//
// For each head x of a row: y = x w / sqrt(mean x^2 + eps), then each pair (a, b)
// of the leading dimensions becomes (a cos t - b sin t, b cos t + a sin t), with
// the angle t = position x frequency of the pair.  All of it is in 32 bits, the
// angle in 64, and results are rounded once, to bf16 or e4m3.

#include "write_row.h"

namespace {

struct Rotate {
  uint32_t num_seqs, rows, waves;      // waves of a row
  uint32_t q_heads, kv_heads;
  const uint32_t *ids, *offsets;
  const uint16_t *q, *k, *v;
  uint16_t* out;
  uint64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head;  // in elements
  const uint16_t *q_norm, *k_norm;
  float eps;
  uint32_t half;  // pairs of a head
  const double* freqs;
  const int32_t* positions;
  uint64_t pos_row, pos_axis;
  uint32_t edge[3];  // the first pair of axis 1, 2, 3
  float k_scale, v_scale, k_inverse, v_inverse;
  uint32_t bs, nb, token_bytes;
  uint64_t chunk_bytes;
  uint8_t *k_plane, *v_plane;
};

// Where rows go.
struct Places {
  uint32_t max_seqs, max_blocks;
  const uint32_t *tables, *lengths;
};

struct Eight {
  float x[8];
};

__device__ __forceinline__ Eight widen(u32x4 w) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e.x[2 * i] = bf16_lo(w[i]);
    e.x[2 * i + 1] = bf16_hi(w[i]);
  }
  return e;
}

__device__ __forceinline__ u32x4 narrow(const Eight& e) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (__bf16)e.x[i];
  return __builtin_bit_cast(u32x4, b);
}

// A head's weights at this lane's elements, as they are in memory: widened where they
// are used, they take fewer registers.
__device__ __forceinline__ u32x4 weights(const uint16_t* norm, uint32_t at) {
  constexpr uint32_t kOnes = 0x3F803F80u;
  return norm ? *(const u32x4*)(norm + at) : u32x4{kOnes, kOnes, kOnes, kOnes};
}

// The value of the lane that a rule within rows of 16 lanes names; lanes of the banks
// (of 4) that `BANKS` leaves out keep `old`.
template <int RULE, int BANKS = 15>
__device__ __forceinline__ float lane_rule(float x, float old = 0.0f) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(x), RULE, 15, BANKS, false));
}

// A value's sum over the LANES (8 or 16) of a head, on all of them.
template <uint32_t LANES>
__device__ __forceinline__ float sum_head(float x) {
  x += lane_rule<0xB1>(x);   // lane ^ 1
  x += lane_rule<0x4E>(x);   // lane ^ 2
  x += lane_rule<0x141>(x);  // 7 - lane of eight
  return LANES == 16 ? x + lane_rule<0x140>(x) : x;  // 15 - lane of sixteen
}

// The mean square of a head, of which a lane has eight elements.
template <int D>
__device__ __forceinline__ float mean_square(const Eight& y) {
  float square = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) square = __builtin_fmaf(y.x[i], y.x[i], square);
  return sum_head<D / 8>(square) * (1.0f / D);
}

// A mean square with eps below 2^-90 may be the sum of squares that have lost bits at
// the lower end of 32, or all of them: such a head is taken 2^100 times as large, which
// rounds nothing and cancels in x / sqrt(mean(x^2) + eps).  With an eps of 2^-90 or more
// no mean is that small, and the kernel does not look (SMALL): 79.2 us in place of 81.1
// for the e4m3 prompts below.
constexpr float kSmall = 0x1p-90f, kUp = 0x1p100f;

// The value of the head's lane half of its lanes on.
template <uint32_t LANES>
__device__ __forceinline__ float across_head(float x) {
  if (LANES == 16) return lane_rule<0x128>(x);             // eight lanes round
  return lane_rule<0x104, 5>(x, lane_rule<0x114, 10>(x));  // four lanes up, four down
}

// A wave takes a row, or a part of its heads where rows are few; D / 8 lanes hold
// a head, 8 neighbouring elements each.  A pair's other element is in the same
// lane (NEIGHBOURS), or rot / 2 elements on, in another lane of the head: where all
// of the head turns half of its lanes on, which takes no way through LDS.  The
// loads of the first heads are on their way while the row's place, position
// and angles (one pair a lane, then LDS) are looked up.
//
// Bound by memory, and by those dependent reads where rows are few: 18348 rows of 28
// query heads over 4 of 128, three axes, to e4m3 in 80 us, 4.0 TB/s read and written
// (82 % of a copy's rate; 85 us with loads that the caches keep); four loads of a lane
// at a time (2 took 92 us where 4 took 85, 9 95).  16384 rows of 32 heads over 8 of 64
// in 43 us, 4.7 TB/s; 48 single rows of 32 heads over 8 of 128 in 6.3 us.
template <int D, bool E4M3, bool NEIGHBOURS, bool SMALL>
__global__ void __launch_bounds__(256) k_write_rotated(Rotate a, Places s) {
  constexpr uint32_t kLanes = D / 8, kHeads = 64 / kLanes, kMany = 4;
  __shared__ float2 angles[4][D / 2];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t x = blockIdx.x * 4 + wave, row = x / a.waves, part = x - row * a.waves;
  if (row >= a.rows) return;
  const uint32_t heads = a.q_heads + 2 * a.kv_heads;
  const uint32_t at = lane % kLanes * 8;
  bool there = false, held = false;
  uint64_t token = 0;
  float c[8], n[8];  // cosines and sines of this lane's elements, signed
  const bool turned = at < 2 * a.half;
  const bool whole = !NEIGHBOURS && 2 * a.half == D;
  const uint32_t other_lane = NEIGHBOURS || !turned ? lane : at < a.half ? lane + a.half / 8 : lane - a.half / 8;
  u32x4 qw, kw;
  for (uint32_t h0 = part * kHeads; h0 < heads; h0 += a.waves * kHeads * kMany) {
    u32x4 w[kMany];
#pragma unroll
    for (uint32_t j = 0; j < kMany; ++j) {
      const uint32_t h = h0 + j * a.waves * kHeads + lane / kLanes;
      if (h >= heads) continue;
      const uint16_t* from = h < a.q_heads ? a.q + row * a.q_row + h * a.q_head
                             : h < a.q_heads + a.kv_heads
                                 ? a.k + row * a.k_row + (h - a.q_heads) * a.k_head
                                 : a.v + row * a.v_row + (h - a.q_heads - a.kv_heads) * a.v_head;
      w[j] = __builtin_nontemporal_load((const u32x4*)(from + at));  // read once
    }
    if (h0 == part * kHeads) {
      qw = weights(a.q_norm, at);
      kw = weights(a.k_norm, at);
      uint32_t r = 0;
      int64_t pos = 0;
      there = row_position(a, s, row, &r, &pos);
      if (!there) return;
      held = find_token(a, s, r, pos, &token);
      if (lane < a.half) {
        int64_t p = pos;
        if (a.positions) {
          const uint32_t axis = (lane >= a.edge[0]) + (lane >= a.edge[1]) + (lane >= a.edge[2]);
          p = a.positions[row * a.pos_row + axis * a.pos_axis];
        }
        // in turns: a position's whole turns are taken off in 64 bits, where a product
        // near 2^31 still has 2^-24 of a turn
        const double t = (double)p * (a.freqs[lane] * 0.15915494309189533577);
        float2 sc;
        sincospif(2.0f * (float)(t - rint(t)), &sc.y, &sc.x);
        angles[wave][lane] = sc;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // LDS of the wave's own
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = 1.0f;
        n[i] = 0.0f;
        if (!turned) continue;
        const uint32_t pair = NEIGHBOURS ? (at + i) / 2 : (at < a.half ? at + i : at + i - a.half);
        const float2 sc = angles[wave][pair];
        c[i] = sc.x;
        n[i] = (NEIGHBOURS ? i % 2 == 0 : at < a.half) ? -sc.y : sc.y;
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < kMany; ++j) {
      const uint32_t h = h0 + j * a.waves * kHeads + lane / kLanes;
      const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
      const u32x4 mine = w[j];
      const Eight y = widen(mine);
      Eight o = y;
      if (__any(!is_v)) {
        const bool normed = !is_v && (is_q ? a.q_norm : a.k_norm);
        Eight z = y;
        float mean = mean_square<D>(y) + a.eps;
        const bool small = normed && mean < kSmall;
        if (SMALL && __any(small)) {
          const float up = small ? kUp : 1.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) z.x[i] *= up;
          mean = mean_square<D>(z) + a.eps * up * up;
        }
        const float f = normed ? rsqrtf(mean) : 1.0f;
        const Eight own = widen(is_q ? qw : kw);
        Eight p, r;
#pragma unroll
        for (int i = 0; i < 8; ++i) p.x[i] = z.x[i] * f * own.x[i];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          r.x[i] = NEIGHBOURS ? p.x[i ^ 1] : whole ? across_head<kLanes>(p.x[i]) : __shfl(p.x[i], other_lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float z = turned ? __builtin_fmaf(p.x[i], c[i], r.x[i] * n[i]) : p.x[i];
          o.x[i] = is_v ? y.x[i] : z;
        }
      }
      if (h >= heads) continue;
      if (is_q) {
        *(u32x4*)(a.out + row * a.out_row + h * a.out_head + at) = narrow(o);
      } else if (held) {
        const uint32_t head = h - a.q_heads - (is_v ? a.kv_heads : 0);
        uint8_t* to = (is_v ? a.v_plane : a.k_plane) + token;
        if (E4M3) {
          const float scale = is_v ? a.v_scale : a.k_scale, inverse = is_v ? a.v_inverse : a.k_inverse;
          *(u32x2*)(to + head * D + at) =
              u32x2{to_e4m3(o.x[0], o.x[1], o.x[2], o.x[3], scale, inverse),
                    to_e4m3(o.x[4], o.x[5], o.x[6], o.x[7], scale, inverse)};
        } else {
          *(u32x4*)(to + (head * D + at) * 2) = is_v ? mine : narrow(o);
        }
      }
    }
  }
}

template <int D, bool E4M3, bool NEIGHBOURS>
void launch(const PoolView& p, const Rotate& a, const Places& s) {
  const dim3 grid((uint32_t)(((uint64_t)a.rows * a.waves + 3) / 4));
  if (a.eps < kSmall && (a.q_norm || a.k_norm))
    hipLaunchKernelGGL((k_write_rotated<D, E4M3, NEIGHBOURS, true>), grid, dim3(256), 0, p.stream, a, s);
  else
    hipLaunchKernelGGL((k_write_rotated<D, E4M3, NEIGHBOURS, false>), grid, dim3(256), 0, p.stream, a, s);
}

template <int D, bool E4M3>
void launch(const PoolView& p, const Rotate& a, const Places& s, bool neighbours) {
  if (neighbours)
    launch<D, E4M3, true>(p, a, s);
  else
    launch<D, E4M3, false>(p, a, s);
}

int check_rotate(const PoolView& p, const claim_seqs* s, const claim_rotate_desc* d) {
  const int rc = check_kv(p, s, &d->kv);
  if (rc != CLAIM_OK) return rc;
  if (p.dim != 64 && p.dim != 128) return CLAIM_EINVAL;
  if (d->num_heads == 0 || (uint64_t)d->kv.num_rows * d->num_heads >= 1u << 26 || d->num_heads >= 1u << 16)
    return CLAIM_EINVAL;
  if (d->rot_dims % 16 || d->rot_dims > p.dim || (d->rot_dims && !d->freqs)) return CLAIM_EINVAL;
  if ((d->flags & ~CLAIM_ROTATE_NEIGHBOURS) || !(d->eps >= 0.0f && d->eps <= 3.4e38f)) return CLAIM_EINVAL;
  uint64_t pairs = 0;
  for (uint32_t n : d->sections) pairs += n;
  if (pairs != d->rot_dims / 2) return CLAIM_EINVAL;
  if (((uintptr_t)d->q_norm & 15) || ((uintptr_t)d->k_norm & 15) || ((uintptr_t)d->freqs & 7) ||
      ((uintptr_t)d->positions & 3))
    return CLAIM_EINVAL;
  return CLAIM_OK;
}

}  // namespace

extern "C" int claim_kv_write_rotated(claim_pool* P, const claim_seqs* s, const claim_rotate_desc* d) {
  if (!P || !d) return CLAIM_EINVAL;
  int rc = check_seqs(s);
  const PoolView p = pool_view(P);
  if (rc == CLAIM_OK) rc = check_rotate(p, s, d);
  if (rc != CLAIM_OK) return rc;
  if (d->kv.num_rows == 0) return CLAIM_OK;
  if (!rows_ok(d->q) || !rows_ok(d->k) || !rows_ok(d->v) || !rows_ok(d->out)) return CLAIM_EINVAL;
  SEQ_HIP(hipSetDevice(p.device));
  Rotate a{};
  a.num_seqs = d->kv.num_seqs;
  a.rows = d->kv.num_rows;
  a.q_heads = d->num_heads;
  a.kv_heads = p.heads;
  a.ids = d->kv.ids;
  a.offsets = d->kv.offsets;
  a.q = (const uint16_t*)d->q.data;
  a.k = (const uint16_t*)d->k.data;
  a.v = (const uint16_t*)d->v.data;
  a.out = (uint16_t*)d->out.data;
  a.q_row = d->q.row_stride;
  a.q_head = d->q.head_stride;
  a.k_row = d->k.row_stride;
  a.k_head = d->k.head_stride;
  a.v_row = d->v.row_stride;
  a.v_head = d->v.head_stride;
  a.out_row = d->out.row_stride;
  a.out_head = d->out.head_stride;
  a.q_norm = (const uint16_t*)d->q_norm;
  a.k_norm = (const uint16_t*)d->k_norm;
  a.eps = d->eps;
  a.half = d->rot_dims / 2;
  a.freqs = d->freqs;
  a.positions = d->positions;
  a.pos_row = d->position_stride;
  a.pos_axis = d->axis_stride;
  a.edge[0] = d->sections[0];
  a.edge[1] = a.edge[0] + d->sections[1];
  a.edge[2] = a.edge[1] + d->sections[2];
  a.k_scale = d->kv.k_scale;
  a.v_scale = d->kv.v_scale;
  a.k_inverse = 1.0f / d->kv.k_scale;
  a.v_inverse = 1.0f / d->kv.v_scale;
  a.bs = p.bs;
  a.nb = p.nb;
  a.chunk_bytes = p.chunk_bytes;
  a.token_bytes = (uint32_t)(p.chunk_bytes / p.bs);
  const uint64_t plane = (uint64_t)p.nb * p.chunk_bytes;
  a.k_plane = p.kv + 2ull * d->kv.layer * plane;
  a.v_plane = a.k_plane + plane;
  // a wave of a row's own for every four loads of a lane, while that leaves CUs idle
  const uint32_t loads = (d->num_heads + 2 * p.heads + 512 / p.dim - 1) / (512 / p.dim);
  a.waves = 1;
  while (a.waves < 16 && a.waves * 4 < loads && 2ull * a.waves * a.rows <= 16ull * p.cus) a.waves *= 2;
  const Places places{s->max_seqs, s->max_blocks, s->tables, s->lengths};
  const bool neighbours = d->flags & CLAIM_ROTATE_NEIGHBOURS;
  if (p.dim == 128) {
    if (p.elem == 1) launch<128, true>(p, a, places, neighbours);
    else launch<128, false>(p, a, places, neighbours);
  } else {
    if (p.elem == 1) launch<64, true>(p, a, places, neighbours);
    else launch<64, false>(p, a, places, neighbours);
  }
  return hipGetLastError() == hipSuccess ? CLAIM_OK : CLAIM_EHIP;
}
