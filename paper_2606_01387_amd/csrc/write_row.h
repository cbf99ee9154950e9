// write_row.h -- rows of keys and values on their way into a pool's blocks
// (library-internal): where a row goes, and rounding to e4m3.
#ifndef CLAIMKV_WRITE_ROW_H
#define CLAIMKV_WRITE_ROW_H

#include "pool_view.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

// Four values to four e4m3 bytes, to nearest even.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float scale, float inverse) {
  const int p = __builtin_amdgcn_cvt_pk_fp8_f32(limit_e4m3(a, scale, inverse), limit_e4m3(b, scale, inverse),
                                                0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(limit_e4m3(c, scale, inverse), limit_e4m3(d, scale, inverse),
                                                   p, true);
}

// The same of four bf16 values (two words).
__device__ __forceinline__ uint32_t to_e4m3(uint32_t w0, uint32_t w1, float scale, float inverse) {
  return to_e4m3(bf16_lo(w0), bf16_hi(w0), bf16_lo(w1), bf16_hi(w1), scale, inverse);
}

// A packed row's row of tables (it may be out of range) and position, or false.
// `a` has the rows' offsets and ids, `s` the sequences.
template <typename A, typename S>
__device__ __forceinline__ bool row_position(const A& a, const S& s, uint32_t row, uint32_t* r, int64_t* pos) {
  uint32_t q = row, i = 0, n = 1;
  if (a.offsets) {
    q = wave_find_seq(a.offsets, a.num_seqs, row);
    const uint32_t o = a.offsets[q], e = a.offsets[q + 1];
    if (o > row || e <= row) return false;  // offsets that do not hold the row
    i = row - o;
    n = e - o;
  }
  *r = a.ids ? a.ids[q] : q;
  *pos = (int64_t)(*r < s.max_seqs ? s.lengths[*r] : 0) - n + i;
  return true;
}

// The byte of a position's token in a plane, or false.
template <typename A, typename S>
__device__ __forceinline__ bool find_token(const A& a, const S& s, uint32_t r, int64_t pos, uint64_t* token_at) {
  if (r >= s.max_seqs || pos < 0) return false;
  const uint32_t at = (uint32_t)pos / a.bs, token = (uint32_t)pos % a.bs;
  if (at >= s.max_blocks) return false;
  const uint32_t b = s.tables[(uint64_t)r * s.max_blocks + at];
  *token_at = (uint64_t)b * a.chunk_bytes + (uint64_t)token * a.token_bytes;
  return b < a.nb;
}

// Where a packed row goes: the byte of its token in a plane, or false.
template <typename A, typename S>
__device__ __forceinline__ bool find_row(const A& a, const S& s, uint32_t row, uint64_t* token_at) {
  uint32_t r;
  int64_t pos;
  return row_position(a, s, row, &r, &pos) && find_token(a, s, r, pos, token_at);
}

}  // namespace

#endif
