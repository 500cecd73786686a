// Device helpers of the calls that fill and read the paged cache.
#pragma once

#include "epikv_internal.h"

namespace epikv {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Cached and new tokens of sequence b; a sequence whose counts are out of
// range has none of either (`bad`).
struct SeqTokens {
  int n, nn;
  bool bad;
};

__device__ __forceinline__ SeqTokens seq_tokens(const PagedArgs& a, int b) {
  SeqTokens t;
  t.n = a.n_cached[b];
  const int given = (a.n_new ? a.n_new : a.n_cached)[b];  // (no branch between two loads)
  t.nn = a.n_new ? given : a.C;
  t.bad = t.nn < 0 || t.nn > a.C || t.n < t.nn || t.n > a.max_tokens;
  if (t.bad) t.n = t.nn = 0;
  return t;
}

// Byte offset of a slot's row inside a (layer, K|V) plane, or -1 where its
// page id is out of range.  0 <= slot < max_tokens.
__device__ __forceinline__ int64_t row_offset(const PagedArgs& a, int b, int slot) {
  const int pi = a.page_shift >= 0 ? slot >> a.page_shift : (int)((uint32_t)slot / (uint32_t)a.page_size);
  const int pg = a.pt[(int64_t)b * a.ld_pt + pi];
  if (pg < 0 || pg >= a.n_pages) return -1;
  return (int64_t)pg * a.s_page + (int64_t)(slot - pi * a.page_size) * a.row_bytes;
}

__device__ __forceinline__ void raise_flag(int32_t* status, int b) {
  if (status) status[b] = EPIKV_SEQ_RANGE;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2 v;
  v[0] = (__bf16)lo;  // (one v_cvt_pk_bf16_f32, to nearest even)
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// The power of two of a 4-bit block's scale byte, as the conversion takes it:
// its exponent alone counts, and that of 255 (a block that held a NaN or an
// infinity) makes every value of the block NaN.
__device__ __forceinline__ float block_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes (two to a byte, the lower first) as bf16 times the scale, two
// to a v_cvt_scalef32_pk_bf16_fp4.
__device__ __forceinline__ u32x4 decode8(uint32_t codes, float scale) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return w;
}

}  // namespace epikv
