// The rotation of 16 channels of one head by its token's position.
#pragma once

#include "cache_impl.h"

namespace epikv {

// A pair by its cosine and sine.  The two products and the sum are rounded
// one by one (never fused), so that the same float32 arithmetic elsewhere
// gives the same bits: what a 4-bit cache quantises must not hang on how a
// compiler contracts.
__device__ __forceinline__ void rotate_pair(float& x, float& y, f32x2 cs, bool transpose) {
#pragma clang fp contract(off)
  const float c = cs.x, s = transpose ? -cs.y : cs.y;
  const float u = x * c - y * s;
  const float v = y * c + x * s;
  x = u;
  y = v;
}

__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(w[i]);
    x[2 * i + 1] = bf16_hi(w[i]);
  }
}

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  return w;
}

template <bool FP32>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
  if constexpr (FP32) {
    const f32x4 u = *reinterpret_cast<const f32x4*>(p);
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = u[i];
      x[4 + i] = v[i];
    }
  } else {
    unpack8(*reinterpret_cast<const u32x4*>(p), x);
  }
}

template <bool FP32>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (FP32) {
    f32x4 u, v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = x[i];
      v[i] = x[4 + i];
    }
    *reinterpret_cast<f32x4*>(p) = u;
    *reinterpret_cast<f32x4*>(p + 16) = v;
  } else {
    *reinterpret_cast<u32x4*>(p) = pack8(x);
  }
}

__device__ __forceinline__ int64_t position_of(const RopeArg& r, int b, int c) {
  return r.ld_pos ? (int64_t)r.positions[(int64_t)b * r.ld_pos + c]
                  : (int64_t)r.positions[b] + c;
}

// Item `it` of head h of token (b, c): the 8-vectors at channels (lo, hi) are
// 8 apart for interleaved pairs and plain channels, rotary_dim / 2 for halves.
template <bool FP32>
__device__ __forceinline__ void rope_item(const RowsArg& x, const RowsArg& y, const RopeArg& r,
                                          int32_t* status, int b, int c, int h, int it) {
  constexpr int ES = FP32 ? 4 : 2;
  const int n_rot = r.table ? r.r / 16 : 0;
  const bool rot = it < n_rot, half = rot && !r.interleaved;
  const int lo = half ? it * 8 : it * 16;
  const int hi = half ? lo + r.r / 2 : lo + 8;
  const char* xp = x.base + (b * x.ld_seq + c * x.ld_tok + h * x.ld_head) * ES;
  char* yp = y.base + (b * y.ld_seq + c * y.ld_tok + h * y.ld_head) * ES;
  int64_t p = 0;
  if (r.table) {
    p = position_of(r, b, c);
    if (p < 0 || p >= r.n_pos) {
      raise_flag(status, b);
      return;
    }
  }
  float u[8], v[8];
  load8<FP32>(xp + lo * ES, u);
  load8<FP32>(xp + hi * ES, v);
  if (rot) {
    const f32x4* t = reinterpret_cast<const f32x4*>(r.table + p * (r.r / 2) + it * 8);
    const f32x4 cs[4] = {t[0], t[1], t[2], t[3]};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f32x2 w = {cs[i / 2][2 * (i % 2)], cs[i / 2][2 * (i % 2) + 1]};
      if (r.interleaved) {
        float* z = i < 4 ? u : v;
        rotate_pair(z[2 * (i % 4)], z[2 * (i % 4) + 1], w, r.transpose);
      } else {
        rotate_pair(u[i], v[i], w, r.transpose);
      }
    }
  }
  store8<FP32>(yp + lo * ES, u);
  store8<FP32>(yp + hi * ES, v);
}

}  // namespace epikv
