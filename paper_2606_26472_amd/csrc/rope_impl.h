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

__device__ __forceinline__ int64_t position_of(const RopeArg& r, int b, int c) {
  return r.ld_pos ? (int64_t)r.positions[(int64_t)b * r.ld_pos + c]
                  : (int64_t)r.positions[b] + c;
}

// Pair i of cosines and sines (cs[i] holds those of pairs 2i and 2i + 1).
__device__ __forceinline__ f32x2 pair_of(const f32x4* cs, int i) {
  return f32x2{cs[i / 2][2 * (i % 2)], cs[i / 2][2 * (i % 2) + 1]};
}

// A 16-byte vector's channels: 8 of bf16, 4 of float32.
template <bool FP32>
struct Vec {
  static constexpr int N = FP32 ? 4 : 8;
  static __device__ __forceinline__ void widen(u32x4 w, float (&x)[N]) {
    if constexpr (FP32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    } else {
      unpack8(w, x);
    }
  }
  static __device__ __forceinline__ u32x4 narrow(const float (&x)[N]) {
    if constexpr (FP32) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
      return w;
    } else {
      return pack8(x);
    }
  }
};

// Item `it` (two vectors) of U heads h, h + step, ... of token (b, c), which
// share the cosines and sines.  The vectors lie half of the rotated channels
// apart (of the plain ones behind them): they are each other's pairs in the
// one layout, and in either neighbouring lanes read and write neighbouring
// vectors, whole lines at a time (32 bytes a lane, past the caches, wrote
// float32 at a third of the speed).
template <bool FP32, int U>
__device__ __forceinline__ void rope_items(const RowsArg& x, const RowsArg& y, const RopeArg& r,
                                           int32_t* status, int b, int c, int h, int step, int it,
                                           int d) {
  using V = Vec<FP32>;
  constexpr int N = V::N, ES = FP32 ? 4 : 2;
  const int turned = r.table ? r.r : 0;  // channels
  const bool rot = it * 2 * N < turned;
  const int lo = rot ? it * N : turned + (it - turned / (2 * N)) * N;
  const int hi = lo + (rot ? turned : d - turned) / 2;
  const char* xp = x.base + (b * x.ld_seq + c * x.ld_tok + h * x.ld_head) * ES;
  char* yp = y.base + (b * y.ld_seq + c * y.ld_tok + h * y.ld_head) * ES;
  u32x4 ru[U], rv[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    ru[i] = ld_stream(xp + (i * step * x.ld_head + lo) * ES);
    rv[i] = ld_stream(xp + (i * step * x.ld_head + hi) * ES);
  }
  int64_t p = 0;
  if (r.table) {
    p = position_of(r, b, c);
    if (p < 0 || p >= r.n_pos) {
      raise_flag(status, b);
      return;
    }
  }
  f32x4 cs[N / 2];
  if (rot) {
    // (N pairs together, or half of them for each vector)
    const float2* row = r.table + p * (r.r / 2);
    const f32x4* t = reinterpret_cast<const f32x4*>(row + (r.interleaved ? lo / 2 : lo));
    const f32x4* t2 = r.interleaved ? reinterpret_cast<const f32x4*>(row + hi / 2) : t + N / 4;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      cs[i] = t[i];
      cs[N / 4 + i] = t2[i];
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float u[N], v[N];
    V::widen(ru[k], u);
    V::widen(rv[k], v);
    if (rot) {
      if (r.interleaved) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          rotate_pair(u[2 * i], u[2 * i + 1], pair_of(cs, i), r.transpose);
          rotate_pair(v[2 * i], v[2 * i + 1], pair_of(cs, N / 2 + i), r.transpose);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) rotate_pair(u[i], v[i], pair_of(cs, i), r.transpose);
      }
    }
    st_stream(yp + (k * step * y.ld_head + lo) * ES, V::narrow(u));
    st_stream(yp + (k * step * y.ld_head + hi) * ES, V::narrow(v));
  }
}

// Threads over (token, item): `per` items a token.  Where they are a multiple
// of the wavefront, a wavefront has one token, and what belongs to the token
// stays in scalar registers.
struct Place {
  int token, item;
  bool in;
};

template <bool WAVE>
__device__ __forceinline__ Place place_of(int64_t block, int per, int64_t tokens) {
  Place p;
  if constexpr (WAVE) {
    const uint32_t waves = (uint32_t)per / 64u;
    const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(block * 4 + (threadIdx.x >> 6)));
    p.token = (int)(w / waves);
    p.item = (int)(w - (uint32_t)p.token * waves) * 64 + (int)(threadIdx.x & 63);
  } else {
    const uint32_t t = (uint32_t)(block * 256 + threadIdx.x);
    p.token = (int)(t / (uint32_t)per);
    p.item = (int)(t - (uint32_t)p.token * (uint32_t)per);
  }
  p.in = p.token < tokens;
  return p;
}

// Threads beyond 2^32 do not fit place_of's numbers.
inline bool threads_fit(int64_t tokens, int per) { return tokens * per < ((int64_t)1 << 32) - 256; }

}  // namespace epikv
