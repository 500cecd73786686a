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

// Where a token's cosines and sines are: the table's row of its position.
struct TableRow {
  static constexpr bool STAGED = false;
  int64_t p;
  __device__ __forceinline__ void stage(const RopeArg&) {}
  // false: the position is out of range
  __device__ __forceinline__ bool find(const RopeArg& r, int b, int c) {
    p = position_of(r, b, c);
    return p >= 0 && p < r.n_pos;
  }
  // M pairs from pair i on (a multiple of M, M of 2).
  template <int M>
  __device__ __forceinline__ void load(const RopeArg& r, int i, f32x4* cs) const {
    const f32x4* t = reinterpret_cast<const f32x4*>(r.table + p * (r.r / 2) + i);
#pragma unroll
    for (int k = 0; k < M / 2; ++k) cs[k] = t[k];
  }
};

// Positions on several axes: every pair is in the row of its axis' position.
// WAVE: the wavefront has one token; its pairs come into LDS, one a lane, and
// from there to the lanes as from a row of the table.  (Pair by pair from the
// table, eight loads a lane, 16384 tokens of 32 heads of 128 take 57 us, so 42.6.)
template <bool WAVE>
struct TableRows {
  static constexpr bool STAGED = WAVE;
  uint32_t p[EPIKV_MAX_AXES];
  float2* lds;  // the wavefront's, of r / 2 pairs
  __device__ __forceinline__ bool find(const RopeAxesArg& r, int b, int c) {
    bool in = true;
#pragma unroll
    for (int a = 0; a < EPIKV_MAX_AXES; ++a) {
      // (no branch between the loads; an axis past the last stands for it)
      const int64_t row = (int64_t)b * r.n_axes + min(a, r.n_axes - 1);
      const int64_t at = r.ld_pos ? (int64_t)r.positions[row * r.ld_pos + c] : (int64_t)r.positions[row] + c;
      in &= at >= 0 && at < r.n_pos;
      p[a] = (uint32_t)at;
    }
    return in;
  }
  // The axes of the eight pairs from i on, two bits each.
  __device__ __forceinline__ uint32_t axes_at(const RopeAxesArg& r, int i) const {
    uint32_t word = 0;
#pragma unroll
    for (int k = 0; k < EPIKV_MAX_AXES; ++k) {  // (those past the last begin past every pair)
      const uint32_t at = (uint32_t)i - r.turns[k] * (((uint32_t)i * r.inverse[k]) >> 16);
      const uint32_t below = (1u << (2 * min(max(r.start[k] - i, 0), 8))) - 1u;  // pairs of the runs before
      word = (word & below) | (r.axes[k] >> (2 * at) & ~below);
    }
    return word;
  }
  __device__ __forceinline__ float2 entry(const RopeAxesArg& r, uint32_t axis, int i) const {
    // (all four read first: as a choice of what to read the compiler puts them in LDS)
    const uint32_t p0 = p[0], p1 = p[1], p2 = p[2], p3 = p[3];
    const uint32_t lo = axis & 1u ? p1 : p0, hi = axis & 1u ? p3 : p2;
    return r.table[(uint64_t)(axis & 2u ? hi : lo) * ((uint32_t)r.r / 2) + (uint32_t)i];
  }
  // All lanes of the wavefront that have an item (its first ones), before load.
  __device__ __forceinline__ void stage(const RopeAxesArg& r) {
    if constexpr (WAVE) {
      const int lanes = __popcll(__ballot(true));
      for (int i = threadIdx.x & 63; i < r.r / 2; i += lanes) lds[i] = entry(r, axes_at(r, i), i);
      wave_sync();
    }
  }
  template <int M>
  __device__ __forceinline__ void load(const RopeAxesArg& r, int i, f32x4* cs) const {
    if constexpr (WAVE) {
#pragma unroll
      for (int k = 0; k < M / 2; ++k) cs[k] = *reinterpret_cast<const f32x4*>(lds + i + 2 * k);
    } else {
      const uint32_t axes = axes_at(r, i);
#pragma unroll
      for (int k = 0; k < M; ++k) {
        const float2 t = entry(r, axes >> (2 * k), i + k);
        cs[k / 2][2 * (k % 2)] = t.x;
        cs[k / 2][2 * (k % 2) + 1] = t.y;
      }
    }
  }
};

// LDS of a workgroup of four wavefronts with a token each.
inline unsigned turns_lds(const RopeArg&) { return 0; }
inline unsigned turns_lds(const RopeAxesArg& r) { return 4 * (r.r / 2) * sizeof(float2); }

template <bool WAVE>
__device__ __forceinline__ TableRow turns_of(const RopeArg&) {
  return TableRow{};
}
template <bool WAVE>
__device__ __forceinline__ TableRows<WAVE> turns_of(const RopeAxesArg& r) {
  extern __shared__ __align__(16) float2 s_turns[];
  TableRows<WAVE> t;
  t.lds = WAVE ? s_turns + (threadIdx.x >> 6) * (r.r / 2) : nullptr;
  return t;
}

// The id of a new token: its position, or where it has several, an input.
__device__ __forceinline__ int32_t id_of(const RopeArg&, const TableRow& t, int, int) { return (int32_t)t.p; }
template <bool WAVE>
__device__ __forceinline__ int32_t id_of(const RopeAxesArg& r, const TableRows<WAVE>&, int b, int c) {
  return r.ld_ids ? r.ids[(int64_t)b * r.ld_ids + c] : r.ids[b] + c;
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
template <bool FP32, bool WAVE, int U, class Rope>
__device__ __forceinline__ void rope_items(const RowsArg& x, const RowsArg& y, const Rope& r,
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
  auto turns = turns_of<WAVE>(r);
  if (r.table) {
    if (!turns.find(r, b, c)) {
      raise_flag(status, b);
      return;
    }
    turns.stage(r);
  }
  f32x4 cs[N / 2];
  if (rot) {
    // (N pairs together, or half of them for each vector)
    turns.template load<N / 2>(r, r.interleaved ? lo / 2 : lo, cs);
    turns.template load<N / 2>(r, r.interleaved ? hi / 2 : lo + N / 2, cs + N / 4);
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

// Threads over (token, item): `per` items a token.  With WAVE a wavefront has one
// token (its last wavefront perhaps fewer items than lanes), and what belongs to
// the token stays in scalar registers.
struct Place {
  int token, item;
  bool in;
};

template <bool WAVE>
__device__ __forceinline__ Place place_of(int64_t block, int per, int64_t tokens) {
  Place p;
  if constexpr (WAVE) {
    const uint32_t waves = ((uint32_t)per + 63u) / 64u;
    const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(block * 4 + (threadIdx.x >> 6)));
    p.token = (int)(w / waves);
    p.item = (int)(w - (uint32_t)p.token * waves) * 64 + (int)(threadIdx.x & 63);
  } else {
    const uint32_t t = (uint32_t)(block * 256 + threadIdx.x);
    p.token = (int)(t / (uint32_t)per);
    p.item = (int)(t - (uint32_t)p.token * (uint32_t)per);
  }
  p.in = p.token < tokens && (!WAVE || p.item < per);
  return p;
}

// Whether a token's items go to wavefronts of their own: where they fill them,
// and with positions on several axes (whose turns come through LDS then) where
// more than two thirds of the lanes have one.  16384 tokens of 24 heads of 64, 96
// items: 22 us so, 28 without; of 14, 56 items: 13.7, 16.5; of 9 of 128, 72 items:
// 30.5, 19.3; of 9 of 64, 36 items: 11.7, 12.7; of 9 of 128 in float32, 144 items:
// 32.1, 29.7.
inline bool by_wave(const RopeArg&, int per) { return per % 64 == 0; }
inline bool by_wave(const RopeAxesArg&, int per) { return 3 * per > 2 * ((per + 63) / 64 * 64); }
inline int64_t threads_of(int64_t tokens, int per, bool wave) { return tokens * (wave ? (per + 63) / 64 * 64 : per); }

// Threads beyond 2^32 do not fit place_of's numbers.
inline bool threads_fit(int64_t tokens, int per) { return tokens * per < ((int64_t)1 << 32) - 256; }

}  // namespace epikv
