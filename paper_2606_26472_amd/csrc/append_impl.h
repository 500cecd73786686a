// New keys and values into the cache's pages, keys (and queries) rotated on
// the way, as bf16 rows or quantised to 4 bits; and rows back as bf16.
#pragma once

#include "rope_impl.h"

namespace epikv {
namespace {

// The largest magnitude's exponent field decides a block's power of two:
// field - 2 puts the block's maximum in [4, 8) units, and past 7 units (a
// mantissa above 0x600000) one more, which costs a value of 6 to 8 units at
// most one unit where clipping would cost more.  Never below 2^-126.
__device__ __forceinline__ uint32_t block_byte(uint32_t top_bits) {
  const int field = (int)(top_bits >> 23);
  if (field == 255) return 255u;
  const int e = field - 2 + ((top_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 1);
}

// Eight channels of U heads h, h + step, ... of a new token's keys or values
// (kv), four lanes to a block of 32.  A key's partner channels are read again
// rather than exchanged (they are in the cache), so that every layout and
// rotary_dim is one code.
template <bool Q4, bool WAVE, int U, class Args>
__device__ __forceinline__ void append_vecs(const Args& a, int b, int c, int kv, int h, int step,
                                            int vec) {
  const PagedArgs& g = a.pg;
  const RowsArg& in = kv ? a.v : a.k;
  const char* x = in.base + (b * in.ld_seq + c * in.ld_tok + h * in.ld_head) * 2;
  const int64_t next = step * in.ld_head * 2;
  const int r = a.rope.r;
  const bool rot = kv == 0 && a.rope.table && vec * 8 < r;
  const bool half = rot && !a.rope.interleaved;
  const int nv = r / 16;  // vectors per half
  const bool upper = half && vec >= nv;
  const int first = upper ? vec - nv : vec;
  u32x4 own[U], partner[U];
#pragma unroll
  for (int i = 0; i < U; ++i) own[i] = *reinterpret_cast<const u32x4*>(x + i * next + vec * 16);
  if (half) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      partner[i] = *reinterpret_cast<const u32x4*>(x + i * next + (upper ? first : vec + nv) * 16);
  }
  const SeqTokens t = seq_tokens(g, b);
  if (c >= t.nn) {
    if (t.bad) raise_flag(g.status, b);
    return;  // (all four lanes of a block are one token's)
  }
  const int slot = t.n - t.nn + c;
  const int64_t off = row_offset(g, b, slot);
  auto turns = turns_of<WAVE>(a.rope);
  bool bad = off < 0;
  if (a.rope.table || a.pos) bad |= !turns.find(a.rope, b, c) && a.rope.table;
  if (bad) {
    raise_flag(g.status, b);
    return;
  }
  if (kv == 0 && h == 0 && vec == 0 && a.pos) {
    if (slot < a.ld_s)
      a.pos[(int64_t)b * a.ld_s + slot] = id_of(a.rope, turns, b, c);
    else
      raise_flag(g.status, b);  // (no place for its id: a step would move one that was never set)
  }
  f32x4 cs[4];
  if constexpr (decltype(turns)::STAGED)
    if (a.rope.table && __any(rot)) turns.stage(a.rope);
  if (rot) {
    const int pair = half ? first * 8 : vec * 4;
    turns.template load<4>(a.rope, pair, cs);
    if (half) turns.template load<4>(a.rope, pair + 4, cs + 2);
  }
  char* row = g.plane[kv] + off;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float u[8];
    unpack8(own[k], u);
    if (half) {
      float w[8];
      unpack8(partner[k], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float lo = upper ? w[i] : u[i], hi = upper ? u[i] : w[i];
        rotate_pair(lo, hi, pair_of(cs, i), false);
        u[i] = upper ? hi : lo;
      }
    } else if (rot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) rotate_pair(u[2 * i], u[2 * i + 1], pair_of(cs, i), false);
    }
    const int head = h + k * step;
    if constexpr (!Q4) {
      st_stream(row + (head * g.d + vec * 8) * 2, rot ? pack8(u) : own[k]);
    } else {
      // (integer order of magnitudes: NaN and infinity sort above all numbers)
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(u[i]) & 0x7fffffffu);
      top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));  // lane ^ 1
      top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));  // lane ^ 2
      const uint32_t byte = block_byte(top);
      const float s = block_scale(byte);
      // (to nearest, ties to the even code, at most 6)
      uint32_t codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, u[0], u[1], s, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[2], u[3], s, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[4], u[5], s, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, u[6], u[7], s, 3);
      *reinterpret_cast<uint32_t*>(row + head * (g.d / 2) + vec * 4) = byte == 255u ? 0u : codes;
      if ((vec & 3) == 0) row[g.H * (g.d / 2) + head * (g.d / 32) + vec / 4] = (char)byte;
    }
  }
}

// Bound by HBM where rows are bf16 (long chunks: 205 MB in 36.6 us, 5.6 TB/s).  With
// 4-bit rows the same chunk's 182 MB take 37.7 us, and by positions on three axes
// either format 42 to 43.7 (4.9 and 4.2 TB/s): not for their bytes, but for the chain
// of loads to a row and its turns, for which wavefronts wait 57 to 60 % of their time
// (vector units are busy 43 to 47 %).  Single tokens: the launch and that chain, 4.3
// us, on three axes 5.0.
//
// Queries: a thread per two vectors of UQ heads (rope_items), in the first
// nq_blocks workgroups; keys and values: a thread per 8 channels of UKV heads.
template <bool Q4, bool WAVE, int UQ, int UKV, class Args>
__global__ __launch_bounds__(256) void k_append(Args a, int64_t nq_blocks, int per_q, int per_kv) {
  const PagedArgs& g = a.pg;
  const int64_t block = linear_block();
  const int64_t tokens = (int64_t)g.B * g.C;
  if (block < nq_blocks) {
    const Place at = place_of<WAVE>(block, per_q, tokens);
    if (!at.in) return;
    const int b = at.token / g.C, c = at.token - b * g.C;
    if (c >= seq_tokens(g, b).nn) return;
    const int iph = g.d / 16, h = at.item / iph;
    rope_items<false, WAVE, UQ>(a.q, a.q_out, a.rope, g.status, b, c, h, a.heads / UQ, at.item - h * iph, g.d);
    return;
  }
  const Place at = place_of<WAVE>(block - nq_blocks, per_kv, tokens);
  if (!at.in) return;
  const int b = at.token / g.C, c = at.token - b * g.C;
  const int vph = g.d / 8, heads = g.H / UKV;
  const int hv = at.item / vph, kv = hv / heads;
  append_vecs<Q4, WAVE, UKV>(a, b, c, kv, hv - kv * heads, heads, at.item - hv * vph);
}

// Heads a thread takes, of queries as of keys and values: the way to a token's
// row (its counts, its page, its position) is as long for one as for two.  A
// prompt of 8191 tokens (32 query heads, 8 KV heads of 128) takes 45.8 us with
// one of each, 39.3 with two KV heads, 37.7 with two of each, 39.1 with four
// query heads.
int heads_at_once(int heads) { return heads % 2 == 0 ? 2 : 1; }

template <bool Q4, int UQ, int UKV, class Args>
void launch_append_heads(const Args& a, hipStream_t s) {
  const int64_t tokens = (int64_t)a.pg.B * a.pg.C;
  const int per_q = a.q.base ? a.heads / UQ * (a.pg.d / 16) : 64;
  const int per_kv = 2 * (a.pg.H / UKV) * (a.pg.d / 8);
  const bool wave = by_wave(a.rope, per_q) && by_wave(a.rope, per_kv);
  const int64_t nq = a.q.base ? (threads_of(tokens, per_q, wave) + 255) / 256 : 0;
  const dim3 grid = linear_grid(nq + (threads_of(tokens, per_kv, wave) + 255) / 256, 256);
  if (wave)
    hipLaunchKernelGGL((k_append<Q4, true, UQ, UKV, Args>), grid, dim3(256), turns_lds(a.rope), s, a, nq, per_q, per_kv);
  else
    hipLaunchKernelGGL((k_append<Q4, false, UQ, UKV, Args>), grid, dim3(256), 0, s, a, nq, per_q, per_kv);
}

template <bool Q4, int UKV, class Args>
void launch_append_kv(const Args& a, hipStream_t s) {
  if (a.q.base && heads_at_once(a.heads) == 2)
    launch_append_heads<Q4, 2, UKV>(a, s);
  else
    launch_append_heads<Q4, 1, UKV>(a, s);
}

template <bool Q4, class Args>
hipError_t launch_append_fmt(const Args& a, hipStream_t s) {
  if (heads_at_once(a.pg.H) == 2)
    launch_append_kv<Q4, 2>(a, s);
  else
    launch_append_kv<Q4, 1>(a, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace epikv
