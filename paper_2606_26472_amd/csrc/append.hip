// New keys and values into the cache's pages, keys (and queries) rotated on
// the way, as bf16 rows or quantised to 4 bits; and rows back as bf16.
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

// e2m1 code of |x| in units, to nearest, ties to the even code, 7 (6.0) at
// most: the values' midpoints.
__device__ __forceinline__ uint32_t e2m1(float x) {
  const float v = fabsf(x);
  uint32_t c = (v > 0.25f) + (v >= 0.75f) + (v > 1.25f) + (v >= 1.75f) + (v > 2.5f) + (v >= 3.5f) +
               (v > 5.0f);
  return c | (__float_as_uint(x) >> 31 << 3);
}

// Eight channels of one head of a new token's key or value, four lanes to a
// block of 32.
template <bool Q4>
__device__ __forceinline__ void append_vec(const AppendArgs& a, int b, int c, int kv, int h, int vec) {
  const PagedArgs& g = a.pg;
  const SeqTokens t = seq_tokens(g, b);
  if (c >= t.nn) {
    if (t.bad) raise_flag(g.status, b);
    return;  // (all four lanes of a block are one token's)
  }
  const int slot = t.n - t.nn + c;
  const int64_t off = row_offset(g, b, slot);
  int64_t p = 0;
  bool bad = off < 0;
  if (a.rope.table || a.pos) p = position_of(a.rope, b, c);
  if (a.rope.table && (p < 0 || p >= a.rope.n_pos)) bad = true;
  if (bad) {
    raise_flag(g.status, b);
    return;
  }
  if (kv == 0 && h == 0 && vec == 0 && a.pos && slot < a.ld_s)
    a.pos[(int64_t)b * a.ld_s + slot] = (int32_t)p;
  const RowsArg& in = kv ? a.v : a.k;
  const char* x = in.base + (b * in.ld_seq + c * in.ld_tok + h * in.ld_head) * 2;
  float u[8];
  u32x4 raw = *reinterpret_cast<const u32x4*>(x + vec * 16);
  unpack8(raw, u);
  const int r = a.rope.r;
  const bool rot = kv == 0 && a.rope.table && vec * 8 < r;
  if (rot) {
    const float2* row = a.rope.table + p * (r / 2);
    if (a.rope.interleaved) {
      const f32x4* t4 = reinterpret_cast<const f32x4*>(row + vec * 4);
      const f32x4 cs[2] = {t4[0], t4[1]};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        rotate_pair(u[2 * i], u[2 * i + 1], f32x2{cs[i / 2][2 * (i % 2)], cs[i / 2][2 * (i % 2) + 1]},
                    false);
    } else {
      const int nv = r / 16;  // vectors per half
      const bool upper = vec >= nv;
      const int first = upper ? vec - nv : vec;
      float w[8];
      unpack8(*reinterpret_cast<const u32x4*>(x + (upper ? first : vec + nv) * 16), w);
      const f32x4* t4 = reinterpret_cast<const f32x4*>(row + first * 8);
      const f32x4 cs[4] = {t4[0], t4[1], t4[2], t4[3]};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float lo = upper ? w[i] : u[i], hi = upper ? u[i] : w[i];
        rotate_pair(lo, hi, f32x2{cs[i / 2][2 * (i % 2)], cs[i / 2][2 * (i % 2) + 1]}, false);
        u[i] = upper ? hi : lo;
      }
    }
    raw = pack8(u);
  }
  char* row = g.plane[kv] + off;
  if constexpr (!Q4) {
    *reinterpret_cast<u32x4*>(row + (h * g.d + vec * 8) * 2) = raw;
  } else {
    // (integer order of magnitudes: NaN and infinity sort above all numbers)
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(u[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t byte = block_byte(top);
    const float inv = __uint_as_float((254u - min(byte, 253u)) << 23);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes |= e2m1(u[i] * inv) << (4 * i);
    *reinterpret_cast<uint32_t*>(row + h * (g.d / 2) + vec * 4) = codes;
    if ((vec & 3) == 0) row[g.H * (g.d / 2) + h * (g.d / 32) + vec / 4] = (char)byte;
  }
}

// A thread per item: 16 channels of a query head (rope_item), or 8 of a key
// or value head.  Block roles: the first nq_blocks rotate queries.
template <bool Q4>
__global__ __launch_bounds__(256) void k_append(AppendArgs a, int64_t nq_blocks) {
  const PagedArgs& g = a.pg;
  const int64_t block = linear_block();
  if (block < nq_blocks) {
    const int64_t t = block * 256 + threadIdx.x;
    const int iph = g.d / 16, ipt = a.heads * iph;
    const int64_t token = t / ipt;
    if (token >= (int64_t)g.B * g.C) return;
    const int it = (int)(t - token * ipt);
    const int b = (int)(token / g.C), c = (int)(token - (int64_t)b * g.C);
    if (c >= seq_tokens(g, b).nn) return;
    const int h = it / iph;
    rope_item<false>(a.q, a.q_out, a.rope, g.status, b, c, h, it - h * iph);
    return;
  }
  const int64_t t = (block - nq_blocks) * 256 + threadIdx.x;
  const int vph = g.d / 8, vpt = 2 * g.H * vph;
  const int64_t token = t / vpt;
  if (token >= (int64_t)g.B * g.C) return;
  const int it = (int)(t - token * vpt);
  const int b = (int)(token / g.C), c = (int)(token - (int64_t)b * g.C);
  const int kv = it / (g.H * vph);
  const int hv = it - kv * g.H * vph;
  append_vec<Q4>(a, b, c, kv, hv / vph, hv % vph);
}

// Rows back: a thread per 8 channels.
template <bool Q4>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  const PagedArgs& g = a.pg;
  const int64_t t = linear_block() * 256 + threadIdx.x;
  const int vph = g.d / 8, vpt = 2 * g.H * vph;
  const int64_t token = t / vpt;
  if (token >= (int64_t)g.B * g.C) return;
  const int it = (int)(t - token * vpt);
  const int b = (int)(token / g.C), c = (int)(token - (int64_t)b * g.C);
  const int kv = it / (g.H * vph);
  const int hv = it - kv * g.H * vph;
  const int h = hv / vph, vec = hv % vph;
  const RowsArg& out = kv ? a.v : a.k;
  if (!out.base) return;
  const int64_t slot = (int64_t)g.n_cached[b] + c;
  const int64_t off = slot >= 0 && slot < g.max_tokens ? row_offset(g, b, (int)slot) : -1;
  u32x4 w = {0, 0, 0, 0};
  if (off < 0) {
    raise_flag(g.status, b);
  } else {
    const char* row = g.plane[kv] + off;
    if constexpr (Q4) {
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(row + h * (g.d / 2) + vec * 4);
      const uint8_t byte = (uint8_t)row[g.H * (g.d / 2) + h * (g.d / 32) + vec / 4];
      w = decode8(codes, block_scale(byte));
    } else {
      w = *reinterpret_cast<const u32x4*>(row + (h * g.d + vec * 8) * 2);
    }
  }
  *reinterpret_cast<u32x4*>(out.base + (b * out.ld_seq + c * out.ld_tok + h * out.ld_head + vec * 8) * 2) = w;
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, bool q4, hipStream_t s) {
  const int64_t tokens = (int64_t)a.pg.B * a.pg.C;
  const int64_t nq = a.q.base ? (tokens * a.heads * (a.pg.d / 16) + 255) / 256 : 0;
  const int64_t nkv = (tokens * 2 * a.pg.H * (a.pg.d / 8) + 255) / 256;
  if (q4)
    hipLaunchKernelGGL(k_append<true>, linear_grid(nq + nkv, 256), dim3(256), 0, s, a, nq);
  else
    hipLaunchKernelGGL(k_append<false>, linear_grid(nq + nkv, 256), dim3(256), 0, s, a, nq);
  return hipGetLastError();
}

hipError_t launch_read(const ReadArgs& a, bool q4, hipStream_t s) {
  const int64_t n = ((int64_t)a.pg.B * a.pg.C * 2 * a.pg.H * (a.pg.d / 8) + 255) / 256;
  if (q4)
    hipLaunchKernelGGL(k_read<true>, linear_grid(n, 256), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_read<false>, linear_grid(n, 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace epikv
