// Attention of the new tokens' queries over the paged cache.
//
// out = sum_j w_j v_j / sum_j w_j with w_j = exp(scale * (q . k_j) - top), in
// one pass over the rows: the running maximum `top` and the sums made with
// it are rescaled when it grows.
#include "attend_impl.h"

namespace epikv {
namespace {

// A wavefront per (query head, token, sequence): each lane holds D / 64
// channels of the query, the running output and the row in flight.
template <int D, bool Q4>
__global__ __launch_bounds__(64) void k_attend_plain(AttendArgs a) {
  constexpr int E = D / 64;
  const PagedArgs& g = a.pg;
  const int lane = threadIdx.x;
  const int64_t w = linear_block();
  const int64_t token = w / a.heads;
  if (token >= (int64_t)g.B * g.C) return;
  const int hq = (int)(w - token * a.heads);
  const int b = (int)(token / g.C), c = (int)(token - (int64_t)b * g.C);
  const int h = hq / a.G;
  const SeqTokens t = seq_tokens(g, b);
  if (t.bad && lane == 0) raise_flag(g.status, b);
  const bool real = c < t.nn;
  const int end = real ? t.n - t.nn + c + 1 : 0;
  float q[E], o[E];
  const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q.base) + b * a.q.ld_seq +
                       c * a.q.ld_tok + hq * a.q.ld_head;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    q[i] = real ? bf16_lo(qp[lane * E + i]) * a.scale2 : 0.f;
    o[i] = 0.f;
  }
  float top = -__builtin_inff(), sum = 0.f;
  for (int j = 0; j < end; ++j) {
    const int64_t off = row_offset(g, b, j);
    if (off < 0) {
      if (lane == 0) raise_flag(g.status, b);
      continue;
    }
    float k[E], v[E];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float* x = kv ? v : k;
      const char* row = g.plane[kv] + off;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int ch = h * D + lane * E + i;
        if constexpr (Q4) {
          const uint32_t byte = (uint8_t)row[g.H * (D / 2) + ch / 32];
          const uint32_t code = ((uint8_t)row[ch / 2] >> (4 * (ch & 1))) & 15u;
          x[i] = bf16_lo(decode8(code, block_scale(byte))[0]);
        } else {
          x[i] = bf16_lo(reinterpret_cast<const uint16_t*>(row)[ch]);
        }
      }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += q[i] * k[i];
    s = wave_sum(s);
    if (s > top) {
      const float f = exp2f(top - s);
      sum *= f;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] *= f;
      top = s;
    }
    const float w = s == -__builtin_inff() ? 0.f : exp2f(s - top);
    sum += w;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] += w * v[i];
  }
  uint16_t* op = reinterpret_cast<uint16_t*>(a.out.base) + b * a.out.ld_seq + c * a.out.ld_tok +
                 hq * a.out.ld_head;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float y = sum == 0.f ? 0.f : o[i] / sum;
    op[lane * E + i] = (uint16_t)pack_bf16(y, 0.f);
  }
  if (a.lse && lane == 0)
    a.lse[((int64_t)b * a.heads + hq) * g.C + c] =
        sum == 0.f ? -__builtin_inff() : (top + log2f(sum)) * 0.69314718055994531f;
}

template <int D>
hipError_t launch_plain(const AttendArgs& a, bool q4, hipStream_t s) {
  const dim3 grid = linear_grid((int64_t)a.pg.B * a.pg.C * a.heads, 64);
  if (q4)
    hipLaunchKernelGGL((k_attend_plain<D, true>), grid, dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL((k_attend_plain<D, false>), grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace(int B, int C, int H, int heads, int d, bool) {
  const int R = C * (heads / H);
  return attend_wave_tiles(R) ? attend_wave_workspace(B, H, R, d) : 0;
}

hipError_t launch_attend(const AttendArgs& a, bool q4, void* ws, hipStream_t s) {
  if (attend_wave_tiles(a.R)) return launch_attend_wave(a, q4, ws, s);
  if (a.pg.d == 64) return launch_plain<64>(a, q4, s);
  if (a.pg.d == 128) return launch_plain<128>(a, q4, s);
  return launch_plain<256>(a, q4, s);
}

}  // namespace epikv
