// New keys and values into the cache's pages (append_impl.h), and rows back.
#include "append_impl.h"

namespace epikv {
namespace {

// Rows back: a thread per 8 channels of U heads.  Bound by HBM: 8191 4-bit tokens
// of 8 heads of 128 (42 MB) 9.4 us, 4.5 TB/s, a launch's 2 us among them.
template <bool Q4, bool WAVE, int U>
__global__ __launch_bounds__(256) void k_read(ReadArgs a, int per) {
  const PagedArgs& g = a.pg;
  const Place at = place_of<WAVE>(linear_block(), per, (int64_t)g.B * g.C);
  if (!at.in) return;
  const int b = at.token / g.C, c = at.token - b * g.C;
  const int vph = g.d / 8, heads = g.H / U;
  const int hv = at.item / vph, kv = hv / heads, h = hv - kv * heads, vec = at.item - hv * vph;
  const RowsArg& out = kv ? a.v : a.k;
  if (!out.base) return;
  const int64_t slot = (int64_t)g.n_cached[b] + c;
  const int64_t off = slot >= 0 && slot < g.max_tokens ? row_offset(g, b, (int)slot) : -1;
  if (off < 0) raise_flag(g.status, b);
  const char* row = g.plane[kv] + max(off, (int64_t)0);
  u32x4 w[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int head = h + i * heads;
    if constexpr (Q4) {
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(row + head * (g.d / 2) + vec * 4);
      const uint8_t byte = (uint8_t)row[g.H * (g.d / 2) + head * (g.d / 32) + vec / 4];
      w[i] = decode8(codes, block_scale(byte));
    } else {
      w[i] = *reinterpret_cast<const u32x4*>(row + (head * g.d + vec * 8) * 2);
    }
    if (off < 0) w[i] = u32x4{0, 0, 0, 0};
  }
  char* o = out.base + (b * out.ld_seq + c * out.ld_tok + h * out.ld_head + vec * 8) * 2;
#pragma unroll
  for (int i = 0; i < U; ++i) st_stream(o + i * heads * out.ld_head * 2, w[i]);
}

template <bool Q4, int U>
hipError_t launch_read_heads(const ReadArgs& a, hipStream_t s) {
  const int per = 2 * (a.pg.H / U) * (a.pg.d / 8);
  const dim3 grid = linear_grid(((int64_t)a.pg.B * a.pg.C * per + 255) / 256, 256);
  if (per % 64 == 0)
    hipLaunchKernelGGL((k_read<Q4, true, U>), grid, dim3(256), 0, s, a, per);
  else
    hipLaunchKernelGGL((k_read<Q4, false, U>), grid, dim3(256), 0, s, a, per);
  return hipGetLastError();
}

}  // namespace

bool append_fits(int64_t tokens, int H, int heads, int d) {
  return threads_fit(tokens, 2 * (H / heads_at_once(H)) * (d / 8)) &&
         (heads == 0 || threads_fit(tokens, heads / heads_at_once(heads) * (d / 16)));
}

hipError_t launch_append(const AppendArgs& a, bool q4, hipStream_t s) {
  return q4 ? launch_append_fmt<true>(a, s) : launch_append_fmt<false>(a, s);
}

hipError_t launch_read(const ReadArgs& a, bool q4, hipStream_t s) {
  if (heads_at_once(a.pg.H) == 2) return q4 ? launch_read_heads<true, 2>(a, s) : launch_read_heads<false, 2>(a, s);
  return q4 ? launch_read_heads<true, 1>(a, s) : launch_read_heads<false, 1>(a, s);
}

}  // namespace epikv
