// Attention that also sums, per slot, the weights that its queries gave.
//
//   weights[b][j] = keep * old[b][j] + gain * sum exp(scale * (q . k_j) - lse)
//
// over the counted rows (tokens times query heads) that see slot j: the sums
// need every row's final log-sum, so they are taken after the attention.
#include "attend_impl.h"

namespace epikv {
namespace {

// A thread per slot, which goes over all KV heads and counted rows.
template <bool Q4>
__global__ __launch_bounds__(256) void k_weigh(AttendArgs a, WeighArgs w, int slot_blocks) {
  const PagedArgs& g = a.pg;
  const int64_t id = linear_block();
  const int b = (int)(id / slot_blocks);
  if (b >= g.B) return;
  const SeqTokens t = seq_tokens(g, b);
  const int j = (int)(id - (int64_t)b * slot_blocks) * 256 + (int)threadIdx.x;
  if (t.nn == 0 || j >= t.n) return;
  if (j >= w.ld_s) {
    raise_flag(g.status, b);
    return;
  }
  const int64_t off = row_offset(g, b, j);
  const int old = t.n - t.nn;
  float sum = 0.f;
  if (off >= 0) {
    for (int c = max(max(0, t.nn - w.watch), j - old); c < t.nn; ++c)
      for (int hq = 0; hq < a.heads; ++hq) {
        const int h = hq / a.G;
        const char* qp = a.q.base + (b * a.q.ld_seq + c * a.q.ld_tok + hq * a.q.ld_head) * 2;
        const char* row = g.plane[0] + off;
        float s = 0.f;
        for (int v = 0; v < g.d / 8; ++v) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(qp + 16 * v);
          u32x4 k;
          if constexpr (Q4) {
            const uint32_t codes = *reinterpret_cast<const uint32_t*>(row + h * (g.d / 2) + v * 4);
            const uint8_t byte = (uint8_t)row[g.H * (g.d / 2) + h * (g.d / 32) + v / 4];
            k = decode8(codes, block_scale(byte));
          } else {
            k = *reinterpret_cast<const u32x4*>(row + (h * g.d + v * 8) * 2);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s = fmaf(bf16_lo(x[i]), bf16_lo(k[i]), s);
            s = fmaf(bf16_hi(x[i]), bf16_hi(k[i]), s);
          }
        }
        const float lse = a.lse[((int64_t)b * a.heads + hq) * g.C + c];
        sum += weight_of(s, a.scale2, lse_of_weights(lse * 1.4426950408889634f));
      }
  }
  write_sum(w, b, j, t, sum);
}

size_t lse_bytes(int B, int C, int heads) { return ((size_t)B * C * heads * 4 + 255) / 256 * 256; }

}  // namespace

size_t attend_weigh_workspace(int B, int C, int H, int heads, int d, int slots, int watch) {
  const int G = heads / H, R = C * G;
  if (R <= kWaveRows) return weigh_wave_workspace(B, H, R, d, G, slots, watch);
  return lse_bytes(B, C, heads) + attend_workspace(B, C, H, heads, d);
}

hipError_t launch_attend_weigh(const AttendArgs& args, const WeighArgs& w, bool q4, void* ws, hipStream_t s) {
  if (args.R <= kWaveRows) return launch_weigh_wave(args, w, q4, ws, s);
  AttendArgs a = args;
  const PagedArgs& g = a.pg;
  if (!a.lse) a.lse = (float*)ws;
  hipError_t e = launch_attend(a, q4, (char*)ws + lse_bytes(g.B, g.C, a.heads), s);
  if (e != hipSuccess) return e;
  const int blocks = (g.max_tokens + 255) / 256;
  const dim3 grid = linear_grid((int64_t)g.B * blocks, 256);
  if (q4)
    hipLaunchKernelGGL(k_weigh<true>, grid, dim3(256), 0, s, a, w, blocks);
  else
    hipLaunchKernelGGL(k_weigh<false>, grid, dim3(256), 0, s, a, w, blocks);
  return hipGetLastError();
}

}  // namespace epikv
