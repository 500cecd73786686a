// Attention that also sums, per slot, the weights that its queries gave.
//
//   weights[b][j] = keep * old[b][j] + gain * sum exp(scale * (q . k_j) - lse)
//
// over the counted rows (tokens times query heads) that see slot j.  The sums
// need every row's final maximum and sum, so they are taken after the attention: from
// scores that it kept where rows are few (weigh_wave.hip), from scores made
// again where they are many (weigh_tile.hip).
//
// Few are those that the attention walks with, 16 a KV head.  32 sequences of 8k-32k
// slots (8 KV heads of 128, 4 query heads each), one to four tokens: kept 189, 228,
// 267, 298 us in 4 bits and 492, 560, 619, 663 in bf16.  k_weigh_tile takes 380 us
// for them, whatever the rows: after the same attention 528 to 549 and 795 to 827.
// One sequence of 32k 22 to 40 and 32 to 47 us kept, 81 to 84 and 75 to 78 with tiles
// for both.  (Kept scores cost 4 bytes a row and slot, so that by their bytes a walk
// over the keys alone, which is not built, would be cheaper from some 5 rows on in 4
// bits, 11 in bf16.)
#include "attend_impl.h"

namespace epikv {
namespace {

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t attend_weigh_workspace(int B, int C, int H, int heads, int d, int slots, int watch) {
  const int G = heads / H, R = C * G;
  if (R <= kWaveRows) return weigh_wave_workspace(B, H, R, d, G, slots, watch);
  return round256((size_t)B * C * heads * sizeof(float2)) +
         std::max(attend_tile_workspace(B, H, R, d), weigh_tile_workspace(B, H, G, d, slots, watch));
}

hipError_t launch_attend_weigh(const AttendArgs& args, const WeighArgs& w, bool q4, void* ws, hipStream_t s) {
  if (args.R <= kWaveRows) return launch_weigh_wave(args, w, q4, ws, s);
  AttendArgs a = args;
  a.norms = (float2*)ws;
  // (the attention is done with its workspace when the sums begin)
  void* rest = (char*)ws + round256((size_t)a.pg.B * a.pg.C * a.heads * sizeof(float2));
  const hipError_t e = launch_attend_tile(a, q4, rest, s);
  return e != hipSuccess ? e : launch_weigh_tile(a, w, q4, rest, s);
}

}  // namespace epikv
