// Attention of the new tokens' queries over the paged cache.
//
// out = sum_j w_j v_j / sum_j w_j with w_j = exp(scale * (q . k_j) - top), in
// one pass over the rows: what was summed so far is rescaled when the running
// maximum `top` grows.  Up to 16 query rows per KV head (tokens times heads of
// its group) are bound by reading the rows and go to a wavefront per share of
// a sequence (attend_wave.hip); more are bound by the matrix cores and go to
// workgroups of 256 rows, or of 128 (attend_tile.hip).
#include "attend_impl.h"

namespace epikv {

size_t attend_workspace(int B, int C, int H, int heads, int d) {
  const int R = C * (heads / H);
  return R <= kWaveRows ? attend_wave_workspace(B, H, R, d) : attend_tile_workspace(B, H, R, d);
}

hipError_t launch_attend(const AttendArgs& a, bool q4, void* ws, hipStream_t s) {
  return a.R <= kWaveRows ? launch_attend_wave(a, q4, ws, s) : launch_attend_tile(a, q4, ws, s);
}

}  // namespace epikv
