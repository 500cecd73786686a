// Attention for few query rows per KV head: the walk (attend_wave_impl.h) and
// the join of its shares.
#include "attend_wave_impl.h"

namespace epikv {
namespace {

template <int D>
__global__ __launch_bounds__(512) void k_attend_join(AttendArgs a, WavePlan p) {
  __shared__ JoinScratch<D> lds;
  join_row<D, false>(a, p, linear_block(), lds);
}

template <int D>
hipError_t launch_wave(const AttendArgs& a, const WavePlan& p, bool q4, hipStream_t s) {
  const hipError_t e = launch_shares<D, false>(a, p, q4, s);
  if (e != hipSuccess || !p.split) return e;
  const int waves = join_waves(p, a.pg.B);
  hipLaunchKernelGGL(k_attend_join<D>, linear_grid((int64_t)a.pg.B * a.pg.H * a.R, waves * 64),
                     dim3(waves * 64), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace

size_t attend_wave_workspace(int B, int H, int R, int d) {
  const WavePlan p = wave_plan(B, H, d);
  if (!p.split) return 0;
  return kSharesBytes + part_ml_bytes(p, B, H, R) + (size_t)(p.n_teams + B) * H * R * d * sizeof(float);
}

hipError_t launch_attend_wave(const AttendArgs& a, bool q4, void* ws, hipStream_t s) {
  const WavePlan p = placed_plan(a, ws);
  if (a.pg.d == 64) return launch_wave<64>(a, p, q4, s);
  if (a.pg.d == 128) return launch_wave<128>(a, p, q4, s);
  return launch_wave<256>(a, p, q4, s);
}

}  // namespace epikv
