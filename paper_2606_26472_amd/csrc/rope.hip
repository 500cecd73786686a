// Rotary positions: the table of cosines and sines, and the rotation of a
// tensor of heads (also its gradient, the transposed rotation).
#include "rope_impl.h"

namespace epikv {
namespace {

// One thread per (position, pair): the pair's frequency, its angle, cosine
// and sine in 64 bits (an angle of 2^24 radians keeps 28 bits after the
// point), rounded to float32 once.  Bound by the 64-bit functions: 131072
// positions of 64 pairs 87 us, once for a model.
__global__ __launch_bounds__(256) void k_rope_table(RopeTableArgs a) {
  const int64_t t = linear_block() * 256 + threadIdx.x;
  if (t >= (int64_t)a.n_pos * a.half) return;
  const int p = (int)(t / a.half), i = (int)(t - (int64_t)p * a.half);
  const double r = 2.0 * a.half;
  double theta = a.theta;
  if (a.scaling == EPIKV_ROPE_NTK) theta *= pow(a.factor, r / (r - 2.0));
  double f = pow(theta, -2.0 * i / r);
  const double two_pi = 6.283185307179586476925;
  if (a.scaling == EPIKV_ROPE_LINEAR) f /= a.factor;
  if (a.scaling == EPIKV_ROPE_BANDS) {
    const double turns = a.original * f / two_pi;
    const double g = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
    f = g * f + (1.0 - g) * f / a.factor;
  }
  if (a.scaling == EPIKV_ROPE_YARN) {
    const double per = 0.5 * r / log(theta);
    const double lo = fmax(floor(per * log(a.original / (two_pi * a.high))), 0.0);
    double hi = fmin(ceil(per * log(a.original / (two_pi * a.low))), r - 1.0);
    if (hi == lo) hi += 0.001;
    const double g = 1.0 - fmin(fmax((i - lo) / (hi - lo), 0.0), 1.0);
    f = g * f + (1.0 - g) * f / a.factor;
  }
  double s, c;
  sincos(p * f, &s, &c);
  a.table[2 * t] = (float)(a.amplitude * c);
  a.table[2 * t + 1] = (float)(a.amplitude * s);
}

// A thread per two 16-byte vectors of a head (rope_items): what a rotation in
// place overwrites it has read.  (Two or four heads a thread share a read of
// the table, which the cache serves as well: 45.0 and 46.3 against 45.3 us for
// 16384 tokens of 32 heads of 128, 44.6 and 45.7 against 43.5 in float32.)
//
// Bound by HBM: every byte of x once and of y once, past the caches; 6.1 TB/s
// there.
template <bool FP32, bool WAVE>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, int per) {
  const Place at = place_of<WAVE>(linear_block(), per, (int64_t)a.B * a.C);
  if (!at.in) return;
  const int b = at.token / a.C, c = at.token - b * a.C;
  const int iph = a.d / (FP32 ? 8 : 16);
  const int h = at.item / iph;
  rope_items<FP32, 1>(a.x, a.y, a.rope, a.status, b, c, h, 0, at.item - h * iph, a.d);
}

template <bool FP32>
hipError_t launch_rope_type(const RopeArgs& a, hipStream_t s) {
  const int per = a.heads * (a.d / (FP32 ? 8 : 16));
  const dim3 grid = linear_grid(((int64_t)a.B * a.C * per + 255) / 256, 256);
  if (per % 64 == 0)
    hipLaunchKernelGGL((k_rope<FP32, true>), grid, dim3(256), 0, s, a, per);
  else
    hipLaunchKernelGGL((k_rope<FP32, false>), grid, dim3(256), 0, s, a, per);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.n_pos * a.half;
  hipLaunchKernelGGL(k_rope_table, linear_grid((n + 255) / 256, 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

bool rope_fits(int64_t tokens, int heads, int d) {
  return threads_fit(tokens, heads * (d / 8));
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  return a.fp32 ? launch_rope_type<true>(a, s) : launch_rope_type<false>(a, s);
}

}  // namespace epikv
