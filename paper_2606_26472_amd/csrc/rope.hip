// Rotary positions: the table of cosines and sines, and the rotation of a
// tensor of heads (also its gradient, the transposed rotation).
#include "rope_impl.h"

namespace epikv {
namespace {

// One thread per (position, pair): the pair's frequency, its angle, cosine
// and sine in 64 bits (an angle of 2^24 radians keeps 28 bits after the
// point), rounded to float32 once.
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

// A thread per item: 16 channels of one head, the two 8-vectors whose pairs
// belong together (or two plain ones past rotary_dim), so a rotation in place
// reads all that it overwrites.
template <bool FP32>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, int ipt, int tpb) {
  const int tk = ipt <= 256 ? threadIdx.x / ipt : 0;
  const int it = ipt <= 256 ? threadIdx.x - tk * ipt : (int)(blockIdx.y * 256 + threadIdx.x);
  const int64_t token = linear_block() * tpb + tk;
  if (tk >= tpb || it >= ipt || token >= (int64_t)a.B * a.C) return;
  const int b = (int)(token / a.C), c = (int)(token - (int64_t)b * a.C);
  const int iph = a.d / 16;
  const int h = it / iph;
  rope_item<FP32>(a.x, a.y, a.rope, a.status, b, c, h, it - h * iph);
}

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.n_pos * a.half;
  hipLaunchKernelGGL(k_rope_table, linear_grid((n + 255) / 256, 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  const int ipt = a.heads * (a.d / 16);
  const int tpb = ipt <= 256 ? 256 / ipt : 1;
  const int64_t tokens = (int64_t)a.B * a.C;
  const dim3 grid = linear_grid((tokens + tpb - 1) / tpb, 256, ipt <= 256 ? 1 : (ipt + 255) / 256);
  if (a.fp32)
    hipLaunchKernelGGL(k_rope<true>, grid, dim3(256), 0, s, a, ipt, tpb);
  else
    hipLaunchKernelGGL(k_rope<false>, grid, dim3(256), 0, s, a, ipt, tpb);
  return hipGetLastError();
}

}  // namespace epikv
