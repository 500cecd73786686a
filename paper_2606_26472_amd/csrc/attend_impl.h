// What the attention kernels share: how the tokens are cut into shares, the
// running softmax, and matrix-core fragments.
#pragma once

#include "cache_impl.h"

namespace epikv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kNegInf = -__builtin_inff();

// Tokens of one step of a wavefront's walk along a sequence, the unit that
// shares are counted in.
constexpr int kUnit = 32;

// One sequence's units are cut over several teams of wavefronts when the
// batch is small: all sequences' units in a row, cut into even shares (of one
// unit at least: 4224 slots 14.2 us in shares of two, 13.1 of one), so that
// ragged lengths cost no balance.  A team's share may
// span sequences; its part of sequence b goes to partial slot team + b, which
// no other (team, sequence) pair of the staircase has.
struct WavePlan {
  int32_t n_teams;  // shares (split) or sequences
  int32_t hw;       // KV heads a team (a workgroup) walks side by side, a wavefront each
  int32_t split;    // sequences are cut
  float* part_o;    // [n_teams + B][H][R][d] unnormalised
  float2* part_ml;  // [n_teams + B][H][R] maximum (base 2) and sum
  int2* shares;     // [B] a sequence's first team and how many it has
  // where the scores are kept (for the sums of the weights alone):
  float* kept;      // [B][H][units][watch * G][kUnit]
  int32_t units;    // that the page tables cover
  int32_t watch;    // tokens counted
  __device__ __forceinline__ int64_t kept_at(int b, int h, int unit, int G, int H) const {
    return (((int64_t)b * H + h) * units + unit) * ((int64_t)watch * G * kUnit);
  }
};
constexpr int kSplitBatch = 1024;  // largest batch whose sequences are cut

__device__ __forceinline__ int units_of(const SeqTokens& t) {
  return t.nn > 0 ? (t.n + kUnit - 1) / kUnit : 0;
}

// Inclusive sum over the lanes up to this one: within rows of 16 lanes, then
// the rows' sums on to the rows after them.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr 2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31
  return v;
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }

// Whether one of a word's two bf16 halves is a NaN or an infinity.
__device__ __forceinline__ bool word_not_finite(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// The lowest n bits (none for n <= 0, all for n >= 32).
__device__ __forceinline__ uint32_t below(int n) {
  return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
}

// Lower / upper halves of two words.
__device__ __forceinline__ uint32_t halves_lo(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}
__device__ __forceinline__ uint32_t halves_hi(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Rows of D channels in LDS: where the 16-byte chunk c of a row goes (and which
// chunk a place holds), so that 16 rows' reads of one chunk meet no bank twice.
template <int D>
__device__ __forceinline__ int row_chunk(int row, int c) {
  return c ^ (D == 64 ? (row >> 1) & 7 : row & 15);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Whether a row counts.  One that sees nothing, or has a NaN or +infinity among its
// scores, has no finite log-sum; from 2^30 on a maximum's rounding, 2^-24 of it, is 64 and
// more, and its exponential passes float32 soon after.  Such a row adds nothing to
// any slot, or one token would leave NaN in sums that go on for good.
__device__ __forceinline__ bool row_counts(float lse) { return fabsf(lse) < 0x1p30f; }

// What makes weights of a row's scores: the maximum (base 2) that its sum was taken
// from, and 1 / sum; {0, 0} for a row that does not count.  Not the log-sum, whose
// own rounding, 2^-24 of it, would be an error of every weight: 1 % where scores are
// 1e5, factors where they are 1e7.
__device__ __forceinline__ float2 norm_of(float top, float sum, float lse) {
  return row_counts(lse) ? make_float2(top, 1.f / sum) : make_float2(0.f, 0.f);
}

// A row's weight of a slot.  (The product with the scale is not rounded before the
// maximum is off.)
__device__ __forceinline__ float weight_of(float score, float scale2, float2 norm) {
  const float w = exp2_fast(fmaf(score, scale2, -norm.x)) * norm.y;
  return norm.y != 0.f ? w : 0.f;  // (the score may be NaN)
}

// A row's log-sum, and its norm, where they are asked for.  some: the sum is not 0.
// NORMS: the kernel is asked for norms at all.
template <bool NORMS>
__device__ __forceinline__ void write_log_sum(const AttendArgs& a, int b, int hq, int c, float top, float sum,
                                              bool some) {
  if (!a.lse && !(NORMS && a.norms)) return;
  const int64_t at = ((int64_t)b * a.heads + hq) * a.pg.C + c;
  const float lse = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : kNegInf;
  if (a.lse) a.lse[at] = lse;
  if (NORMS && a.norms) a.norms[at] = norm_of(top, sum, lse);
}

// A slot's sum: what is kept of the old one and this call's.  j < ld_s.
__device__ __forceinline__ float kept_sum(const WeighArgs& w, int b, int64_t j, const SeqTokens& t) {
  const float keep = j < t.n - t.nn ? w.keep_old : w.keep_new;
  return keep != 0.f ? keep * w.old[b * w.ld_s + j] : 0.f;  // (kept by 0: not read)
}
__device__ __forceinline__ void write_sum(const WeighArgs& w, int b, int64_t j, float kept, float sum) {
  w.weights[b * w.ld_s + j] = fmaf(w.gain, sum, kept);
}

// Query rows per KV head up to which the wavefront kernel is taken: the columns
// of one of its instructions.  (At 32 rows of 128 channels over 8 x 8192 slots
// it took 103 us with two sets of them, the tile kernel takes 60; 16 rows 62.)
constexpr int kWaveRows = 16;
size_t attend_wave_workspace(int B, int H, int R, int d);
hipError_t launch_attend_wave(const AttendArgs& a, bool q4, void* ws, hipStream_t s);
// The same, its scores kept and the weights summed.
size_t weigh_wave_workspace(int B, int H, int R, int d, int G, int slots, int watch);
hipError_t launch_weigh_wave(const AttendArgs& a, const WeighArgs& w, bool q4, void* ws, hipStream_t s);
size_t attend_tile_workspace(int B, int H, int R, int d);
size_t weigh_tile_workspace(int B, int H, int G, int d, int slots, int watch);
// After the attention, which left a.norms.
hipError_t launch_weigh_tile(const AttendArgs& a, const WeighArgs& w, bool q4, void* ws, hipStream_t s);
hipError_t launch_attend_tile(const AttendArgs& a, bool q4, void* ws, hipStream_t s);

}  // namespace epikv
