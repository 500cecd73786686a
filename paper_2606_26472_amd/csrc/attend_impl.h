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

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Query rows per KV head up to which the wavefront kernel is taken: the columns
// of one of its instructions.  (At 32 rows of 128 channels over 8 x 8192 slots
// it took 103 us with two sets of them, the tile kernel takes 60; 16 rows 62.)
constexpr int kWaveRows = 16;
size_t attend_wave_workspace(int B, int H, int R, int d);
hipError_t launch_attend_wave(const AttendArgs& a, bool q4, void* ws, hipStream_t s);
size_t attend_tile_workspace(int B, int H, int R, int d);
hipError_t launch_attend_tile(const AttendArgs& a, bool q4, void* ws, hipStream_t s);

}  // namespace epikv
