// Attention for few query rows per KV head that sums its weights per slot.
//
// The walk keeps its scores (attend_wave_impl.h): 4 bytes a row and slot, where
// the keys they come from have 256 (128 channels in bf16) for a KV head's rows
// together.  One launch then joins the shares and, in workgroups of their own
// that make the rows' log-sums from the shares' once more, turns the scores to
// weights and adds them up.
#include "attend_wave_impl.h"

namespace epikv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWeighSlots = 256;   // of a workgroup, four to a lane
constexpr int kWeighRows = 512;    // rows whose log-sums a workgroup holds at a time
constexpr int kMaxTiles = 16384;   // workgroups, about; each goes on to further slots
constexpr int kRowThreads = 8;     // that read a row's shares

struct WeighScratch {
  float lse[kWeighRows];                       // base 2
  __attribute__((aligned(16))) float sums[8][kWeighSlots];
};

__device__ __forceinline__ void weigh_slots(const AttendArgs& a, const WavePlan& p, const WeighArgs& w, int b,
                                            int tile, const SeqTokens& t, WeighScratch& lds) {
  const PagedArgs& g = a.pg;
  const int j0 = tile * kWeighSlots;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int first = max(0, t.nn - w.watch) * a.G;      // rows of a KV head that count: [first, nn * G)
  const int per_head = t.nn * a.G - first, rows = per_head * g.H;
  const int2 place = p.split ? p.shares[b] : make_int2(0, 1);
  const int j = j0 + 4 * lane;
  const bool some = j < t.n;  // (scores are there to the end of a unit)
  const float* kept = p.kept + p.kept_at(b, 0, j / kUnit, a.G, g.H) + j % kUnit;
  const int64_t per_kv_head = p.kept_at(0, 1, 0, a.G, g.H);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int at = 0; at < rows; at += kWeighRows) {
    const int n = min(kWeighRows, rows - at);
    if (at) __syncthreads();
    for (int i = threadIdx.x / kRowThreads; i < n; i += blockDim.x / kRowThreads) {
      const int h = (at + i) / per_head, r = first + (at + i) - h * per_head;
      const int part = threadIdx.x % kRowThreads;
      float lse;
      if (place.y == 1) {  // whole: the walk wrote it
        const int c = r / a.G, hq = h * a.G + (r - c * a.G);
        lse = a.lse[((int64_t)b * a.heads + hq) * g.C + c] * kLog2e;
      } else {
        const int64_t from = ((int64_t)(place.x + b) * g.H + h) * a.R + r, step = (int64_t)g.H * a.R;
        float top = kNegInf, s = 0.f;
        for (int k = part; k < place.y; k += 4 * kRowThreads) {
          float2 ml[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            ml[u] = p.part_ml[from + min(k + u * kRowThreads, place.y - 1) * step];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (k + u * kRowThreads >= place.y) continue;
            const float grown = fmaxf(top, ml[u].x);
            const float base2 = grown == kNegInf ? 0.f : grown;
            s = s * exp2_fast(top - base2) + ml[u].y * exp2_fast(ml[u].x - base2);
            top = grown;
          }
        }
#pragma unroll
        for (int m = 1; m < kRowThreads; m <<= 1) {
          const float top2 = __shfl_xor(top, m), s2 = __shfl_xor(s, m);
          const float grown = fmaxf(top, top2);
          const float base2 = grown == kNegInf ? 0.f : grown;
          s = s * exp2_fast(top - base2) + s2 * exp2_fast(top2 - base2);
          top = grown;
        }
        lse = top + __builtin_amdgcn_logf(s);
      }
      if (part == 0) lds.lse[i] = lse_of_weights(lse);
    }
    __syncthreads();
    if (!some) continue;
    constexpr int AHEAD = 8;
    for (int i = wave; i < n; i += AHEAD * waves) {
      f32x4 x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int q = at + min(i + u * waves, n - 1);
        const int h = q / per_head;
        x[u] = *reinterpret_cast<const f32x4*>(kept + h * per_kv_head + (q - h * per_head) * kUnit);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (i + u * waves >= n) continue;
        const float lse = lds.lse[i + u * waves];
        // (a slot that the row does not see has -infinity, whatever its log-sum)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[u][e] == kNegInf ? 0.f : weight_of(x[u][e], a.scale2, lse);
      }
    }
  }
  *reinterpret_cast<f32x4*>(&lds.sums[wave][4 * lane]) = sum;
  __syncthreads();
  for (int i = threadIdx.x; i < kWeighSlots; i += blockDim.x) {
    if (j0 + i >= t.n) continue;
    if (j0 + i >= w.ld_s) {
      raise_flag(g.status, b);
      continue;
    }
    float y = 0.f;
    for (int k = 0; k < waves; ++k) y += lds.sums[k][i];
    write_sum(w, b, j0 + i, t, y);
  }
}

// Workgroups of the join, then those of the sums: both need what the walk left
// and nothing of each other.
template <int D>
__global__ __launch_bounds__(512) void k_join_weigh(AttendArgs a, WavePlan p, WeighArgs w, int64_t n_join, int tiles) {
  __shared__ union {
    JoinScratch<D> join;
    WeighScratch weigh;
  } lds;
  const int64_t block = linear_block();
  if (block < n_join) {
    join_row<D>(a, p, block, lds.join);
    return;
  }
  const int64_t at = block - n_join, b = at / tiles;
  if (b >= a.pg.B) return;
  const SeqTokens t = seq_tokens(a.pg, (int)b);
  if (t.nn == 0) return;
  // (a table may cover far more than the sequence holds)
  for (int tile = (int)(at - b * tiles); (int64_t)tile * kWeighSlots < t.n; tile += tiles) {
    weigh_slots(a, p, w, (int)b, tile, t, lds.weigh);
    __syncthreads();
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int units_in(int slots) { return (slots + kUnit - 1) / kUnit; }

template <int D>
hipError_t launch_weigh(const AttendArgs& a, const WavePlan& p, const WeighArgs& w, bool q4, hipStream_t s) {
  const hipError_t e = launch_shares<D, true>(a, p, q4, s);
  if (e != hipSuccess) return e;
  const int waves = p.split ? join_waves(p, a.pg.B) : 4;
  const int tiles = std::min((a.pg.max_tokens + kWeighSlots - 1) / kWeighSlots, std::max(1, kMaxTiles / a.pg.B));
  const int64_t n_join = p.split ? (int64_t)a.pg.B * a.pg.H * a.R : 0;
  hipLaunchKernelGGL(k_join_weigh<D>, linear_grid(n_join + (int64_t)a.pg.B * tiles, waves * 64), dim3(waves * 64), 0, s,
                     a, p, w, n_join, tiles);
  return hipGetLastError();
}

}  // namespace

size_t weigh_wave_workspace(int B, int H, int R, int d, int G, int slots, int watch) {
  return round256(attend_wave_workspace(B, H, R, d)) + round256((size_t)B * H * R * sizeof(float)) +
         (size_t)B * units_in(slots) * (H * watch * G) * kUnit * sizeof(float);
}

hipError_t launch_weigh_wave(const AttendArgs& args, const WeighArgs& w, bool q4, void* ws, hipStream_t s) {
  AttendArgs a = args;
  const PagedArgs& g = a.pg;
  WavePlan p = placed_plan(a, ws);
  char* at = (char*)ws + round256(attend_wave_workspace(g.B, g.H, a.R, g.d));
  if (!a.lse) a.lse = (float*)at;
  p.kept = (float*)(at + round256((size_t)g.B * g.H * a.R * sizeof(float)));
  p.units = units_in(g.max_tokens);
  p.watch = w.watch;
  if (g.d == 64) return launch_weigh<64>(a, p, w, q4, s);
  if (g.d == 128) return launch_weigh<128>(a, p, w, q4, s);
  return launch_weigh<256>(a, p, w, q4, s);
}

}  // namespace epikv
