// Attention for few query rows per KV head that sums its weights per slot.
//
// The walk keeps its scores (attend_wave_impl.h): 4 bytes a row and slot, where
// the keys they come from have 256 (128 channels in bf16) for a KV head's rows
// together.  One launch then joins the shares and, in workgroups of their own
// that make the rows' maxima and sums from the shares' once more, turns the scores
// to weights and adds them up.
//
// The walk is bound by HBM still, its writes at a quarter of the reads' rate: 32
// sequences of 8k-32k slots (8 KV heads of 128, 4 query heads each) 470 us, 406
// without the scores (84 MB beside 2.69 GB); in 4 bits 166, 138.  The sums there
// 17.5 us after the join's 5.7 (4.8 TB/s), one sequence of 4224 slots 7.1 with it
// (the join alone 5.6): latency.
#include "attend_wave_impl.h"

namespace epikv {
namespace {

constexpr int kWeighSlots = 256;   // of a workgroup, four to a lane
constexpr int kWeighRows = kWaveRows * (kMaxRowChannels / 64);  // that count, of all KV heads, at most
constexpr int kMaxTiles = 16384;   // workgroups, about; each goes on to further slots

struct WeighScratch {
  float2 norm[kWeighRows];
  __attribute__((aligned(16))) float sums[8][kWeighSlots];
};

// What makes weights of one row's scores (norm_of), from its shares, by `lanes`
// lanes that each take some, two at a time.  (A launch fetches its instructions
// anew, and more of them cost more than loads that wait for each other: one sequence
// of 4224 slots 14.4 us so, 14.9 with four at a time, 15.5 with eight; so it is with
// the rows below.)
__device__ __forceinline__ float2 norm_of_shares(const AttendArgs& a, const WavePlan& p, int b, int h, int r,
                                                 int2 place, int part, int lanes) {
  constexpr int AHEAD = 2;
  const int64_t from = ((int64_t)(place.x + b) * a.pg.H + h) * a.R + r, step = (int64_t)a.pg.H * a.R;
  float top = kNegInf, s = 0.f;
  for (int k = part; k < place.y; k += AHEAD * lanes) {
    float2 ml[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ml[u] = p.part_ml[from + min(k + u * lanes, place.y - 1) * step];
    float grown = top;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) grown = fmaxf(grown, ml[u].x);
    const float base2 = grown == kNegInf ? 0.f : grown;
    s *= exp2_fast(top - base2);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) s += k + u * lanes < place.y ? ml[u].y * exp2_fast(ml[u].x - base2) : 0.f;
    top = grown;
  }
  for (int m = 1; m < lanes; m <<= 1) {
    const float top2 = __shfl_xor(top, m), s2 = __shfl_xor(s, m);
    const float grown = fmaxf(top, top2);
    const float base2 = grown == kNegInf ? 0.f : grown;
    s = s * exp2_fast(top - base2) + s2 * exp2_fast(top2 - base2);
    top = grown;
  }
  return norm_of(top, s, (top + __builtin_amdgcn_logf(s)) * kLn2);
}

// The sums of 256 slots, four to a lane, a workgroup's wavefronts taking turns
// over the counted rows.  SHARES: the rows' norms are made from their shares here;
// else (and where a row has one share, the whole) they are in a.norms.
template <bool SHARES>
__device__ __forceinline__ void weigh_slots(const AttendArgs& a, const WavePlan& p, const WeighArgs& w, int b,
                                            int tile, const SeqTokens& t, WeighScratch& lds) {
  constexpr int AHEAD = SHARES ? 4 : 8;  // rows of a wavefront on their way
  const PagedArgs& g = a.pg;
  const int j0 = tile * kWeighSlots;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int first = max(0, t.nn - w.watch) * a.G;      // rows of a KV head that count: [first, nn * G)
  const int per_head = t.nn * a.G - first, rows = per_head * g.H;
  // (rows are divided by 16 at most: one division here, a product each)
  const uint32_t inverse = 0xffffffffu / (uint32_t)per_head + 1u, inverse_g = 0xffffffffu / (uint32_t)a.G + 1u;
  auto head_of = [&](int row) { return per_head == 1 ? row : (int)__umulhi((uint32_t)row, inverse); };
  const int2 place = SHARES ? p.shares[b] : make_int2(0, 1);
  const int j = j0 + 4 * lane;
  const bool some = j < t.n;  // (scores are there to the end of a unit)
  const float* kept = p.kept + p.kept_at(b, 0, j / kUnit, a.G, g.H) + j % kUnit;
  const int64_t per_kv_head = p.kept_at(0, 1, 0, a.G, g.H);
  auto norm_at = [&](int h, int r) {
    const int c = a.G == 1 ? r : (int)__umulhi((uint32_t)r, inverse_g), hq = h * a.G + (r - c * a.G);
    return a.norms[((int64_t)b * a.heads + hq) * g.C + c];
  };
  // (a workgroup has a thread for every slot; the old sum is on its way meanwhile)
  const bool live = threadIdx.x < kWeighSlots && j0 + (int)threadIdx.x < t.n;
  const bool mine = live && j0 + (int)threadIdx.x < w.ld_s;
  if (live && !mine) raise_flag(g.status, b);
  const float kept_old = mine ? kept_sum(w, b, j0 + (int)threadIdx.x, t) : 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if constexpr (SHARES) {
    // (as many lanes to a row as the rows leave each, a power of two)
    int lanes = 1;
    while (lanes < 64 && 2 * lanes * rows <= (int)blockDim.x) lanes *= 2;
    for (int i = threadIdx.x / lanes; i < rows; i += blockDim.x / lanes) {
      const int h = head_of(i), r = first + i - h * per_head;
      const int part = threadIdx.x & (lanes - 1);
      // (whole: the walk wrote it)
      const float2 norm = place.y == 1 ? norm_at(h, r) : norm_of_shares(a, p, b, h, r, place, part, lanes);
      if (part == 0) lds.norm[i] = norm;
    }
    __syncthreads();
  }
  for (int i = wave; i < rows; i += AHEAD * waves) {
    f32x4 x[AHEAD];
    float2 norm[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int k = min(i + u * waves, rows - 1), h = head_of(k), r = k - h * per_head;
      // (they are not read again; that and the products in the divisions' place: 32
      // sequences in 4 bits 191.4 -> 190.0 us, in bf16 496 -> 493.5)
      if (some) x[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(kept + h * per_kv_head + r * kUnit));
      norm[u] = SHARES ? lds.norm[k] : norm_at(h, first + r);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i + u * waves >= rows) continue;
      // (a slot that the row does not see has -infinity.  No branch over rows that
      // do not count: one sequence of 4224 slots 16.1 us so, 17.4 with it)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += weight_of(x[u][e], a.scale2, norm[u]);
    }
  }
  *reinterpret_cast<f32x4*>(&lds.sums[wave][4 * lane]) = sum;
  __syncthreads();
  if (mine) {
    float y = 0.f;
    for (int k = 0; k < waves; ++k) y += lds.sums[k][threadIdx.x];
    write_sum(w, b, j0 + (int)threadIdx.x, kept_old, y);
  }
}

template <bool SHARES>
__device__ __forceinline__ void weigh_tiles(const AttendArgs& a, const WavePlan& p, const WeighArgs& w, int64_t block,
                                            int tiles, WeighScratch& lds) {
  const int64_t b = block / tiles;
  if (b >= a.pg.B) return;
  const SeqTokens t = seq_tokens(a.pg, (int)b);
  if (t.nn == 0) return;
  // (a table may cover far more than the sequence holds)
  for (int tile = (int)(block - b * tiles); (int64_t)tile * kWeighSlots < t.n; tile += tiles) {
    weigh_slots<SHARES>(a, p, w, (int)b, tile, t, lds);
    __syncthreads();
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
  if (block < n_join)
    join_row<D, true>(a, p, block, lds.join);
  else
    weigh_tiles<true>(a, p, w, block - n_join, tiles, lds.weigh);
}

// The sums alone, after a join that leaves every row's norm.
__global__ __launch_bounds__(256) void k_weigh(AttendArgs a, WavePlan p, WeighArgs w, int tiles) {
  __shared__ WeighScratch lds;
  weigh_tiles<false>(a, p, w, linear_block(), tiles, lds);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int units_in(int slots) { return (slots + kUnit - 1) / kUnit; }

// Tiles of all sequences up to which their rows' norms are made beside the join, in
// every tile's workgroup anew; more wait for it.  A launch less against that work:
// one sequence of 32k slots 31.6 us beside, 35.1 after; of 64k 60.9, 61.0; of 128k
// 108.7, 105.7.
constexpr int kMergeTiles = 256;

template <int D>
hipError_t launch_weigh(const AttendArgs& a, const WavePlan& p, const WeighArgs& w, bool q4, hipStream_t s) {
  hipError_t e = launch_shares<D, true>(a, p, q4, s);
  if (e != hipSuccess) return e;
  const int all_tiles = (a.pg.max_tokens + kWeighSlots - 1) / kWeighSlots;
  const int tiles = std::min(all_tiles, std::max(1, kMaxTiles / a.pg.B));
  const int64_t blocks = (int64_t)a.pg.B * tiles;
  const bool merge = p.split && (int64_t)a.pg.B * all_tiles <= kMergeTiles;
  if (p.split) {
    const int waves = join_waves(p, a.pg.B);
    const int64_t n_join = (int64_t)a.pg.B * a.pg.H * a.R;
    hipLaunchKernelGGL(k_join_weigh<D>, linear_grid(n_join + (merge ? blocks : 0), waves * 64), dim3(waves * 64), 0, s, a,
                       p, w, n_join, tiles);
    e = hipGetLastError();
    if (e != hipSuccess || merge) return e;
  }
  hipLaunchKernelGGL(k_weigh, linear_grid(blocks, 256), dim3(256), 0, s, a, p, w, tiles);
  return hipGetLastError();
}

}  // namespace

size_t weigh_wave_workspace(int B, int H, int R, int d, int G, int slots, int watch) {
  return round256(attend_wave_workspace(B, H, R, d)) + round256((size_t)B * H * R * sizeof(float2)) +
         (size_t)B * units_in(slots) * (H * watch * G) * kUnit * sizeof(float);
}

hipError_t launch_weigh_wave(const AttendArgs& args, const WeighArgs& w, bool q4, void* ws, hipStream_t s) {
  AttendArgs a = args;
  const PagedArgs& g = a.pg;
  WavePlan p = placed_plan(a, ws);
  char* at = (char*)ws + round256(attend_wave_workspace(g.B, g.H, a.R, g.d));
  a.norms = (float2*)at;
  p.kept = (float*)(at + round256((size_t)g.B * g.H * a.R * sizeof(float2)));
  p.units = units_in(g.max_tokens);
  p.watch = w.watch;
  if (g.d == 64) return launch_weigh<64>(a, p, w, q4, s);
  if (g.d == 128) return launch_weigh<128>(a, p, w, q4, s);
  return launch_weigh<256>(a, p, w, q4, s);
}

}  // namespace epikv
