// The sums of many query rows' weights per slot (prefill, long chunks), after
// the attention itself.
//
// A row's weights need its log-sum, which is known when the attention ends, so
// the scores are made a second time: a wavefront keeps 64 keys (32 of 256 channels)
// of a KV head in registers as the first operand of v_mfma 32x32x16 and the query rows stream
// past through LDS, 64 at a time and two tiles deep.  S^T = K Q^T, in the
// attention's order of channels (the same scores, bit for bit): lane (n, g) =
// (lane % 32, lane / 32) has query row n's scores of keys 8i + 4g + 0..3, so a
// row's log-sum is one register a lane, and a key's sum stays in one register
// a lane from the first row to the last.  Only then do lanes meet.
#include "attend_impl.h"

namespace epikv {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

constexpr int kWaves = 4;
// Blocks of 32 keys that a wavefront holds (two of 256 channels spill).
constexpr int key_blocks(int d) { return d == 256 ? 1 : 2; }
constexpr int slots_of_group(int d) { return kWaves * 32 * key_blocks(d); }
constexpr int kRows = 64;                  // query rows of a tile, at most
constexpr int kMaxPieces = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLargeLse = 4194304.f;     // from 2^22 on weights are held to 1 one by one

// How the work is dealt out: the slots of every (sequence, KV head) in tiles,
// each tile's rows in `pieces`.
struct WeighPlan {
  int32_t slot_tiles, pieces;
  int32_t tokens;        // of a tile of rows: whole tokens where 64 rows hold a token's
  int32_t head_tiles;    // tiles of a token, where they do not
  int64_t ld;            // of a row of partial sums
  float* part;           // [pieces][B][H][ld]
};

template <int D, bool Q4>
__global__ __launch_bounds__(64 * kWaves, 2) void k_weigh_tile(AttendArgs a, WeighArgs w, WeighPlan p) {
  constexpr int NB = key_blocks(D), kKeys = 32 * NB, kSlots = slots_of_group(D);
  constexpr int KS = D / 16;            // instructions of a product
  constexpr int RC = D / 8;             // 16-byte chunks of a row
  constexpr int RPI = 1024 / (D * 2);   // rows a load of a wavefront
  constexpr int NI = kRows / kWaves / RPI;
  __shared__ __align__(1024) char s_q[2][kRows * D * 2];
  const PagedArgs& g = a.pg;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n = lane & 31, gh = lane >> 5;

  // Heads first, as in the attention: those of one share an XCD's cache.  Slots
  // in rising order: the first are seen by most rows.
  int64_t id = linear_block();
  const int h = (int)(id % g.H);
  id /= g.H;
  const int piece = (int)(id % p.pieces);
  id /= p.pieces;
  const int b = (int)(id / p.slot_tiles);
  if (b >= g.B) return;
  const SeqTokens tk = seq_tokens(g, b);
  const int old = tk.n - tk.nn;

  for (int st = (int)(id % p.slot_tiles); (int64_t)st * kSlots < tk.n && tk.nn > 0; st += p.slot_tiles) {
    const int k0 = st * kSlots, kw = k0 + wave * kKeys;
    // tokens that are counted and see one of these slots
    const int c_lo = max(max(tk.nn - w.watch, k0 - old), 0), c_hi = tk.nn;
    const int tiles = c_lo < c_hi ? (c_hi - c_lo + p.tokens - 1) / p.tokens * p.head_tiles : 0;
    const int t0 = (int)((int64_t)tiles * piece / p.pieces), t1 = (int)((int64_t)tiles * (piece + 1) / p.pieces);

    bf16x8 kf[NB][KS];
    uint64_t ok = 0;  // which of the wavefront's keys exist
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int j = kw + 32 * i + n;
      const int64_t off = j < tk.n ? row_offset(g, b, j) : -1;
      ok |= (__ballot(off >= 0) & 0xffffffffull) << (32 * i);
      const char* row = g.plane[0] + max(off, (int64_t)0);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int ch = 16 * s + 8 * gh;
        u32x4 x;
        if constexpr (Q4) {
          const uint32_t codes = *reinterpret_cast<const uint32_t*>(row + h * (D / 2) + ch / 2);
          const uint8_t byte = (uint8_t)row[g.H * (D / 2) + h * (D / 32) + ch / 32];
          x = decode8(codes, block_scale(byte));
        } else {
          x = *reinterpret_cast<const u32x4*>(row + (h * D + ch) * 2);
        }
        if (off < 0) x = u32x4{0, 0, 0, 0};
        kf[i][s] = as_bf16x8(x);
      }
    }

    // The rows of tile t: tokens from c_of(t), heads of the group from g_of(t).
    auto c_of = [&](int t) { return c_lo + t / p.head_tiles * p.tokens; };
    auto g_of = [&](int t) { return t % p.head_tiles * kRows; };
    const int per = min(a.G, kRows);  // rows of a token in a tile
    // Row `row` of tile t; false: there is none.
    auto has_row = [&](int t, int row) {
      return row / per < min(p.tokens, c_hi - c_of(t)) && g_of(t) + row % per < a.G;
    };
    // (where the lane's rows are from the tile's first one on)
    int64_t q_off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = wave * (kRows / kWaves) + i * RPI + lane / RC;
      q_off[i] = (row / per * a.q.ld_tok + row % per * a.q.ld_head) * 2;
    }
    auto stage = [&](int t, int buf) {
      const char* base = a.q.base + (b * a.q.ld_seq + c_of(t) * a.q.ld_tok + (h * a.G + g_of(t)) * a.q.ld_head) * 2;
      const bool whole = p.tokens * per == kRows && c_hi - c_of(t) >= p.tokens && a.G - g_of(t) >= per;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int first = wave * (kRows / kWaves) + i * RPI;
        const int row = first + lane / RC;
        int64_t off = q_off[i];
        if (!whole && !has_row(t, row)) off = 0;  // (stands for a row that is there)
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) uint32_t*)(base + off + row_chunk<D>(row, lane % RC) * 16),
            (__attribute__((address_space(3))) uint32_t*)(s_q[buf] + first * D * 2), 16, 0, 0);
      }
    };
    // Minus the lane's rows' log-sums; minus infinity where there is no row.
    int64_t lse_off[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) lse_off[i] = (int64_t)((32 * i + n) % per) * g.C + (32 * i + n) / per;
    auto load_lse = [&](int t, float (&neg)[2]) {
      const float* base = a.lse + ((int64_t)b * a.heads + h * a.G + g_of(t)) * g.C + c_of(t);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool there = has_row(t, 32 * i + n);
        const float lse = base[there ? lse_off[i] : 0];
        neg[i] = there ? -lse_of_weights(lse * kLog2e) : kNegInf;
      }
    };
    auto arrived = [&] {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };

    float sum[NB][16];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[i][e] = 0.f;
    const uint32_t q_base = (uint32_t)(uintptr_t)(lds_char*)&s_q[0][0] + n * D * 2 + row_chunk<D>(n, gh) * 16;

    if (t0 < t1) {
      float neg[2], neg_next[2];
      stage(t0, 0);
      load_lse(t0, neg);
      arrived();
      int buf = 0;
      for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) {
          stage(t + 1, buf ^ 1);
          load_lse(t + 1, neg_next);
        }
        const bool all = ok == (NB == 2 ? ~0ull : 0xffffffffull) && old + c_of(t) + 1 >= kw + kKeys;  // every row sees every key
        const uint32_t at = q_base + buf * (kRows * D * 2);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          f32x16 s[NB];
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const bf16x8 q = as_bf16x8(*(const lds_u32x4*)(uintptr_t)((at ^ (32 * k)) + r * 64 * D));
#pragma unroll
            for (int i = 0; i < NB; ++i) s[i] = mfma32(kf[i][k], q, s[i]);
          }
          const bool large = __any(fabsf(neg[r]) > kLargeLse && neg[r] != kNegInf);
          if (all && !large) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
              for (int e = 0; e < 16; ++e) sum[i][e] += exp2_fast(fmaf(s[i][e], a.scale2, neg[r]));
          } else {
            const int row = 32 * r + n;
            const int lim = has_row(t, row) ? old + c_of(t) + row / per + 1 : 0;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              const uint32_t mine = ((uint32_t)(ok >> (32 * i)) & below(lim - kw - 32 * i)) >> (4 * gh);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float x = weight_of(s[i][e], a.scale2, -neg[r]);
                sum[i][e] += mine >> (8 * (e / 4) + e % 4) & 1u ? x : 0.f;
              }
            }
          }
        }
        neg[0] = neg_next[0];
        neg[1] = neg_next[1];
        buf ^= 1;
        arrived();
      }
    }

    // Over the 32 rows' lanes; then key 8(e/4) + 4gh + e%4 of block i is written
    // by lane e of its half.
    float* out = p.part + (((int64_t)piece * g.B + b) * g.H + h) * p.ld + kw;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      float mine = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float v = sum[i][e];
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) v += __shfl_xor(v, m);
        if (n == e) mine = v;
      }
      if (n < 16) out[32 * i + 8 * (n / 4) + 4 * gh + n % 4] = mine;
    }
  }
}

// The partial sums of a slot, in order, on what is kept of the old one.
__global__ __launch_bounds__(256) void k_weigh_reduce(AttendArgs a, WeighArgs w, WeighPlan p, int blocks) {
  const PagedArgs& g = a.pg;
  const int64_t id = linear_block();
  const int b = (int)(id / blocks);
  if (b >= g.B) return;
  const SeqTokens t = seq_tokens(g, b);
  if (t.nn == 0) return;
  const int n_part = p.pieces * g.H;
  for (int64_t j = (id % blocks) * 256 + threadIdx.x; j < t.n; j += (int64_t)blocks * 256) {
    if (j >= w.ld_s) {
      raise_flag(g.status, b);
      return;
    }
    float sum = 0.f;
    for (int i = 0; i < n_part; ++i) {
      const int piece = i / g.H, h = i - piece * g.H;
      sum += p.part[(((int64_t)piece * g.B + b) * g.H + h) * p.ld + j];
    }
    write_sum(w, b, (int)j, t, sum);
  }
}

constexpr int kMaxTiles = 16384;  // slot tiles of all sequences, about; a workgroup goes on to further ones

WeighPlan weigh_plan(int B, int H, int G, int d, int slots, int watch) {
  WeighPlan p;
  const int kSlots = slots_of_group(d);
  const int64_t cus = std::max(1, device_cus());
  const int tiles = (slots + kSlots - 1) / kSlots;
  p.slot_tiles = std::min(tiles, std::max(1, kMaxTiles / B));
  p.tokens = G <= kRows ? kRows / G : 1;
  p.head_tiles = (G + kRows - 1) / kRows;
  const int64_t row_tiles = (int64_t)((watch + p.tokens - 1) / p.tokens) * p.head_tiles;
  const int64_t blocks = (int64_t)B * H * p.slot_tiles;
  p.pieces = (int)std::max<int64_t>(
      1, std::min<int64_t>(std::min<int64_t>(kMaxPieces, row_tiles / 8), 8 * cus / blocks));
  p.ld = (int64_t)tiles * kSlots;
  p.part = nullptr;
  return p;
}

template <int D>
void launch_tiles(const AttendArgs& a, const WeighArgs& w, const WeighPlan& p, bool q4, hipStream_t s) {
  const dim3 grid = linear_grid((int64_t)a.pg.B * a.pg.H * p.pieces * p.slot_tiles, 64 * kWaves);
  if (q4)
    hipLaunchKernelGGL((k_weigh_tile<D, true>), grid, dim3(64 * kWaves), 0, s, a, w, p);
  else
    hipLaunchKernelGGL((k_weigh_tile<D, false>), grid, dim3(64 * kWaves), 0, s, a, w, p);
}

}  // namespace

size_t weigh_tile_workspace(int B, int H, int G, int d, int slots, int watch) {
  const WeighPlan p = weigh_plan(B, H, G, d, slots, watch);
  return (size_t)p.pieces * B * H * p.ld * sizeof(float);
}

hipError_t launch_weigh_tile(const AttendArgs& a, const WeighArgs& w, bool q4, void* ws, hipStream_t s) {
  WeighPlan p = weigh_plan(a.pg.B, a.pg.H, a.G, a.pg.d, a.pg.max_tokens, w.watch);
  p.part = (float*)ws;
  if (a.pg.d == 64)
    launch_tiles<64>(a, w, p, q4, s);
  else if (a.pg.d == 128)
    launch_tiles<128>(a, w, p, q4, s);
  else
    launch_tiles<256>(a, w, p, q4, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = std::min((a.pg.max_tokens + 255) / 256, std::max(1, kMaxTiles / a.pg.B));
  hipLaunchKernelGGL(k_weigh_reduce, linear_grid((int64_t)a.pg.B * blocks, 256), dim3(256), 0, s, a, w, p, blocks);
  return hipGetLastError();
}

}  // namespace epikv
