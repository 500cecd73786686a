// The sums of many query rows' weights per slot (prefill, long chunks), after
// the attention itself.
//
// A row's weights need its maximum and sum, known when the attention ends, so
// the scores are made a second time: a wavefront keeps 64 keys (32 of 256
// channels) of a KV head in registers, as the first operand of v_mfma 32x32x16,
// and the query rows stream past through LDS, 64 at a time and two tiles deep.
// S^T = K Q^T, in the attention's order of channels (the same scores, bit for
// bit): lane (n, g) = (lane % 32, lane / 32) has query row n's scores of keys
// 8i + 4g + 0..3, so a row's norm is two registers a lane, and a key's sum stays
// in one register a lane from the first row to the last.  Only then do lanes meet.
//
// Bound by its instructions at the clock that they leave: an exponential, two
// multiply-adds and their share of the matrix instructions a score.
// 4096 tokens of 32 heads of 128 over 16k slots 493-510 us, 0.94-0.97 PFLOP/s at
// 2.0 GHz, matrix cores busy 45 % of the time and vector units 67 %; 8 chunks of
// 128 over 32k slots in 4 bits 345-363 us, 34 % and 62 %.  (15 % fewer clocks, with
// a third wavefront to a SIMD, were 8 % of the time: the clock fell by 7 %.)
#include "attend_impl.h"

namespace epikv {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef uint16_t uint16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
// Blocks of 32 keys that a wavefront holds (two of 256 channels spill).
constexpr int key_blocks(int d) { return d == 256 ? 1 : 2; }
constexpr int slots_of_group(int d) { return kWaves * 32 * key_blocks(d); }
constexpr int kRows = 64;                  // query rows of a tile, at most
constexpr int kMaxPieces = 64;

// How the work is dealt out: the slots of every (sequence, KV head) in tiles,
// each tile's rows in `pieces`.
struct WeighPlan {
  int32_t slot_tiles, pieces;
  int32_t tokens;        // of a tile of rows: whole tokens where 64 rows hold a token's
  int32_t head_tiles;    // tiles of a token, where they do not
  uint32_t per_inverse;  // of the rows of a token in a tile: 2^16 / per, rounded up (row / per is exact below 64)
  int32_t near;          // a tile's queries lie within 2^31 bytes
  int64_t ld;            // of a row of partial sums
  float* part;           // [pieces][B][H][ld]
};

// Two values' sums over pairs of lanes that a move exchanges: of the first on
// the lanes below, of the second on those above (`up`).
template <int MOVE>
__device__ __forceinline__ float fold(float a, float b, bool up) {
  return (up ? b : a) + dpp_move<MOVE>(up ? a : b);
}

// Sums over the 32 lanes of a half: lane n gets that of value n % K.  Each step
// halves the lanes of a sum and the values of a lane.
template <int K>
__device__ __forceinline__ float half_sums(const float (&v)[K], int n) {
  float x[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k + (K - 16)]), false, false);
    x[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = fold<0x128>(x[k], x[k + 8], n & 8);  // row_ror:8
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = fold<0x141>(x[k], x[k + 4], n & 4);  // row_half_mirror (lane ^ 7)
#pragma unroll
  for (int k = 0; k < 2; ++k) x[k] = fold<0x4E>(x[k], x[k + 2], n & 2);   // quad_perm [2,3,0,1]
  return fold<0xB1>(x[0], x[1], n & 1);                                   // quad_perm [1,0,3,2]
}

// The same number, what is made of it to be made anew (kept from tile to tile it
// takes the registers of a third wavefront).
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <int D, bool Q4>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 2 : D == 64 ? 4 : 3) void k_weigh_tile(AttendArgs a, WeighArgs w,
                                                                                            WeighPlan p) {
  constexpr int NB = key_blocks(D), kKeys = 32 * NB, kSlots = slots_of_group(D);
  constexpr uint64_t kAllKeys = NB == 2 ? ~0ull : 0xffffffffull;
  constexpr int KS = D / 16;            // instructions of a product
  constexpr int RC = D / 8;             // 16-byte chunks of a row
  constexpr int RPI = 1024 / (D * 2);   // rows a load of a wavefront
  constexpr int NI = kRows / kWaves / RPI;
  __shared__ __align__(1024) char s_q[2][kRows * D * 2];
  __shared__ float s_neg[2][kRows];  // minus a row's maximum (minus infinity: no such row)
  __shared__ float s_inv[2][kRows];  // 1 / its sum
  constexpr float kNotCounted = -kNegInf;
  __shared__ int s_lim[2][kRows];    // the slots that it sees
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

    // A tile's rows: tokens from c on, heads of the group from g on.
    struct Rows {
      int c, g;
    };
    auto rows_of = [&](int t) {
      const int c = t / p.head_tiles;
      return Rows{c_lo + c * p.tokens, (t - c * p.head_tiles) * kRows};
    };
    auto after = [&](Rows x) {
      x.g += kRows;
      return x.g < a.G ? x : Rows{x.c + p.tokens, 0};
    };
    const int per = min(a.G, kRows);  // rows of a token in a tile
    auto token_of = [&](int row) { return (int)(((uint32_t)row * p.per_inverse) >> 16); };
    // Whether every row of a tile is there, and whether a row (of token c and head
    // gr of the tile) is.
    auto whole = [&](Rows x) {
      return p.tokens * per == kRows && c_hi - x.c >= p.tokens && a.G - x.g >= per;
    };
    auto has_row = [&](Rows x, int c, int gr) { return c < min(p.tokens, c_hi - x.c) && x.g + gr < a.G; };
    // (where the lane's rows are from the tile's first one on; near where 31 bits
    // hold that, which saves registers)
    int q_off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = wave * (kRows / kWaves) + i * RPI + lane / RC;
      const int c = token_of(row);
      q_off[i] = (int)((c * a.q.ld_tok + (row - c * per) * a.q.ld_head) * 2) + row_chunk<D>(row, lane % RC) * 16;
    }
    // A tile's rows, straight to LDS; the first, which always is there, for one that
    // is not.
    auto fetch = [&](Rows x, int buf) {
      const char* base = a.q.base + (b * a.q.ld_seq + x.c * a.q.ld_tok + (h * a.G + x.g) * a.q.ld_head) * 2;
      char* to = s_q[buf] + wave * (kRows / kWaves) * D * 2;
      auto load = [&](const char* from, int i) {
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) uint32_t*)(uintptr_t)from,
            (__attribute__((address_space(3))) uint32_t*)(uint32_t)(uintptr_t)(lds_char*)(to + i * 1024), 16, 0, 0);
      };
      if (p.near && whole(x)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) load(base + (uint32_t)anew(q_off[i]), i);
      } else {
        const int l = anew(lane);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int row = wave * (kRows / kWaves) + i * RPI + l / RC, c = token_of(row), gr = row - c * per;
          int64_t off = row_chunk<D>(row, l % RC) * 16;
          if (has_row(x, c, gr)) off += (c * a.q.ld_tok + gr * a.q.ld_head) * 2;
          load(base + off, i);
        }
      }
    };
    auto tile_sync = [&] {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    // The rows' norms, some of a tile by every wavefront: loaded two tiles ahead,
    // put to LDS one ahead (and nothing is done with them before, or every tile
    // waits for its load).
    constexpr int RW = kRows / kWaves;
    auto load_norm = [&](Rows x) {
      const int my_row = wave * RW + (anew(lane) & (RW - 1)), my_c = token_of(my_row), my_g = my_row - my_c * per;
      const float2* base = a.norms + ((int64_t)b * a.heads + h * a.G + x.g) * g.C + x.c;
      return base[has_row(x, my_c, my_g) ? my_g * g.C + my_c : 0];
    };
    auto put_norm = [&](Rows x, int buf, float2 norm) {
      const int l = anew(lane);
      if (l < RW) {
        const int my_row = wave * RW + l, my_c = token_of(my_row), my_g = my_row - my_c * per;
        const bool there = has_row(x, my_c, my_g);
        const bool counts = there && norm.y != 0.f;
        s_neg[buf][my_row] = counts ? -norm.x : there ? kNotCounted : kNegInf;
        s_inv[buf][my_row] = counts ? norm.y : 0.f;
        s_lim[buf][my_row] = counts ? old + x.c + my_c + 1 : 0;
      }
    };

    // (the first rows are on their way while the keys' places are looked up)
    Rows now = rows_of(t0);
    float2 norm = {0.f, 0.f};
    if (t0 < t1) {
      fetch(now, 0);
      norm = load_norm(now);
    }
    bf16x8 kf[NB][KS];
    uint64_t ok = 0;  // which of the wavefront's keys exist
    uint16x2 top = {0, 0};  // of the magnitudes' bits, or of the blocks' scales
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int l = anew(lane), gh = l >> 5, j = kw + 32 * i + (l & 31);
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
          top[0] = max(top[0], byte);
        } else {
          x = *reinterpret_cast<const u32x4*>(row + (h * D + ch) * 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(uint16x2, x[e] & 0x7fff7fffu));
        }
        if (off < 0) x = u32x4{0, 0, 0, 0};
        kf[i][s] = as_bf16x8(x);
      }
    }
    // 0 times one of its channels may be NaN.  (6 * 2^(252 - 127) is finite still,
    // and past it blocks may be; a key that is not there may be one, too.)
    const bool odd_key = __any(max(top[0], top[1]) >= (Q4 ? 253 : 0x7f80));

    float sum[NB][16];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[i][e] = 0.f;
    const uint32_t q_base = (uint32_t)(uintptr_t)(lds_char*)&s_q[0][0] + n * D * 2 + row_chunk<D>(n, gh) * 16;

    // The weights of 32 rows to the sums: the scores, and then 2^(scale * x + plus) / sum
    // of each; the other wavefronts' matrix instructions run beside a wavefront's
    // exponentials.  (Two wavefronts of a SIMD that each mix theirs, twice the
    // scores in registers: 1466 us for the chunk of 4096 over 16k slots, attention
    // and all, 1426 so.)
    auto rows32 = [&](uint32_t at, int buf, int r, bool all, auto meanwhile) {
      constexpr int AHEAD = 2;  // steps that operands are read ahead
      auto read = [&](int k) { return as_bf16x8(*(const lds_u32x4*)(uintptr_t)(at ^ (32 * k))); };
      bf16x8 q[KS];
      f32x16 s[NB];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) q[k] = read(k);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if (k + AHEAD < KS) q[k + AHEAD] = read(k + AHEAD);
#pragma unroll
        for (int i = 0; i < NB; ++i)
          s[i] = mfma32(kf[i][k], q[k], k ? s[i] : f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
        __builtin_amdgcn_sched_barrier(0);
      }
      const float neg = s_neg[buf][32 * r + n], first_neg = s_neg[buf][0], inv = s_inv[buf][32 * r + n];
      const int lim = s_lim[buf][32 * r + n];
      __builtin_amdgcn_sched_barrier(0);
      meanwhile();
      // Hidden keys, rows that do not count (and, with a key or a first row that is
      // not finite, rows that are not there): the exponents here, one by one.
      float scale = a.scale2, plus = neg;
      const bool odd = !all || __any(neg == kNotCounted || (neg == kNegInf && (odd_key || first_neg == kNotCounted)));
      if (__builtin_amdgcn_readfirstlane((int)odd)) {  // (one branch for the wavefront)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const uint32_t mine = ((uint32_t)(ok >> (32 * i)) & below(lim - kw - 32 * i)) >> (4 * (anew(lane) >> 5));
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = fmaf(s[i][e], a.scale2, neg);
            s[i][e] = mine >> (8 * (e / 4) + e % 4) & 1u ? y : kNegInf;
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        scale = 1.f;
        plus = 0.f;
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[i][e] = fmaf(exp2_fast(fmaf(s[i][e], scale, plus)), inv, sum[i][e]);
#pragma unroll
      for (int u = 0; u < 16 * NB; ++u) asm volatile("" : "+v"(sum[u / 16][u % 16]));
    };

    if (t0 < t1) {
      put_norm(now, 0, norm);
      Rows next = t0 + 1 < t1 ? after(now) : now;
      norm = load_norm(next);
      tile_sync();
      int buf = 0;
      for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) put_norm(next, buf ^ 1, norm);
        const Rows then = t + 2 < t1 ? after(next) : next;
        const bool all = ok == kAllKeys && old + now.c + 1 >= kw + kKeys;  // every row sees every key
        const uint32_t at = q_base + buf * (kRows * D * 2);
        rows32(at, buf, 0, all, [] {});
        rows32(at + 64 * D, buf, 1, all, [&] {
          // (when this tile's rows have been read: a read waits for whatever is on its way to LDS)
          if (t + 1 < t1) fetch(next, buf ^ 1);
          norm = load_norm(then);
        });
        buf ^= 1;
        now = next;
        next = then;
        tile_sync();
      }
    }

    // Over the 32 rows' lanes: value 16 i + e, of key 8(e/4) + 4gh + e%4 of block
    // i, to lane n.
    float all[16 * NB];
#pragma unroll
    for (int u = 0; u < 16 * NB; ++u) all[u] = sum[u / 16][u % 16];
    const int l = anew(lane), n = l & 31, gh = l >> 5;
    const float mine = half_sums(all, n);
    float* out = p.part + (((int64_t)piece * g.B + b) * g.H + h) * p.ld + kw;
    if (n < 16 * NB) out[32 * (n / 16) + 8 * (n % 16 / 4) + 4 * gh + n % 4] = mine;
  }
}

// The partial sums of a slot, in a fixed order, on what is kept of the old one:
// four slots a lane, a workgroup's wavefronts taking turns over the partial sums,
// four on their way at a time.  Bound by latency (16384 slots of 32 partial sums
// 13 us with a thread for a slot's).
__global__ __launch_bounds__(256) void k_weigh_reduce(AttendArgs a, WeighArgs w, WeighPlan p, int blocks) {
  constexpr int SLOTS = 256, AHEAD = 4;
  __shared__ f32x4 s_sum[4][SLOTS / 4];
  const PagedArgs& g = a.pg;
  const int64_t id = linear_block();
  const int b = (int)(id / blocks);
  if (b >= g.B) return;
  const SeqTokens t = seq_tokens(g, b);
  if (t.nn == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n_part = p.pieces * g.H;
  for (int64_t j0 = (id % blocks) * SLOTS; j0 < t.n; j0 += (int64_t)blocks * SLOTS) {
    const int64_t j = j0 + threadIdx.x;
    const float old_sum = j < t.n && j < w.ld_s ? kept_sum(w, b, j, t) : 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (j0 + 4 * lane < p.ld) {
      const float* part = p.part + (int64_t)b * g.H * p.ld + j0 + 4 * lane;
      for (int i = wave; i < n_part; i += 4 * AHEAD) {
        f32x4 x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int k = i + 4 * u, piece = k / g.H;
          x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (k < n_part)
            x[u] = *reinterpret_cast<const f32x4*>(part + ((int64_t)piece * g.B * g.H + (k - piece * g.H)) * p.ld);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) sum += x[u];
      }
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (j < t.n) {
      const int v = threadIdx.x / 4, e = threadIdx.x % 4;
      if (j < w.ld_s)
        write_sum(w, b, j, old_sum, (s_sum[0][v][e] + s_sum[1][v][e]) + (s_sum[2][v][e] + s_sum[3][v][e]));
      else
        raise_flag(g.status, b);
    }
    __syncthreads();
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
  // Pieces: of two tiles at least while they give every compute unit its two
  // workgroups, of eight where there are more (what a workgroup takes to begin and
  // to end is worth about two).  512 tokens alone 51.5 us so, 59.9 without pieces
  // of two; 2048 alone 105 so, 118 with pieces of two throughout.
  const auto pieces = [&](int64_t least, int64_t most) { return std::min(row_tiles / least, most / blocks); };
  p.pieces = (int)std::max<int64_t>(
      1, std::min<int64_t>(kMaxPieces, std::max(pieces(2, 2 * cus), pieces(8, 8 * cus))));
  p.ld = (int64_t)tiles * kSlots;
  const int per = std::min(G, kRows);
  p.per_inverse = (uint32_t)((65536 + per - 1) / per);
  p.near = 0;
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
  p.near = ((p.tokens - 1) * a.q.ld_tok + (std::min(a.G, kRows) - 1) * a.q.ld_head + a.pg.d) * 2 < INT32_MAX;
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
