// Attention for many query rows per KV head (prefill, long chunks): a
// workgroup takes 256 rows of one KV head (128 when there are no more, or rows
// of 256 channels), 32 to a wavefront, and walks the slots in tiles of 64 whose
// key and value rows pass through LDS as bf16, the next tile on its way while
// one is worked on.
//
// As with few rows, S^T = K Q^T and O^T = V^T P^T, here with v_mfma 32x32x16:
// lane (n, g) = (lane % 32, lane / 32) holds query row n, and of each 16
// tokens the 8 numbered 4g .. 4g+3 and 8 + 4g .. 8 + 4g+3, in the first
// product's result as in the second's operand.  V^T comes out of LDS by
// transposing reads of 4 tokens x 16 channels.
//
// Bound by the matrix cores and the softmax's arithmetic together (32 scores
// a lane and tile: 32 exponentials beside 32 matrix instructions).  A chunk of
// 4096 tokens over 16k slots (32 query heads of 128) 890-930 us by machine, 1.03-1.08
// PFLOP/s; 8 chunks of 128 over 32k in 4 bits 560-580 us, 0.94-0.98.
#include <type_traits>

#include "attend_impl.h"

namespace epikv {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <int D>
struct Tile {
  static constexpr int KT = D == 256 ? 32 : 64;  // tokens
  static constexpr int RC = D / 8;               // 16-byte chunks of a row
  static constexpr int BYTES = KT * D * 2;
  // Chunks change places within a row so that the lanes that read together
  // hit different banks: keys are read at one chunk of 16 rows, values at
  // four chunks (a 64-byte run) of 4 rows (and the change within a run keeps
  // the writes of decoded rows apart).  The change is an exclusive or of
  // the chunk's number, so a fragment's address is a lane's base address,
  // exclusive or the fragment's offset in the row, plus its rows' offset.
  __device__ static int key_chunk(int row, int c) { return row_chunk<D>(row, c); }
  __device__ static int value_chunk(int row, int c) {
    return c ^ (D == 64 ? (row >> 1) & 1 : row & 3) * 5;
  }
};

// How the rows are dealt out: row tiles of every (sequence, KV head), each
// walked whole or in `splits` even pieces (partial slots [splits][B]).
struct TilePlan {
  int32_t row_tiles, splits, waves, paired;
  float* part_o;    // [splits][B][H][R][d]
  float2* part_ml;  // [splits][B][H][R]
};

template <int D, bool Q4, int W>
__global__ __launch_bounds__(64 * W, D == 256 ? 1 : 2) void k_attend_tile(AttendArgs a, TilePlan p) {
  using T = Tile<D>;
  constexpr int kRows = 32 * W;
  constexpr int KT = T::KT, KS = D / 16, CT = D / 32, TB = KT / 32, PS = KT / 16;
  __shared__ __align__(1024) char s_kv[2][2][T::BYTES];  // [buffer][K, V]
  const PagedArgs& g = a.pg;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n = lane & 31, gh = lane >> 5;

  // Heads first: workgroups side by side in the launch go to different XCDs,
  // so that those of one head share an XCD's cache.  The last, longest rows of
  // a chunk start first; when all rows are under way at once (`paired`), the
  // second half comes shortest first, so that a compute unit's two workgroups
  // have as much to do as any other's.
  int64_t id = linear_block();
  const int h = (int)(id % g.H);
  id /= g.H;
  const int k = (int)(id % p.row_tiles);
  const int rt = p.paired && 2 * k >= p.row_tiles ? k - (p.row_tiles + 1) / 2 : p.row_tiles - 1 - k;
  id /= p.row_tiles;
  const int piece = (int)(id % p.splits);
  const int64_t bb = id / p.splits;
  if (bb >= g.B) return;
  const int b = (int)bb;
  const SeqTokens tk = seq_tokens(g, b);
  if (tk.bad && threadIdx.x == 0) raise_flag(g.status, b);
  const int rows = tk.nn * a.G;
  const int r0 = rt * kRows, w0 = r0 + 32 * wave;
  const int r = w0 + n;
  const int c = r / a.G, hq = h * a.G + (r - c * a.G);
  const bool real = r < rows;
  const int old = tk.n - tk.nn;  // slots before the new tokens
  const int lim = real ? old + c + 1 : 0;
  // slots seen by any row of the workgroup and of the wavefront, by all of the former
  const int end_wg = r0 < rows ? old + (min(r0 + kRows, rows) - 1) / a.G + 1 : 0;
  const int end_w = w0 < rows ? old + (min(w0 + 32, rows) - 1) / a.G + 1 : 0;
  const int all_wg = old + r0 / a.G + 1;
  const int tiles = (end_wg + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * piece / p.splits);
  const int t1 = (int)((int64_t)tiles * (piece + 1) / p.splits);

  bf16x8 qf[KS];
  {
    const char* qp = a.q.base + (b * a.q.ld_seq + c * a.q.ld_tok + hq * a.q.ld_head) * 2;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 w = {0, 0, 0, 0};
      if (real) w = *reinterpret_cast<const u32x4*>(qp + (16 * s + 8 * gh) * 2);
      qf[s] = as_bf16x8(w);
    }
  }
  f32x16 o[CT];
#pragma unroll
  for (int j = 0; j < CT; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
  float top = kNegInf, sum = 0.f;

  // The page table 64 entries at a time, the next 64 on their way; tokens past
  // the end stand for the last one.
  const int32_t* pt = g.pt + (int64_t)b * g.ld_pt;
  auto page_index = [&](int tok) {
    return g.page_shift >= 0 ? tok >> g.page_shift : (int)((uint32_t)tok / (uint32_t)g.page_size);
  };
  const int last_page = page_index(max(end_wg - 1, 0));
  auto load_pages = [&](int first) { return pt[min(first + lane, last_page)]; };
  int page0 = page_index(t0 * KT), pages = 0, pages_next = 0;
  bool any_bad = false;
  int64_t my_off = 0;  // the row of this lane's token of the tile to be loaded
  auto offsets = [&](int t) -> uint64_t {
    const int tok = t * KT + (lane & (KT - 1));
    const int at = min(tok, end_wg - 1), pi = page_index(at);
    if (page_index(min(t * KT, end_wg - 1)) - page0 >= 64) {
      page0 += 64;
      pages = pages_next;
      pages_next = load_pages(page0 + 64);
    }
    const int rel = pi - page0;
    int pg = __shfl(pages, rel & 63);
    if (__any(rel >= 64)) {
      const int beyond = __shfl(pages_next, rel & 63);
      pg = rel < 64 ? pg : beyond;
    }
    const bool good = pg >= 0 && pg < g.n_pages;
    my_off = good ? (int64_t)pg * g.s_page + (int64_t)(at - pi * g.page_size) * g.row_bytes : 0;
    any_bad |= !good;
    return __ballot(good && tok < end_wg);
  };
  auto offset_of = [&](int row) -> int64_t {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)my_off, row);
    const int hi = __shfl((int)(my_off >> 32), row);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | lo);
  };

  // bf16 rows go to LDS directly, 1 KiB an instruction.
  auto stage = [&](int buf) {
    constexpr int RPI = 1024 / (D * 2);           // rows an instruction
    constexpr int NI = KT / W / RPI;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int first = wave * (KT / W) + i * RPI;
      const int row = first + lane / T::RC, cpos = lane % T::RC;
      const int64_t off = offset_of(row) + h * (D * 2);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) uint32_t*)(g.plane[0] + off + T::key_chunk(row, cpos) * 16),
          (__attribute__((address_space(3))) uint32_t*)(s_kv[buf][0] + first * D * 2), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) uint32_t*)(g.plane[1] + off + T::value_chunk(row, cpos) * 16),
          (__attribute__((address_space(3))) uint32_t*)(s_kv[buf][1] + first * D * 2), 16, 0, 0);
    }
  };
  // 4-bit rows pass through registers: a thread decodes CH channels of one token.
  constexpr int TPT = 64 * W / KT, CH = D / TPT;
  const int q_row = threadIdx.x / TPT, q_part = threadIdx.x % TPT;
  uint32_t raw[2][CH / 8];
  uint32_t raw_s[2] = {0, 0};
  auto fetch = [&] {
    const int64_t off = offset_of(q_row);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const char* row = g.plane[kv] + off;
      const char* x = row + h * (D / 2) + q_part * (CH / 2);
      if constexpr (CH == 8) {
        raw[kv][0] = *reinterpret_cast<const uint32_t*>(x);
      } else if constexpr (CH == 16) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(x);
        raw[kv][0] = w[0];
        raw[kv][1] = w[1];
      } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[kv][i] = w[i];
      }
      raw_s[kv] = reinterpret_cast<const uint8_t*>(row)[g.H * (D / 2) + h * (D / 32) + q_part * CH / 32];
    }
  };
  auto decode = [&](int buf) {
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const float s = block_scale(raw_s[kv]);
      char* row = s_kv[buf][kv] + q_row * D * 2;
#pragma unroll
      for (int i = 0; i < CH / 8; ++i) {
        const int chunk = q_part * (CH / 8) + i;
        const int at = kv ? T::value_chunk(q_row, chunk) : T::key_chunk(q_row, chunk);
        *reinterpret_cast<u32x4*>(row + at * 16) = decode8(raw[kv][i], s);
      }
    }
  };
  auto arrived = [&] {  // this wavefront's part of the next tile is in LDS; then everybody's
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  const uint32_t lds = (uint32_t)(uintptr_t)(lds_char*)&s_kv[0][0][0];
  const uint32_t k_base = lds + n * D * 2 + T::key_chunk(n, gh) * 16;
  const int v_row = 4 * gh + ((lane & 15) >> 2);
  const int v_chan = 16 * ((lane >> 4) & 1) + (lane & 3) * 4;
  const uint32_t v_base = lds + T::BYTES + v_row * D * 2 + T::value_chunk(v_row, v_chan >> 3) * 16 +
                          (v_chan & 7) * 2;
  // K of tokens 32i .. and channels 16k ..
  auto key_frag = [&](uint32_t at, int i, int k) {
    return as_bf16x8(*(const lds_u32x4*)(uintptr_t)((at ^ (32 * k)) + i * 64 * D));
  };
  // V^T of channels 32j .. and tokens 16s ..: two transposing reads.
  auto value_frag = [&](uint32_t at, int j, int s) -> u32x4 {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2 x = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                     (lds_s16x4*)(uintptr_t)((at ^ (64 * j)) + (16 * s + 8 * i) * D * 2)));
      w[2 * i] = x[0];
      w[2 * i + 1] = x[1];
    }
    return w;
  };

  // A tile; MASKED: some of its tokens are hidden from some rows or do not exist.
  auto work = [&](auto masked, int t, int buf, uint64_t ok) {
    constexpr bool MASKED = decltype(masked)::value;
    const uint32_t kt = k_base + buf * 2 * T::BYTES;
    const uint32_t vt = v_base + buf * 2 * T::BYTES;
    const int base = t * KT;
    f32x16 s[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
    // (in an order in which neighbours do not add to the same result)
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < TB; ++i) s[i] = mfma32(key_frag(kt, i, k), qf[k], s[i]);
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        const uint32_t seen = (uint32_t)(ok >> (32 * i)) & below(lim - base - 32 * i);
        const uint32_t mine = seen >> (4 * gh);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[i][e] = mine >> (8 * (e / 4) + e % 4) & 1u ? s[i][e] : kNegInf;
      }
    }
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, s[i][e]);
    m *= a.scale2;
    if (__any(m > top + 8.f)) {  // (the maximum may lag by 2^8)
      m = fmaxf(m, __shfl_xor(m, 32));
      const float grown = fmaxf(top, m);
      const float f = grown == top ? 1.f : exp2_fast(top - grown);
      top = grown;
      sum *= f;
#pragma unroll
      for (int j = 0; j < CT; ++j) o[j] *= f;
    }
    const float base2 = top == kNegInf ? 0.f : top;
    bf16x8 pf[PS];
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = exp2_fast(fmaf(s[i][8 * u + e], a.scale2, -base2));
          sum += w[e];
        }
        // (bf16 weights as with few rows; a second product with what the
        // rounding leaves took 886 -> 1206 us, 564 -> 734)
        pf[2 * i + u] = as_bf16x8(u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]),
                                        pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])});
      }
    if constexpr (!MASKED) {
#pragma unroll
      for (int k = 0; k < PS; ++k)
#pragma unroll
        for (int j = 0; j < CT; ++j) o[j] = mfma32(as_bf16x8(value_frag(vt, j, k)), pf[k], o[j]);
      return;
    }
    // What does not exist counts as 0, whatever its bytes are.  A NaN or an
    // infinity that some rows see and others do not (0 times it is NaN) needs
    // a pass for each token, without the values hidden from it.
    auto masks = [&](int k, int seen) {
      const uint32_t mine =
          ((uint32_t)(ok >> (32 * (k / 2))) & below(seen - base - 32 * (k / 2))) >> (16 * (k % 2) + 4 * gh);
      u32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 8 * (i / 2) + 2 * (i % 2);
        x[i] = (mine >> j & 1u ? 0xffffu : 0u) | (mine >> (j + 1) & 1u ? 0xffff0000u : 0u);
      }
      return x;
    };
    bool odd = false;
    if (tk.nn > 1) {
      for (int k = 0; k < PS; ++k) {
        const u32x4 x = masks(k, tk.n);
        for (int j = 0; j < CT; ++j) {
          const u32x4 w = value_frag(vt, j, k) & x;
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= word_not_finite(w[i]);
        }
      }
    }
    const bool by_token = __any(odd);
    const int c_last = (min(w0 + 32, rows) - 1) / a.G;
    for (int cc = by_token ? w0 / a.G : c_last; cc <= c_last; ++cc) {
      const int seen = old + cc + 1;
      const bool mine = !by_token || lim == seen;
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        f32x16 y = o[j];
#pragma unroll
        for (int k = 0; k < PS; ++k) y = mfma32(as_bf16x8(value_frag(vt, j, k) & masks(k, seen)), pf[k], y);
#pragma unroll
        for (int e = 0; e < 16; ++e) o[j][e] = mine ? y[e] : o[j][e];
      }
    }
  };

  if (t0 < t1) {
    pages = load_pages(page0);
    pages_next = load_pages(page0 + 64);
    uint64_t ok = offsets(t0);
    if constexpr (Q4) {
      fetch();
      decode(0);
    } else {
      stage(0);
    }
    arrived();
    int t = t0, buf = 0;
    auto turn = [&](auto masked) {
      uint64_t ok_next = 0;
      if (t + 1 < t1) {
        ok_next = offsets(t + 1);
        if constexpr (Q4)
          fetch();
        else
          stage(buf ^ 1);
      }
      if (t * KT < end_w) work(masked, t, buf, ok);
      if constexpr (Q4) {
        if (t + 1 < t1) decode(buf ^ 1);
      }
      ok = ok_next;
      ++t;
      buf ^= 1;
      arrived();
    };
    // The tiles that every row sees whole, then (from the first that is not
    // so) the others: both conditions are the workgroup's.
    constexpr uint64_t FULL = KT == 64 ? ~0ull : 0xffffffffull;
    while (t < t1 && (t + 1) * KT <= all_wg && (ok & FULL) == FULL) turn(std::false_type{});
    while (t < t1) turn(std::true_type{});
    if (__any(any_bad) && threadIdx.x == 0) raise_flag(g.status, b);
  }

  sum += __shfl_xor(sum, 32);
  if (r >= a.R) return;
  // (lane (n, gh) holds channels 32j + 8i + 4gh + 0..3 of row r)
  if (p.splits == 1) {
    const bool some = real && sum != 0.f;
    const float inv = 1.f / sum;
    char* op = a.out.base + (b * a.out.ld_seq + c * a.out.ld_tok + hq * a.out.ld_head + 4 * gh) * 2;
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x2 w = {0u, 0u};
        if (some) {
          w[0] = pack_bf16(o[j][4 * i] * inv, o[j][4 * i + 1] * inv);
          w[1] = pack_bf16(o[j][4 * i + 2] * inv, o[j][4 * i + 3] * inv);
        }
        *reinterpret_cast<u32x2*>(op + (32 * j + 8 * i) * 2) = w;
      }
    if (gh == 0) write_log_sum<true>(a, b, hq, c, top, sum, some);
  } else if (real) {
    const int64_t at = (((int64_t)piece * g.B + b) * g.H + h) * a.R + r;
    if (gh == 0) p.part_ml[at] = make_float2(top, sum);
    if (t0 < t1) {  // (an empty piece has weight 0 and is not read)
      float* po = p.part_o + at * D + 4 * gh;
#pragma unroll
      for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(po + 32 * j + 8 * i) =
              f32x4{o[j][4 * i], o[j][4 * i + 1], o[j][4 * i + 2], o[j][4 * i + 3]};
    }
  }
}

// Joins the pieces of a row: four channels a lane, so that a wavefront has
// several rows' loads on their way.  Bound by HBM's latency: 32768 rows of 128
// channels in two pieces 10.9 us, 3.9 TB/s (a wavefront per row, 17.2).
template <int D>
__global__ __launch_bounds__(256) void k_attend_tile_join(AttendArgs a, TilePlan p) {
  constexpr int LANES = D / 4, AHEAD = 4;
  const PagedArgs& g = a.pg;
  const int x = threadIdx.x % LANES;
  // (32 bits: 2^32 rows of output are more than the memory)
  const uint32_t id = (uint32_t)linear_block() * (256 / LANES) + threadIdx.x / LANES;
  const uint32_t head_rows = id / (uint32_t)a.R, bb = head_rows / (uint32_t)g.H;
  if (bb >= (uint32_t)g.B) return;
  const int b = (int)bb, h = (int)(head_rows - bb * (uint32_t)g.H), r = (int)(id - head_rows * (uint32_t)a.R);
  const SeqTokens tk = seq_tokens(g, b);
  const int c = r / a.G, hq = h * a.G + (r - c * a.G);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float top = kNegInf, sum = 0.f;
  if (r < tk.nn * a.G) {
    const int64_t at = (((int64_t)b) * g.H + h) * a.R + r, step = (int64_t)g.B * g.H * a.R;
    for (int s = 0; s < p.splits; s += AHEAD) {
      float2 ml[AHEAD];
      f32x4 y[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        ml[k] = make_float2(kNegInf, 0.f);
        if (s + k < p.splits) {
          const int64_t from = at + (s + k) * step;
          ml[k] = p.part_ml[from];
          y[k] = *reinterpret_cast<const f32x4*>(p.part_o + from * D + 4 * x);
        }
      }
      float grown = top;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) grown = fmaxf(grown, ml[k].x);
      const float base2 = grown == kNegInf ? 0.f : grown;
      const float f = exp2_fast(top - base2);
      sum *= f;
      o *= f;
      top = grown;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        if (ml[k].x == kNegInf && ml[k].y == 0.f) continue;  // (nothing seen; a NaN sum stays)
        const float w = exp2_fast(ml[k].x - base2);
        sum += w * ml[k].y;
        o += w * y[k];
      }
    }
  }
  const bool some = sum != 0.f;
  const float inv = 1.f / sum;
  u32x2 w = {0u, 0u};
  if (some) w = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  *reinterpret_cast<u32x2*>(a.out.base + (b * a.out.ld_seq + c * a.out.ld_tok + hq * a.out.ld_head) * 2 + 8 * x) = w;
  if (x == 0) write_log_sum<true>(a, b, hq, c, top, sum, some);
}

// Pieces of a row tile at most.  How long the sequences are only the device
// knows: 8, 16, 32 pieces take 228, 126, 81 us for 17 tokens over 64k slots (8 KV
// heads), 58.0, 57.5, 56.0 for 200 over 8k, but 23.3, 20.0, 21.1 for 17 over 4000
// and 13.7, 13.9, 15.8 for 40 over 1000.
constexpr int kMaxSplits = 16;

// Wavefronts of a workgroup: eight halve what each of them does to bring a tile
// to LDS (a 4096-token chunk over 16k slots 1008 us with four, 914 with eight).
// Four where eight would leave one workgroup of uneven rows to each compute
// unit, in chunks of many row tiles (a prompt of 2048 tokens, 32 tiles, whose
// first rows see little and whose last see all: 76.7 us with eight, 71.9 with
// four, 67.5 with those in pairs; 1500 tokens after 1500, 24 tiles: 107.5,
// 103.6, 102.6; but 1000 alone, 16 tiles: 44.5, 49.4, 49.0, and 512 after 7680,
// 8 tiles: 98, 107, 110).
// Pieces: as many as give every compute unit eight wavefronts.
TilePlan tile_plan(int B, int H, int R, int d) {
  TilePlan p;
  const int64_t cus = std::max(1, device_cus());
  auto tiles = [&](int waves) { return (R + 32 * waves - 1) / (32 * waves); };
  p.waves = d <= 128 && R > 128 ? 8 : 4;
  if (p.waves == 8 && tiles(8) >= 24 && (int64_t)B * H * tiles(8) < 2 * cus) p.waves = 4;
  p.row_tiles = tiles(p.waves);
  const int64_t blocks = (int64_t)B * H * p.row_tiles;
  const int64_t want = cus * 8 / p.waves;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, want / blocks));
  // (rows of 256 channels have one workgroup to a unit, the next when it ends;
  // two sequences in pairs 45.0 us, as without, for 1000 tokens of 4 KV heads)
  p.paired = p.waves == 4 && d <= 128 && p.splits == 1 && B == 1 && blocks <= want;
  p.part_o = nullptr;
  p.part_ml = nullptr;
  return p;
}

size_t part_rows(const TilePlan& p, int B, int H, int R) { return (size_t)p.splits * B * H * R; }

size_t part_ml_bytes(const TilePlan& p, int B, int H, int R) {
  return (part_rows(p, B, H, R) * sizeof(float2) + 255) / 256 * 256;
}

template <int D, int W>
void launch_tile_waves(const AttendArgs& a, const TilePlan& p, bool q4, hipStream_t s) {
  const dim3 grid = linear_grid((int64_t)a.pg.B * a.pg.H * p.row_tiles * p.splits, 64 * W);
  if (q4)
    hipLaunchKernelGGL((k_attend_tile<D, true, W>), grid, dim3(64 * W), 0, s, a, p);
  else
    hipLaunchKernelGGL((k_attend_tile<D, false, W>), grid, dim3(64 * W), 0, s, a, p);
}

template <int D>
hipError_t launch_tile(const AttendArgs& a, const TilePlan& p, bool q4, hipStream_t s) {
  if constexpr (D <= 128) {
    if (p.waves == 8)
      launch_tile_waves<D, 8>(a, p, q4, s);
    else
      launch_tile_waves<D, 4>(a, p, q4, s);
  } else {
    launch_tile_waves<D, 4>(a, p, q4, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(k_attend_tile_join<D>,
                     linear_grid(((int64_t)a.pg.B * a.pg.H * a.R + 1024 / D - 1) / (1024 / D), 256), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace

size_t attend_tile_workspace(int B, int H, int R, int d) {
  const TilePlan p = tile_plan(B, H, R, d);
  if (p.splits == 1) return 0;
  return part_ml_bytes(p, B, H, R) + part_rows(p, B, H, R) * d * sizeof(float);
}

hipError_t launch_attend_tile(const AttendArgs& a, bool q4, void* ws, hipStream_t s) {
  TilePlan p = tile_plan(a.pg.B, a.pg.H, a.R, a.pg.d);
  if (p.splits > 1) {
    p.part_ml = (float2*)ws;
    p.part_o = (float*)((char*)ws + part_ml_bytes(p, a.pg.B, a.pg.H, a.R));
  }
  if (a.pg.d == 64) return launch_tile<64>(a, p, q4, s);
  if (a.pg.d == 128) return launch_tile<128>(a, p, q4, s);
  return launch_tile<256>(a, p, q4, s);
}

}  // namespace epikv
