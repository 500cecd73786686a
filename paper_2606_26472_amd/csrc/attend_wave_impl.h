// Attention for few query rows per KV head (single tokens, short chunks): a
// wavefront per (KV head, share of a sequence), which walks the rows once,
// straight from memory into matrix-core operands.
//
// Scores are made transposed, S^T = K Q^T, so that a step's weights are
// already laid out as the second operand of O^T = V^T P^T: with v_mfma
// 16x16x32, lane (n, g) = (lane % 16, lane / 16) gets the scores of query row
// n against tokens 4g .. 4g+3 of each 16-token tile, and 32 tokens make its 8
// values of the second product.  Nothing passes through LDS but row addresses
// (and 4-bit values and scales), and the running maximum's growth is the only
// exchange between lanes.
//
// Bound by HBM: 32 sequences of 8k-32k tokens (8 KV heads of 128, 4 query heads
// each) 2.69 GB in 406 us, 6.6 TB/s; in 4 bits 0.72 GB in 138 us, 5.2 TB/s, with
// the vector units busy 45 % of the time.  One sequence of 4k: 8 us, latency.
//
// With KEEP the scores go to memory as well, for the sums of the weights that
// follow (attend_weigh.hip); nothing else changes, bit for bit.
#pragma once

#include "attend_impl.h"

namespace epikv {
namespace {

// What a lane holds of 32 tokens: of each of 8 of them, VC channels.
template <int D, bool Q4>
struct Values {
  static constexpr int VC = D / 16;  // instructions of the second product
  static constexpr int VW = Q4 ? (VC + 7) / 8 : VC / 2;
  uint32_t v[8][VW];
  uint32_t scale[Q4 ? 8 : 1];
};

// 32 tokens on their way from memory.  bf16 rows come as the products take
// them.  Of 4-bit rows a lane loads a quarter of a key and of a value of two
// tokens, and one token's scale bytes: five loads a step, where loads as the
// second product takes them would be 22 (with those the kernel ran at half
// its speed); values and scales then change lanes through LDS.
template <int D, bool Q4>
struct Step {
  static constexpr int KS = D / 32;  // first product: 32 channels an instruction
  uint32_t k[2][KS * 4];
  Values<D, false> val;
};
template <int D>
struct Step<D, true> {
  static constexpr int KS = D / 32;
  uint32_t k[2][KS], v[2][KS];
  uint32_t sc[D == 256 ? 2 : 1];
};

// A wavefront's part of LDS.
template <int D, bool Q4>
struct Scratch {
  int64_t off[kUnit];  // a step's row offsets
};
template <int D>
struct Scratch<D, true> {
  // bytes between tokens' codes: reads of 4 tokens at a time meet no bank twice
  static constexpr int ROW = D == 64 ? 48 : D == 128 ? 80 : 160;
  static constexpr int SB = D / 32;
  int64_t off[kUnit];
  __attribute__((aligned(16))) char codes[kUnit * ROW];
  __attribute__((aligned(8))) uint8_t scales[2 * kUnit * SB];  // keys', then values'
};

// W words; ONCE marks them as not to be kept in the caches.
template <int W, bool ONCE = false>
__device__ __forceinline__ void load_words(uint32_t* to, const char* p) {
  if constexpr (W == 2) {
    const u32x2* q = reinterpret_cast<const u32x2*>(p);
    const u32x2 w = ONCE ? __builtin_nontemporal_load(q) : *q;
    to[0] = w[0];
    to[1] = w[1];
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4* q = reinterpret_cast<const u32x4*>(p + 16 * i);
      const u32x4 w = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
      for (int j = 0; j < 4; ++j) to[4 * i + j] = w[j];
    }
  }
}

template <int D, bool ONCE>
__device__ __forceinline__ void load_k(Step<D, false>& st, const AttendArgs& a, const int64_t* off, int h,
                                       int n, int g) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const char* p = a.pg.plane[0] + off[16 * t + n] + h * (D * 2) + g * 16;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) load_words<4, ONCE>(&st.k[t][4 * i], p + 64 * i);
  }
}

template <int D, bool ONCE>
__device__ __forceinline__ void load_v(Step<D, false>& st, const AttendArgs& a, const int64_t* off, int h,
                                       int n, int g) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    load_words<D / 32, ONCE>(st.val.v[e], a.pg.plane[1] + off[(e < 4 ? 0 : 12) + 4 * g + e] + h * (D * 2) + n * (D / 8));
}

template <int D, bool>
__device__ __forceinline__ void load_k(Step<D, true>& st, const AttendArgs& a, const int64_t* off, int h,
                                       int n, int g) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
    load_words<D / 32>(st.k[t], a.pg.plane[0] + off[16 * t + n] + h * (D / 2) + g * (D / 8));
}

// Values, and the scale bytes of the token whose row is at `own`: lanes below
// 32 take its key's, the others its value's.
template <int D, bool>
__device__ __forceinline__ void load_v(Step<D, true>& st, const AttendArgs& a, const int64_t* off,
                                       int64_t own, int h, int n, int g) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
    load_words<D / 32>(st.v[t], a.pg.plane[1] + off[16 * t + n] + h * (D / 2) + g * (D / 8));
  const char* p = (g < 2 ? a.pg.plane[0] : a.pg.plane[1]) + own + a.pg.H * (D / 2) + h * (D / 32);
  if constexpr (D == 64) st.sc[0] = *reinterpret_cast<const uint16_t*>(p);
  if constexpr (D == 128) st.sc[0] = *reinterpret_cast<const uint32_t*>(p);
  if constexpr (D == 256) load_words<2>(st.sc, p);
}

template <int D>
__device__ __forceinline__ void stash(const Step<D, true>& st, Scratch<D, true>& lds, int lane) {
  using L = Scratch<D, true>;
  const int n = lane & 15, g = lane >> 4;
  wave_sync();
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    char* p = lds.codes + (16 * t + n) * L::ROW + g * (D / 8);
    if constexpr (D == 64) {
      *reinterpret_cast<u32x2*>(p) = u32x2{st.v[t][0], st.v[t][1]};
    } else {
#pragma unroll
      for (int i = 0; i < D / 128; ++i)
        *reinterpret_cast<u32x4*>(p + 16 * i) =
            u32x4{st.v[t][4 * i], st.v[t][4 * i + 1], st.v[t][4 * i + 2], st.v[t][4 * i + 3]};
    }
  }
  uint8_t* s = lds.scales + lane * L::SB;
  if constexpr (D == 64) *reinterpret_cast<uint16_t*>(s) = (uint16_t)st.sc[0];
  if constexpr (D == 128) *reinterpret_cast<uint32_t*>(s) = st.sc[0];
  if constexpr (D == 256) *reinterpret_cast<u32x2*>(s) = u32x2{st.sc[0], st.sc[1]};
  wave_sync();
}

template <int D>
__device__ __forceinline__ void fetch(Values<D, true>& x, const Scratch<D, true>& lds, int lane) {
  using L = Scratch<D, true>;
  const int n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int tok = (e < 4 ? 0 : 12) + 4 * g + e;
    const char* p = lds.codes + tok * L::ROW + n * (D / 32);
    if constexpr (D == 64) x.v[e][0] = *reinterpret_cast<const uint16_t*>(p);
    if constexpr (D == 128) x.v[e][0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (D == 256) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
      x.v[e][0] = w[0];
      x.v[e][1] = w[1];
    }
    x.scale[e] = lds.scales[(kUnit + tok) * L::SB + n * (D / 16) / 32];
  }
}

// Word w (two channels) of the values that a lane holds of token e.
template <int D, bool Q4>
__device__ __forceinline__ uint32_t v_word(const Values<D, Q4>& x, int e, int w) {
  if constexpr (!Q4) return x.v[e][w];
  const uint32_t codes = x.v[e][w / 4];
  const float s = block_scale(x.scale[Q4 ? e : 0]);
  switch (w % 4) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
  }
}

// Steps on their way at a time: what the registers hold beside the query and
// the outputs, and enough bytes in flight for memory's latency.
template <int D, bool Q4>
constexpr int steps_ahead() {
  if (Q4) return D == 64 ? 3 : 2;
  return D == 64 ? 2 : 1;
}

// LDS that a wavefront gathers its scores in: what leaves a compute unit its
// wavefronts (eight, or four of 256 channels).
template <int D, bool Q4>
constexpr int kKeepFloats = ((160 * 1024 / (D == 256 ? 4 : 8) - 1280 - (int)sizeof(Scratch<D, Q4>)) / 4) & ~127;

// Units [u0, u1) of sequence b for KV head h.  whole: the units are all of the
// sequence's, the result is final; else it goes to partial slot `slot`.
template <int D, bool Q4, bool ONCE, bool KEEP>
__device__ __forceinline__ void attend_share(const AttendArgs& a, const WavePlan& p, int b, int h, const SeqTokens& tk,
                             int u0, int u1, bool whole, int slot, Scratch<D, Q4>& lds, float* keep, int lane) {
  using S = Step<D, Q4>;
  constexpr int KS = S::KS, VC = D / 16;
  const PagedArgs& g = a.pg;
  const int n = lane & 15, q4 = lane >> 4;
  const int rows = tk.nn * a.G;  // rows of real tokens
  const int begin = u0 * kUnit, end = min(tk.n, u1 * kUnit);  // this share's slots (end > begin)
  const int seen_by_all = tk.n - tk.nn + 1;
  // The page table 64 entries at a time, the next 64 on their way; tokens past
  // the share's end stand for the last one, whose row costs no more traffic.
  const int32_t* pt = g.pt + (int64_t)b * g.ld_pt;
  auto page_index = [&](int tok) {
    return g.page_shift >= 0 ? tok >> g.page_shift : (int)((uint32_t)tok / (uint32_t)g.page_size);
  };
  const int last_page = page_index(end - 1);
  auto load_pages = [&](int first) { return pt[min(first + lane, last_page)]; };
  int page0 = page_index(begin);
  int pages = load_pages(page0), pages_next = load_pages(page0 + 64);

  bf16x8 qf[KS];
  f32x4 o[VC];
  float top = kNegInf, sum = 0.f;
  const int r = n;  // this lane's row
  const int c = r / a.G, hq = h * a.G + (r - c * a.G);
  const bool real = r < rows;
  const char* qp = a.q.base + (b * a.q.ld_seq + c * a.q.ld_tok + hq * a.q.ld_head) * 2;
  const int lim = real ? tk.n - tk.nn + c + 1 : 0;  // slots it sees
  // Scores are gathered in LDS and written in runs as long as it holds, past the
  // caches: memory that reads at its full rate has no room for a few lines of
  // writes a step.  (32 sequences of 8k-32k tokens, 84 MB of scores beside 2.69 GB
  // of rows: 587 us for the call with a store a step, 527 in runs through the
  // caches, 506 past them, 495 with each wavefront's runs in one piece; 431
  // without the writes.)
  const int first_kept = KEEP ? max(0, tk.nn - p.watch) * a.G : 0;
  const int kept_rows = KEEP ? rows - first_kept : 1, in_keep = KEEP ? kKeepFloats<D, Q4> / (kept_rows * kUnit) : 0;
  float* to_keep = nullptr;  // this lane's place there, if its row is counted
  int n_kept = 0;            // steps gathered
  if constexpr (KEEP) {
    if (real && r >= first_kept) to_keep = keep + (r - first_kept) * kUnit + 4 * q4;
  }
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int ch = Q4 ? (D / 4) * q4 + 8 * s : 32 * s + 8 * q4;
    u32x4 w = {0, 0, 0, 0};
    if (real) w = *reinterpret_cast<const u32x4*>(qp + ch * 2);
    qf[s] = as_bf16x8(w);
  }
#pragma unroll
  for (int j = 0; j < VC; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int at32 = lane & (kUnit - 1);
  bool any_bad = false;
  int64_t own = 0;  // the row of this lane's token
  // A step's row offsets to LDS; returns which of its tokens exist.
  auto put_offsets = [&](int base) -> uint32_t {
    if (page_index(min(base, end - 1)) - page0 >= 64) {
      page0 += 64;
      pages = pages_next;
      pages_next = load_pages(page0 + 64);
    }
    const int tok = min(base + at32, end - 1);
    const int pi = page_index(tok), rel = pi - page0;
    int pg = __shfl(pages, rel & 63);
    if (__any(rel >= 64)) {  // (a branch, not to wait for the next entries before they are due)
      const int beyond = __shfl(pages_next, rel & 63);
      pg = rel < 64 ? pg : beyond;
    }
    const bool good = pg >= 0 && pg < g.n_pages;
    const int64_t at = (int64_t)pg * g.s_page + (int64_t)(tok - pi * g.page_size) * g.row_bytes;
    own = good ? at : 0;
    wave_sync();
    lds.off[at32] = own;
    wave_sync();
    any_bad |= !good;
    return (uint32_t)__ballot(good && base + at32 < end);
  };

  constexpr int P = steps_ahead<D, Q4>();
  Step<D, Q4> steps[P];
  uint32_t exist[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    exist[i] = put_offsets(begin + i * kUnit);
    load_k<D, ONCE>(steps[i], a, lds.off, h, n, q4);
    if constexpr (Q4)
      load_v<D, ONCE>(steps[i], a, lds.off, own, h, n, q4);
    else
      load_v<D, ONCE>(steps[i], a, lds.off, h, n, q4);
  }
  // One step of 32 tokens; the keys of the one P steps on are on their way
  // once this one's are used up, and so its values.
  auto step = [&](Step<D, Q4>& st, uint32_t& exists, int base) {
    const uint32_t ok = exists;
    // 4-bit rows of two heads and more share lines: the heads' wavefronts keep
    // together (they walk the same share, and so come here equally often), or
    // lines leave the cache before the last of them has read its part.
    if constexpr (Q4) __builtin_amdgcn_s_barrier();
    uint32_t key_scale[2] = {0, 0};
    if constexpr (Q4) stash<D>(st, lds, lane);
    exists = put_offsets(base + P * kUnit);
    if constexpr (Q4) {
      load_v<D, ONCE>(st, a, lds.off, own, h, n, q4);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* x = lds.scales + (16 * i + n) * Scratch<D, true>::SB;
        if constexpr (D == 64) key_scale[i] = x[q4 / 2];
        if constexpr (D == 128) key_scale[i] = x[q4];
        if constexpr (D == 256) key_scale[i] = *reinterpret_cast<const uint16_t*>(x + 2 * q4);
      }
    }
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32x4 w;
        if constexpr (Q4) {
          const uint32_t byte =
              D == 256 ? (k < KS / 2 ? key_scale[i] & 255u : key_scale[i] >> 8) : key_scale[i];
          w = decode8(st.k[i][k], block_scale(byte));
        } else {
          w = u32x4{st.k[i][4 * k], st.k[i][4 * k + 1], st.k[i][4 * k + 2], st.k[i][4 * k + 3]};
        }
        s[i] = mfma16(as_bf16x8(w), qf[k], s[i]);
      }
    // (a share's last steps bring nothing more: one sequence 15.0 -> 14.6 us.
    // 4-bit steps are no faster with the branch.)
    const bool more = Q4 || base + P * kUnit < end;
    if (more) load_k<D, ONCE>(st, a, lds.off, h, n, q4);
    const bool special = ok != 0xffffffffu || base + 32 > seen_by_all;
    bf16x8 pf;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s[e / 4][e % 4];
    if (special) {
      asm volatile("");  // (kept a branch: the masks are not for every step)
      const uint32_t mine = (ok & below(lim - base)) >> (4 * q4);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = mine >> ((e < 4 ? 0 : 12) + e) & 1u ? x[e] : kNegInf;
    }
    if constexpr (KEEP) {
      if (to_keep) {
        float* to = to_keep + n_kept * (kept_rows * kUnit);
        *reinterpret_cast<f32x4*>(to) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(to + 16) = f32x4{x[4], x[5], x[6], x[7]};
      }
      ++n_kept;
      if (n_kept == in_keep || base + kUnit >= end) {
        wave_sync();
        const int per = kept_rows * (kUnit / 4);  // vectors a step
        float* out = p.kept + p.kept_at(b, h, base / kUnit + 1 - n_kept, a.G, g.H);
        for (int i = lane; i < n_kept * per; i += 64) {
          const int u = i / per;
          __builtin_nontemporal_store(*reinterpret_cast<const f32x4*>(keep + 4 * i),
                                      reinterpret_cast<f32x4*>(out + u * (p.watch * a.G * kUnit) + 4 * (i - u * per)));
        }
        wave_sync();
        n_kept = 0;
      }
    }
    float m = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) m = fmaxf(m, x[e]);
    m *= a.scale2;
    // The maximum may lag by 2^8: weights up to 256 lose nothing, and most
    // steps then exchange and rescale nothing.
    if (__any(m > top + 8.f)) {
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float grown = fmaxf(top, m);
      const float f = grown == top ? 1.f : exp2_fast(top - grown);
      top = grown;
      sum *= f;
#pragma unroll
      for (int j = 0; j < VC; ++j) o[j] *= f;
    }
    const float base2 = top == kNegInf ? 0.f : top;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = exp2_fast(fmaf(x[e], a.scale2, -base2));
      sum += w[e];
    }
    // (The product takes its operands in one type, and V has bf16: a weight is
    // rounded to 8 bits, off by 2^-8 of itself at most, and the sum keeps what
    // it was.  With random signs that leaves the result 2.4e-3 off where its own
    // rounding leaves 1.7e-3.  A second product with what the rounding leaves
    // would make an infinite value NaN, 0 times it; it took 1 % more for 32
    // sequences in 4 bits, 3 to 10 % for short ones, none where HBM waits.)
    pf = as_bf16x8(u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]),
                            pack_bf16(w[6], w[7])});
    Values<D, Q4> fetched;
    if constexpr (Q4) fetch<D>(fetched, lds, lane);
    Values<D, Q4>& val = [&]() -> Values<D, Q4>& {
      if constexpr (Q4)
        return fetched;
      else
        return st.val;
    }();
    // V: an instruction takes one channel's 8 tokens, two channels come of 8
    // words.
    if (!special) {
#pragma unroll
      for (int w = 0; w < VC / 2; ++w) {
        u32x4 c0, c1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = v_word(val, 2 * i, w), y = v_word(val, 2 * i + 1, w);
          c0[i] = halves_lo(x, y);
          c1[i] = halves_hi(x, y);
        }
        o[2 * w] = mfma16(as_bf16x8(c0), pf, o[2 * w]);
        o[2 * w + 1] = mfma16(as_bf16x8(c1), pf, o[2 * w + 1]);
      }
    } else {
      // What does not exist counts as 0, whatever its bytes are.  A NaN or an
      // infinity that some rows see and others do not (0 times it is NaN)
      // needs a pass for each token c, without the values hidden from it.
      auto masks = [&](int seen) {
        const uint32_t mine = (ok & below(seen - base)) >> (4 * q4);
        u32x4 m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = (i < 2 ? 0 : 12) + 2 * i;
          m[i] = (mine >> j & 1u ? 0xffffu : 0u) | (mine >> (j + 1) & 1u ? 0xffff0000u : 0u);
        }
        return m;
      };
      const u32x4 there = masks(tk.n);
      bool odd = false;
      if (tk.nn > 1) {
#pragma unroll
        for (int w = 0; w < VC / 2; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = v_word(val, 2 * i, w), y = v_word(val, 2 * i + 1, w);
            odd |= word_not_finite(halves_lo(x, y) & there[i]) | word_not_finite(halves_hi(x, y) & there[i]);
          }
      }
      const bool by_token = __any(odd);
      for (int c = by_token ? 0 : tk.nn - 1; c < tk.nn; ++c) {
        const int seen = tk.n - tk.nn + c + 1;
        const u32x4 m = masks(seen);
        // (what a pass makes of the values is made anew: kept for the next
        // one it would take a register file of its own)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < Values<D, Q4>::VW; ++w) asm volatile("" : "+v"(val.v[e][w]));
#pragma unroll
        for (int w = 0; w < VC / 2; ++w) {
          u32x4 c0, c1;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = v_word(val, 2 * i, w), y = v_word(val, 2 * i + 1, w);
            c0[i] = halves_lo(x, y) & m[i];
            c1[i] = halves_hi(x, y) & m[i];
          }
          const f32x4 y0 = mfma16(as_bf16x8(c0), pf, o[2 * w]);
          const f32x4 y1 = mfma16(as_bf16x8(c1), pf, o[2 * w + 1]);
          if (!by_token || lim == seen) {
            o[2 * w] = y0;
            o[2 * w + 1] = y1;
          }
        }
      }
    }
    if constexpr (!Q4)
      if (more) load_v<D, ONCE>(st, a, lds.off, h, n, q4);
  };
#pragma clang loop unroll(disable)
  for (int base = begin; base < end; base += P * kUnit) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (base + i * kUnit < end) step(steps[i], exist[i], base + i * kUnit);
  }
  if (__any(any_bad) && lane == 0) raise_flag(g.status, b);

  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (r >= a.R) return;
  // (lane (n, q4) holds channels D/4*q4 + VC*i + j of row r)
  if (whole) {
    const bool some = real && sum != 0.f;
    const float inv = 1.f / sum;
    char* op = a.out.base + (b * a.out.ld_seq + c * a.out.ld_tok + hq * a.out.ld_head + (D / 4) * q4) * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VC; j += 4) {
        u32x2 w = {0u, 0u};
        if (some) {
          w[0] = pack_bf16(o[j][i] * inv, o[j + 1][i] * inv);
          w[1] = pack_bf16(o[j + 2][i] * inv, o[j + 3][i] * inv);
        }
        *reinterpret_cast<u32x2*>(op + (VC * i + j) * 2) = w;
      }
    if (q4 == 0) write_log_sum<KEEP>(a, b, hq, c, top, sum, some);
  } else if (real) {
    const int64_t at = ((int64_t)slot * g.H + h) * a.R + r;
    float* po = p.part_o + at * D + (D / 4) * q4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VC; j += 4)
        *reinterpret_cast<f32x4*>(po + VC * i + j) =
            f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
    if (q4 == 0) p.part_ml[at] = make_float2(top, sum);
  }
}

// The outputs of a sequence with nothing to see.
template <int D, bool KEEP>
__device__ void attend_nothing(const AttendArgs& a, int b, int h, int lane) {
  for (int i = lane; i < a.R * (D / 8); i += 64) {
    const int r = i / (D / 8), x = i - r * (D / 8);
    const int c = r / a.G, hq = h * a.G + (r - c * a.G);
    *reinterpret_cast<u32x4*>(a.out.base + (b * a.out.ld_seq + c * a.out.ld_tok + hq * a.out.ld_head + x * 8) * 2) =
        u32x4{0, 0, 0, 0};
    if (x == 0) write_log_sum<KEEP>(a, b, hq, c, kNegInf, 0.f, false);
  }
}

// A team's share: units [lo, hi) of all sequences' in a row (`total` of them),
// which begin in sequence b, whose own begin at `before`.
struct Share {
  int b, before, lo, hi, per, total;
  SeqTokens t;
};

// Units of a share: enough to leave no team without, and, where the teams
// would outnumber what is worth joining, enough to balance a step's time with
// a join's per share (about 40 to 1, so sqrt(units of a sequence / 40)).  One KV
// head, 64k slots: 51 us in single units, 19 so; 600k: 92, 76; one sequence of
// 4k slots, 8 KV heads, 13.1 both.
__device__ __forceinline__ int units_per_team(int total, int n_teams, int B) {
  const int balanced = (int)sqrtf((float)total / (40.f * (float)B));
  return max(max(1, balanced), (total + n_teams - 1) / n_teams);
}

// All sequences' units, a lane each (their loads at once), and where this
// team's share begins among them; false if it is empty.
template <int SETS>
__device__ __forceinline__ bool find_share(const PagedArgs& g, int n_teams, int team, int lane, Share& x) {
  int n[SETS], nn[SETS], upto[SETS], total = 0;
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    const int b = 64 * i + lane;
    const SeqTokens t = seq_tokens(g, min(b, g.B - 1));  // (no branch between the loads)
    n[i] = b < g.B ? t.n : 0;
    nn[i] = b < g.B ? t.nn : 0;
  }
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    upto[i] = total;
    if (64 * i < g.B) {
      upto[i] += wave_scan(units_of(SeqTokens{n[i], nn[i], false}));
      total = __builtin_amdgcn_readlane(upto[i], 63);
    }
  }
  x.total = total;
  x.per = units_per_team(total, n_teams, g.B);
  x.lo = team * x.per;
  x.hi = min(total, x.lo + x.per);
  if (x.lo >= x.hi) return false;
  x.b = x.before = 0;
  x.t = {0, 0, false};
#pragma unroll
  for (int i = 0; i < SETS; ++i) {
    const uint64_t past = __ballot(upto[i] > x.lo);
    if (past && x.t.nn == 0) {
      const int k = __ffsll((unsigned long long)past) - 1;
      x.t.n = __builtin_amdgcn_readlane(n[i], k);
      x.t.nn = __builtin_amdgcn_readlane(nn[i], k);
      x.before = __builtin_amdgcn_readlane(upto[i], k) - units_of(x.t);
      x.b = 64 * i + k;
    }
  }
  return true;
}

// bf16 rows are not kept in the caches when the sequences hold more than half
// of the last-level cache: 32 sequences of 8k-32k tokens 453 -> 415 us, 4 of 16k
// (256 MiB) 55.2 -> 50.7.  Fewer may still be there at the next token: 2 of 16k
// 29.0 us kept, 31.0 not; 4224 slots 13.3, 14.5; 32 of 1024 29.3, 31.8.
// (4-bit rows share lines between wavefronts and are kept: no difference.)
constexpr int64_t kCacheBytes = 128 << 20;

// LARGE: the page tables cover more than that; whether the sequences hold as
// much, their counts say.
template <int D, bool Q4, bool LARGE, bool KEEP>
__global__ __launch_bounds__(D == 256 ? 256 : 512) void k_attend_wave(AttendArgs a, WavePlan p) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const PagedArgs& g = a.pg;
  const int h = blockIdx.y * p.hw + wave;
  const int64_t team = linear_block();
  if (h >= g.H || team >= p.n_teams) return;
  Scratch<D, Q4>* scratch;
  float* keep = nullptr;
  if constexpr (KEEP) {  // (as many as the workgroup has wavefronts: Scratch, then the scores)
    extern __shared__ __align__(16) char s_dynamic[];
    scratch = reinterpret_cast<Scratch<D, Q4>*>(s_dynamic);
    keep = reinterpret_cast<float*>(s_dynamic + p.hw * sizeof(Scratch<D, Q4>)) + wave * kKeepFloats<D, Q4>;
  } else {
    __shared__ Scratch<D, Q4> s_scratch[D == 256 ? 4 : 8];
    scratch = s_scratch;
  }
  Scratch<D, Q4>& lds = scratch[wave];
  Share x;
  if (!p.split) {  // a sequence to a team
    x.b = (int)team;
    x.t = seq_tokens(g, x.b);
    if (x.t.bad && lane == 0) raise_flag(g.status, x.b);
    x.before = x.lo = 0;
    x.hi = units_of(x.t);
    if (x.hi == 0) {
      attend_nothing<D, KEEP>(a, x.b, h, lane);
      return;
    }
  } else if (g.B <= 64) {
    // (a launch fetches its instructions anew: one sequence of 4k slots 13.1 us
    // with this, 15.1 through the code for 1024)
    if (!find_share<1>(g, p.n_teams, (int)team, lane, x)) return;
  } else {
    if (!find_share<kSplitBatch / 64>(g, p.n_teams, (int)team, lane, x)) return;
  }
  // (without shares a team knows one sequence of more than a thousand: too many
  // to be there at the next token, unless all are short)
  const bool once = LARGE && (!p.split || (int64_t)x.total * (2 * kUnit) * g.row_bytes > kCacheBytes);
  for (;;) {
    const int u = units_of(x.t);
    if (u > 0) {
      const int u0 = x.lo - x.before, u1 = min(u, x.hi - x.before);
      // (who has a sequence's first unit tells the join where its shares are)
      if (p.split && u0 == 0 && h == 0 && lane == 0)
        p.shares[x.b] = make_int2((int)team, (x.before + u - 1) / x.per - (int)team + 1);
      const bool whole = u0 == 0 && u1 == u;
      if (once)
        attend_share<D, Q4, LARGE, KEEP>(a, p, x.b, h, x.t, u0, u1, whole, (int)team + x.b, lds, keep, lane);
      else
        attend_share<D, Q4, false, KEEP>(a, p, x.b, h, x.t, u0, u1, whole, (int)team + x.b, lds, keep, lane);
      x.lo = x.before + u1;
      x.before += u;
    }
    if (x.lo >= x.hi) break;
    x.t = seq_tokens(g, ++x.b);
  }
}

template <int D>
struct JoinScratch {
  float o[8][D], top[8], sum[8];
};

// Joins the shares of one row: a workgroup per (sequence, query row), its
// wavefronts taking turns over the shares, 16 at a time, in a fixed order,
// and then their results.  Bound by latency: after the shares' place two round
// trips (a pass for the maximum and one for the sums took a third).  5.4 us
// for 132 shares of 32 rows and for 32 sequences of 8 shares each, 1.5 of them
// the launch.
template <int D, bool KEEP>
__device__ __forceinline__ void join_row(const AttendArgs& a, const WavePlan& p, int64_t row, JoinScratch<D>& lds) {
  constexpr int E = D / 64, AHEAD = 16;
  float (&s_o)[8][D] = lds.o;
  float (&s_top)[8] = lds.top;
  float (&s_sum)[8] = lds.sum;
  const PagedArgs& g = a.pg;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t id = (uint32_t)row, per_seq = (uint32_t)(a.R * g.H);
  const int b = (int)(id / per_seq);
  if (b >= g.B) return;
  const int hr = (int)(id - (uint32_t)b * per_seq);
  const int h = hr / a.R, r = hr - h * a.R;
  const int2 place = p.shares[b];  // (nothing there if the sequence has no units)
  const SeqTokens t = seq_tokens(g, b);
  if (t.bad && threadIdx.x == 0 && hr == 0) raise_flag(g.status, b);
  const int c = r / a.G, hq = h * a.G + (r - c * a.G);
  char* op = a.out.base + (b * a.out.ld_seq + c * a.out.ld_tok + hq * a.out.ld_head) * 2;
  const bool any = units_of(t) > 0;
  if (any && place.y == 1) return;  // written whole
  if (!any || r >= t.nn * a.G) {
    if (threadIdx.x < D / 8) reinterpret_cast<u32x4*>(op)[threadIdx.x] = u32x4{0, 0, 0, 0};
    if (threadIdx.x == 0) write_log_sum<KEEP>(a, b, hq, c, kNegInf, 0.f, false);
    return;
  }
  const int n = place.y;
  const int64_t at = ((int64_t)(place.x + b) * g.H + h) * a.R + r;  // + share * H * R
  const int64_t step = (int64_t)g.H * a.R;
  float top = kNegInf, sum = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i = wave; i < n; i += waves * AHEAD) {
    float2 ml[AHEAD];
    float x[AHEAD][E];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i + k * waves < n) {
        const int64_t from = at + (i + k * waves) * step;
        ml[k] = p.part_ml[from];
#pragma unroll
        for (int e = 0; e < E; ++e) x[k][e] = p.part_o[from * D + lane * E + e];
      } else {
        ml[k] = make_float2(kNegInf, 0.f);
      }
    }
    float grown = top;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) grown = fmaxf(grown, ml[k].x);
    const float base2 = grown == kNegInf ? 0.f : grown;
    const float f = exp2_fast(top - base2);
    sum *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= f;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float w = exp2_fast(ml[k].x - base2);
      if (i + k * waves < n) {  // (0 times an infinity would not be 0)
        sum += w * ml[k].y;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += w * x[k][e];
      }
    }
    top = grown;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[wave][lane * E + e] = o[e];
  if (lane == 0) {
    s_top[wave] = top;
    s_sum[wave] = sum;
  }
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  top = kNegInf;
  for (int w = 0; w < waves; ++w) top = fmaxf(top, s_top[w]);
  const float base2 = top == kNegInf ? 0.f : top;
  float x = 0.f, y = 0.f;
  sum = 0.f;
  for (int w = 0; w < waves; ++w) {
    const float f = exp2_fast(s_top[w] - base2);
    sum += f * s_sum[w];
    x += f * s_o[w][2 * threadIdx.x];
    y += f * s_o[w][2 * threadIdx.x + 1];
  }
  const bool some = sum != 0.f;
  const float inv = 1.f / sum;
  reinterpret_cast<uint32_t*>(op)[threadIdx.x] = some ? pack_bf16(x * inv, y * inv) : 0u;
  if (threadIdx.x == 0) write_log_sum<KEEP>(a, b, hq, c, top, sum, some);
}

// Wavefronts resident per SIMD that the shares are counted for.
constexpr int kWavesPerSimd = 2;

WavePlan wave_plan(int B, int H, int d) {
  WavePlan p;
  const int most = d == 256 ? 4 : 8;  // wavefronts of a workgroup (rows of 256 take 512 registers)
  const int groups = (H + most - 1) / most;
  p.hw = (H + groups - 1) / groups;
  p.split = B <= kSplitBatch;
  p.n_teams = B;
  if (p.split) {
    const int waves = std::max(1, device_cus()) * 4 * (d == 256 ? 1 : kWavesPerSimd);
    p.n_teams = (waves + p.hw * groups - 1) / (p.hw * groups);
  }
  p.part_o = nullptr;
  p.part_ml = nullptr;
  p.shares = nullptr;
  p.kept = nullptr;
  p.units = 0;
  p.watch = 0;
  return p;
}

template <int D, bool KEEP>
hipError_t launch_shares(const AttendArgs& a, const WavePlan& p, bool q4, hipStream_t s) {
  const dim3 grid = linear_grid(p.n_teams, p.hw * 64, (a.pg.H + p.hw - 1) / p.hw);
  const dim3 block(p.hw * 64);
  const auto lds = [&](size_t scratch, int floats) { return KEEP ? (unsigned)(p.hw * (scratch + floats * 4)) : 0u; };
  if (q4)
    hipLaunchKernelGGL((k_attend_wave<D, true, false, KEEP>), grid, block,
                       lds(sizeof(Scratch<D, true>), kKeepFloats<D, true>), s, a, p);
  else if ((int64_t)a.pg.B * a.pg.max_tokens * 2 * a.pg.row_bytes > kCacheBytes)
    hipLaunchKernelGGL((k_attend_wave<D, false, true, KEEP>), grid, block,
                       lds(sizeof(Scratch<D, false>), kKeepFloats<D, false>), s, a, p);
  else
    hipLaunchKernelGGL((k_attend_wave<D, false, false, KEEP>), grid, block,
                       lds(sizeof(Scratch<D, false>), kKeepFloats<D, false>), s, a, p);
  return hipGetLastError();
}

// Wavefronts of a workgroup that joins.
int join_waves(const WavePlan& p, int B) {
  const int shares = p.n_teams / B;  // of a sequence, about
  return shares >= 16 ? 8 : 4;
}

size_t part_ml_bytes(const WavePlan& p, int B, int H, int R) {
  return ((size_t)(p.n_teams + B) * H * R * sizeof(float2) + 255) / 256 * 256;
}

constexpr size_t kSharesBytes = kSplitBatch * sizeof(int2);

// The plan with its places in the workspace.
WavePlan placed_plan(const AttendArgs& a, void* ws) {
  WavePlan p = wave_plan(a.pg.B, a.pg.H, a.pg.d);
  if (p.split) {
    p.shares = (int2*)ws;
    p.part_ml = (float2*)((char*)ws + kSharesBytes);
    p.part_o = (float*)((char*)p.part_ml + part_ml_bytes(p, a.pg.B, a.pg.H, a.R));
  }
  return p;
}

}  // namespace
}  // namespace epikv
