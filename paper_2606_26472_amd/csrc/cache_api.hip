// C-ABI host layer of the calls that fill and read the paged cache: argument
// validation and launches.  Every host-detectable error is returned before
// anything is enqueued.
#include <math.h>
#include <string.h>

#include "epikv_internal.h"

#define EPIKV_EXPORT extern "C" __attribute__((visibility("default")))

namespace epikv {
namespace {

constexpr int kMaxChunk = 1 << 24;
constexpr int kMaxHeads = 1024;
constexpr int kMaxTokens = 1 << 25;  // of one sequence: sums over sequences stay in 32 bits

int check_rope_cfg(const epikv_rope_cfg* r) {
  if (!r) return EPIKV_EINVAL_NULL;
  if (r->layout < EPIKV_ROPE_HALF || r->layout > EPIKV_ROPE_INTERLEAVED) return EPIKV_EINVAL_PARAM;
  if (r->scaling < EPIKV_ROPE_PLAIN || r->scaling > EPIKV_ROPE_YARN) return EPIKV_EINVAL_PARAM;
  if (!(r->theta > 1.f) || !isfinite(r->theta)) return EPIKV_EINVAL_PARAM;
  if (!(r->amplitude > 0.f) || !isfinite(r->amplitude)) return EPIKV_EINVAL_PARAM;
  if (r->scaling != EPIKV_ROPE_PLAIN && (!(r->factor > 0.f) || !isfinite(r->factor)))
    return EPIKV_EINVAL_PARAM;
  if (r->scaling >= EPIKV_ROPE_BANDS &&
      (!(r->turns_low > 0.f) || !(r->turns_high > r->turns_low) || !isfinite(r->turns_high) ||
       r->original < 1))
    return EPIKV_EINVAL_PARAM;
  if (r->rotary_dim < 16 || r->rotary_dim > 1024 || r->rotary_dim % 16) return EPIKV_EINVAL_SHAPE;
  if (r->n_pos < 1 || r->n_pos > (1 << 24)) return EPIKV_EINVAL_SHAPE;
  return EPIKV_OK;
}

int check_axes(const epikv_rope_cfg* r, const epikv_axes* x) {
  const int st = check_rope_cfg(r);
  if (st) return st;
  if (!x) return EPIKV_EINVAL_NULL;
  if (x->order < EPIKV_AXES_SECTIONS || x->order > EPIKV_AXES_TURNS) return EPIKV_EINVAL_PARAM;
  if (x->frequencies < EPIKV_AXES_SHARED || x->frequencies > EPIKV_AXES_APART) return EPIKV_EINVAL_PARAM;
  if (x->n_axes < 1 || x->n_axes > EPIKV_MAX_AXES) return EPIKV_EINVAL_SHAPE;
  const int least = x->frequencies == EPIKV_AXES_APART && r->scaling == EPIKV_ROPE_NTK ? 2 : 1;
  int64_t sum = 0;
  for (int a = 0; a < x->n_axes; ++a) {
    if (x->pairs[a] < least) return EPIKV_EINVAL_SHAPE;
    sum += x->pairs[a];
  }
  return sum == r->rotary_dim / 2 ? EPIKV_OK : EPIKV_EINVAL_SHAPE;
}

// Every pair's place on its axis and how many pairs that has, of checked axes.
void deal_pairs(const epikv_axes* x, uint16_t (&place)[512], uint16_t (&count)[512]) {
  int used[EPIKV_MAX_AXES] = {0, 0, 0, 0};
  int total = 0, a = 0;
  for (int k = 0; k < x->n_axes; ++k) total += x->pairs[k];
  for (int i = 0; i < total; ++i) {
    while (used[a] == x->pairs[a]) a = (a + 1) % x->n_axes;
    count[i] = (uint16_t)x->pairs[a];
    place[i] = (uint16_t)used[a]++;
    if (x->order == EPIKV_AXES_TURNS) a = (a + 1) % x->n_axes;
  }
}

// Query heads: a multiple of the KV heads, the rows of one KV head counted in
// 32 bits.
bool heads_fit(int32_t chunk, int32_t n_kv_heads, int32_t n_heads) {
  return n_heads >= 1 && n_heads <= kMaxHeads && n_heads % n_kv_heads == 0 &&
         (int64_t)chunk * n_heads <= INT32_MAX / 2;
}

// Strides of a [B][chunk][heads][d] tensor, and the bytes it spans.
int check_rows(const epikv_rows* x, bool aligned_base = true) {
  if (!x->base) return EPIKV_EINVAL_NULL;
  if (x->ld_seq < 0 || x->ld_tok < 0 || x->ld_head < 0) return EPIKV_EINVAL_SHAPE;
  if (x->ld_seq % 8 || x->ld_tok % 8 || x->ld_head % 8) return EPIKV_EALIGN;
  if (aligned_base && !aligned16(x->base)) return EPIKV_EALIGN;
  return EPIKV_OK;
}

size_t rows_span(const epikv_rows* x, int B, int C, int heads, int d, int es) {
  return (size_t)((int64_t)(B - 1) * x->ld_seq + (int64_t)(C - 1) * x->ld_tok +
                  (int64_t)(heads - 1) * x->ld_head + d) * (size_t)es;
}

// A tensor that is written must have a place of its own for every row: its
// axes of more than one entry, by rising stride, each past those before it.
bool rows_apart(const epikv_rows* x, int B, int C, int heads, int d) {
  struct Axis {
    int64_t stride, n;
  } axis[3] = {{x->ld_seq, B}, {x->ld_tok, C}, {x->ld_head, heads}};
  std::sort(axis, axis + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  int64_t span = d;
  for (const Axis& a : axis) {
    if (a.n == 1) continue;
    if (a.stride < span) return false;
    span += a.stride * (a.n - 1);
  }
  return true;
}

int check_out_rows(const epikv_rows* x, int B, int C, int heads, int d) {
  const int st = check_rows(x);
  if (st) return st;
  return rows_apart(x, B, C, heads, d) ? EPIKV_OK : EPIKV_EINVAL_SHAPE;
}

bool same_rows(const epikv_rows* x, const epikv_rows* y) {
  return x->base == y->base && x->ld_seq == y->ld_seq && x->ld_tok == y->ld_tok &&
         x->ld_head == y->ld_head;
}

// Whether an element of x (hx heads) may be one of y (hy heads).  Spans that
// overlap may still hold rows between each other's, as slices of one fused
// projection do: by the remainders of a period P, which every stride that is a
// multiple of P leaves as they are, x has [0, wx) and y [at, at + wy).  The
// periods tried are the strides.
bool rows_meet(const epikv_rows* x, int hx, const epikv_rows* y, int hy, int B, int C, int d, int es) {
  if (!overlap(x->base, rows_span(x, B, C, hx, d, es), y->base, rows_span(y, B, C, hy, d, es)))
    return false;
  struct Axis {
    int64_t stride, n;
  };
  const Axis ax[3] = {{x->ld_seq, B}, {x->ld_tok, C}, {x->ld_head, hx}};
  const Axis ay[3] = {{y->ld_seq, B}, {y->ld_tok, C}, {y->ld_head, hy}};
  const int64_t between = (int64_t)((uintptr_t)y->base - (uintptr_t)x->base) / es;
  auto width = [&](const Axis* a, int64_t period) {
    int64_t w = d;
    for (int i = 0; i < 3; ++i)
      if (a[i].n > 1 && a[i].stride % period) w += (a[i].n - 1) * a[i].stride;
    return w;
  };
  for (const Axis* a : {ax, ay})
    for (int i = 0; i < 3; ++i) {
      const int64_t period = a[i].stride;
      if (a[i].n == 1 || period == 0) continue;
      const int64_t at = (between % period + period) % period;
      if (at >= width(ax, period) && at + width(ay, period) <= period) return false;
    }
  return true;
}

// y may be x itself or lie apart from it.
int check_alias(const epikv_rows* x, const epikv_rows* y, int B, int C, int heads, int d, int es) {
  if (same_rows(x, y)) return EPIKV_OK;
  return rows_meet(x, heads, y, heads, B, C, d, es) ? EPIKV_EALIAS : EPIKV_OK;
}

int check_positions(const int32_t* positions, int64_t ld_pos, int32_t chunk) {
  if (!positions) return EPIKV_EINVAL_NULL;
  if (ld_pos != 0 && ld_pos < chunk) return EPIKV_EINVAL_SHAPE;
  return EPIKV_OK;
}

int check_paged(const epikv_cfg* c, const epikv_pool* pool, int32_t layer, int32_t chunk,
                const int32_t* pt, int64_t ld_pt) {
  int st = check_cfg(c);
  if (st) return st;
  if (chunk < 1 || chunk > kMaxChunk || (int64_t)c->batch * chunk > INT32_MAX)
    return EPIKV_EINVAL_SHAPE;
  if (layer < 0 || layer >= c->n_layers) return EPIKV_EINVAL_SHAPE;
  st = check_pool(pool);
  if (st) return st;
  if (!pt) return EPIKV_EINVAL_NULL;
  if (ld_pt < 1) return EPIKV_EINVAL_SHAPE;
  return EPIKV_OK;
}

RowsArg rows_arg(const epikv_rows* x) {
  return RowsArg{(char*)x->base, x->ld_seq, x->ld_tok, x->ld_head};
}

RopeArg rope_arg(const epikv_rope_cfg* r, const float* table, const int32_t* positions,
                 int64_t ld_pos, int32_t transpose) {
  RopeArg a;
  memset(&a, 0, sizeof(a));
  a.positions = positions;
  a.ld_pos = ld_pos;
  if (r) {
    a.table = (const float2*)table;
    a.r = r->rotary_dim;
    a.n_pos = r->n_pos;
    a.interleaved = r->layout == EPIKV_ROPE_INTERLEAVED;
    a.transpose = transpose != 0;
  }
  return a;
}

// Slots that a page table of ld_pt entries covers.
int32_t slots_of(const epikv_cfg* c, int64_t ld_pt) {
  return (int32_t)std::min<int64_t>(std::min<int64_t>(ld_pt, INT32_MAX) * c->page_size, kMaxTokens);
}

RopeAxesArg rope_axes_arg(const epikv_rope_cfg* r, const epikv_axes* x, const float* table,
                          const int32_t* positions, int64_t ld_pos, int32_t transpose) {
  RopeAxesArg a = {};
  static_cast<RopeArg&>(a) = rope_arg(r, table, positions, ld_pos, transpose);
  a.n_axes = x->n_axes;
  // Runs: of one axis each, or of those that still take turns.
  int left[EPIKV_MAX_AXES], first = 0, n_runs = 0;
  for (int k = 0; k < x->n_axes; ++k) left[k] = x->pairs[k];
  for (int k = 0; k < EPIKV_MAX_AXES; ++k) {  // (runs past the last: past every pair)
    a.start[k] = 1 << 20;
    a.turns[k] = 1;
    a.inverse[k] = 65536;
  }
  while (first < r->rotary_dim / 2) {
    int turning[EPIKV_MAX_AXES], m = 0, rounds = INT32_MAX;
    for (int k = 0; k < x->n_axes; ++k)
      if (left[k] > 0 && (m == 0 || x->order == EPIKV_AXES_TURNS)) {
        turning[m++] = k;
        rounds = std::min(rounds, left[k]);
      }
    const int run = n_runs++;
    a.start[run] = first;
    a.turns[run] = (uint32_t)m;
    a.inverse[run] = (uint32_t)((65536 + m - 1) / m);
    // (pair i is turned by turning[(i - first) % m])
    for (int i = 0; i < 16; ++i)
      a.axes[run] |= (uint32_t)turning[((i - first) % m + m) % m] << (2 * i);
    for (int k = 0; k < m; ++k) left[turning[k]] -= rounds;
    first += m * rounds;
  }
  return a;
}

RopeTableArgs table_args(const epikv_rope_cfg* rope, float* table) {
  RopeTableArgs a;
  a.table = table;
  a.n_pos = rope->n_pos;
  a.half = rope->rotary_dim / 2;
  a.scaling = rope->scaling;
  a.original = rope->original;
  a.theta = rope->theta;
  a.factor = rope->factor;
  a.low = rope->turns_low;
  a.high = rope->turns_high;
  a.amplitude = rope->amplitude;
  return a;
}

PagedArgs paged_args(const epikv_cfg* c, const epikv_pool* pool, int32_t layer, int32_t chunk,
                     const int32_t* pt, int64_t ld_pt, const int32_t* n_cached,
                     const int32_t* n_new, int32_t* status) {
  PagedArgs a;
  char* base = (char*)pool->base + (int64_t)layer * pool->stride_layer;
  a.plane[0] = base;
  a.plane[1] = base + pool->stride_kv;
  a.s_page = pool->stride_page;
  a.n_pages = pool->n_pages;
  a.pt = pt;
  a.ld_pt = ld_pt;
  a.n_cached = n_cached;
  a.n_new = n_new;
  a.status = status;
  a.B = c->batch;
  a.C = chunk;
  a.H = c->n_kv_heads;
  a.d = c->head_dim;
  a.page_size = c->page_size;
  a.page_shift = -1;
  for (int sh = 0; sh <= 10; ++sh)
    if ((1 << sh) == c->page_size) a.page_shift = sh;
  a.row_bytes = row_bytes(c);
  a.max_tokens = slots_of(c, ld_pt);
  return a;
}

bool is_q4(const epikv_cfg* c) { return c->kv_format == EPIKV_KV_MXFP4; }

}  // namespace
}  // namespace epikv

using namespace epikv;

EPIKV_EXPORT int epikv_default_rope(epikv_rope_cfg* rope) {
  if (!rope) return EPIKV_EINVAL_NULL;
  rope->rotary_dim = 128;
  rope->layout = EPIKV_ROPE_HALF;
  rope->scaling = EPIKV_ROPE_PLAIN;
  rope->n_pos = 32768;
  rope->original = 8192;
  rope->theta = 10000.f;
  rope->factor = 1.f;
  rope->turns_low = 1.f;
  rope->turns_high = 4.f;
  rope->amplitude = 1.f;
  return EPIKV_OK;
}

EPIKV_EXPORT int epikv_check_rope(const epikv_rope_cfg* rope) { return check_rope_cfg(rope); }

EPIKV_EXPORT size_t epikv_rope_table_bytes(const epikv_rope_cfg* rope) {
  if (check_rope_cfg(rope)) return 0;
  return (size_t)rope->n_pos * (size_t)rope->rotary_dim * sizeof(float);
}

EPIKV_EXPORT int epikv_rope_table(const epikv_rope_cfg* rope, float* table, hipStream_t stream) {
  const int st = check_rope_cfg(rope);
  if (st) return st;
  if (!table) return EPIKV_EINVAL_NULL;
  if (!aligned16(table)) return EPIKV_EALIGN;
  return launched(launch_rope_table(table_args(rope, table), stream));
}

EPIKV_EXPORT int epikv_check_axes(const epikv_rope_cfg* rope, const epikv_axes* axes) {
  return check_axes(rope, axes);
}

EPIKV_EXPORT int epikv_rope_axes_table(const epikv_rope_cfg* rope, const epikv_axes* axes, float* table,
                                       hipStream_t stream) {
  const int st = check_axes(rope, axes);
  if (st) return st;
  if (!table) return EPIKV_EINVAL_NULL;
  if (!aligned16(table)) return EPIKV_EALIGN;
  if (axes->frequencies == EPIKV_AXES_SHARED)
    return launched(launch_rope_table(table_args(rope, table), stream));
  RopeAxesTableArgs a = {};
  a.t = table_args(rope, table);
  deal_pairs(axes, a.place, a.count);
  return launched(launch_rope_axes_table(a, stream));
}

namespace epikv {
namespace {

// What epikv_rope and epikv_rope_axes check alike (rope is checked), and their
// arguments but the positions.
template <class Args>
int prepare_rope(Args& a, const epikv_rope_cfg* rope, const float* table, int32_t dtype, int32_t batch,
                 int32_t chunk, int32_t n_heads, int32_t head_dim, const epikv_rows* x, const epikv_rows* y,
                 const int32_t* positions, int64_t ld_pos, int32_t* seq_status) {
  if (!table || !x || !y) return EPIKV_EINVAL_NULL;
  if (dtype != EPIKV_DTYPE_BF16 && dtype != EPIKV_DTYPE_FP32) return EPIKV_EINVAL_PARAM;
  if (batch < 1 || chunk < 1 || (int64_t)batch * chunk > INT32_MAX) return EPIKV_EINVAL_SHAPE;
  if (n_heads < 1 || n_heads > kMaxHeads) return EPIKV_EINVAL_SHAPE;
  if (head_dim < 16 || head_dim > 1024 || head_dim % 16 || rope->rotary_dim > head_dim)
    return EPIKV_EINVAL_SHAPE;
  if (!rope_fits((int64_t)batch * chunk, n_heads, head_dim)) return EPIKV_EINVAL_SHAPE;
  if (!aligned16(table)) return EPIKV_EALIGN;
  int st = check_rows(x);
  if (st) return st;
  st = check_out_rows(y, batch, chunk, n_heads, head_dim);
  if (st) return st;
  st = check_positions(positions, ld_pos, chunk);
  if (st) return st;
  st = check_alias(x, y, batch, chunk, n_heads, head_dim, dtype == EPIKV_DTYPE_FP32 ? 4 : 2);
  if (st) return st;
  a.x = rows_arg(x);
  a.y = rows_arg(y);
  a.B = batch;
  a.C = chunk;
  a.heads = n_heads;
  a.d = head_dim;
  a.fp32 = dtype == EPIKV_DTYPE_FP32;
  a.status = seq_status;
  return EPIKV_OK;
}

}  // namespace
}  // namespace epikv

EPIKV_EXPORT int epikv_rope(const epikv_rope_cfg* rope, const float* table, int32_t dtype,
                            int32_t batch, int32_t chunk, int32_t n_heads, int32_t head_dim,
                            const epikv_rows* x, const epikv_rows* y, const int32_t* positions,
                            int64_t ld_pos, int32_t transpose, int32_t* seq_status,
                            hipStream_t stream) {
  int st = check_rope_cfg(rope);
  if (st) return st;
  RopeArgs a;
  st = prepare_rope(a, rope, table, dtype, batch, chunk, n_heads, head_dim, x, y, positions, ld_pos, seq_status);
  if (st) return st;
  a.rope = rope_arg(rope, table, positions, ld_pos, transpose);
  return launched(launch_rope(a, stream));
}

EPIKV_EXPORT int epikv_rope_axes(const epikv_rope_cfg* rope, const epikv_axes* axes, const float* table,
                                 int32_t dtype, int32_t batch, int32_t chunk, int32_t n_heads,
                                 int32_t head_dim, const epikv_rows* x, const epikv_rows* y,
                                 const int32_t* positions, int64_t ld_pos, int32_t transpose,
                                 int32_t* seq_status, hipStream_t stream) {
  int st = check_axes(rope, axes);
  if (st) return st;
  RopeAxesArgs a;
  st = prepare_rope(a, rope, table, dtype, batch, chunk, n_heads, head_dim, x, y, positions, ld_pos, seq_status);
  if (st) return st;
  a.rope = rope_axes_arg(rope, axes, table, positions, ld_pos, transpose);
  return launched(launch_rope_axes(a, stream));
}

namespace epikv {
namespace {

// What epikv_append and epikv_append_axes check alike, and their arguments but
// the rotation.
template <class Args>
int prepare_append(Args& a, const epikv_cfg* cfg, const epikv_append_io* io) {
  if (!cfg || !io) return EPIKV_EINVAL_NULL;
  int st = check_paged(cfg, &io->pool, io->layer, io->chunk, io->page_table, io->ld_pt);
  if (st) return st;
  if (!io->n_cached) return EPIKV_EINVAL_NULL;
  const int B = cfg->batch, C = io->chunk, H = cfg->n_kv_heads, d = cfg->head_dim;
  st = check_rows(&io->k);
  if (st) return st;
  st = check_rows(&io->v);
  if (st) return st;
  if (io->rope) {
    st = check_rope_cfg(io->rope);
    if (st) return st;
    if (io->rope->rotary_dim > d) return EPIKV_EINVAL_SHAPE;
    if (!io->rope_table) return EPIKV_EINVAL_NULL;
    if (!aligned16(io->rope_table)) return EPIKV_EALIGN;
  }
  if (io->rope || io->pos) {
    st = check_positions(io->positions, io->ld_pos, C);
    if (st) return st;
  }
  if (io->pos && io->ld_s < 1) return EPIKV_EINVAL_SHAPE;
  if (io->q.base) {
    if (io->n_heads < 1 || io->n_heads > kMaxHeads) return EPIKV_EINVAL_SHAPE;
    st = check_rows(&io->q);
    if (st) return st;
    st = check_out_rows(&io->q_out, B, C, io->n_heads, d);
    if (st) return st;
    st = check_alias(&io->q, &io->q_out, B, C, io->n_heads, d, 2);
    if (st) return st;
    // (the launch reads keys and values while it writes the queries, in place or not)
    if (rows_meet(&io->q_out, io->n_heads, &io->k, H, B, C, d, 2) ||
        rows_meet(&io->q_out, io->n_heads, &io->v, H, B, C, d, 2))
      return EPIKV_EALIAS;
  }
  if (!append_fits((int64_t)B * C, H, io->q.base ? io->n_heads : 0, d)) return EPIKV_EINVAL_SHAPE;
  a = {};
  a.pg = paged_args(cfg, &io->pool, io->layer, C, io->page_table, io->ld_pt, io->n_cached,
                    io->n_new, io->seq_status);
  a.k = rows_arg(&io->k);
  a.v = rows_arg(&io->v);
  if (io->q.base) {
    a.q = rows_arg(&io->q);
    a.q_out = rows_arg(&io->q_out);
    a.heads = io->n_heads;
  }
  a.pos = io->pos;
  a.ld_s = io->ld_s;
  return EPIKV_OK;
}

}  // namespace
}  // namespace epikv

EPIKV_EXPORT int epikv_append(const epikv_cfg* cfg, const epikv_append_io* io,
                              hipStream_t stream) {
  AppendArgs a;
  const int st = prepare_append(a, cfg, io);
  if (st) return st;
  a.rope = rope_arg(io->rope, io->rope_table, io->positions, io->ld_pos, 0);
  return launched(launch_append(a, is_q4(cfg), stream));
}

EPIKV_EXPORT int epikv_append_axes(const epikv_cfg* cfg, const epikv_append_io* io, const epikv_axes* axes,
                                   const int32_t* ids, int64_t ld_ids, hipStream_t stream) {
  if (!cfg || !io || !axes || !io->rope) return EPIKV_EINVAL_NULL;
  AppendAxesArgs a;
  int st = prepare_append(a, cfg, io);
  if (st) return st;
  st = check_axes(io->rope, axes);
  if (st) return st;
  if (io->pos) {
    st = check_positions(ids, ld_ids, io->chunk);
    if (st) return st;
  }
  a.rope = rope_axes_arg(io->rope, axes, io->rope_table, io->positions, io->ld_pos, 0);
  a.rope.ids = ids;
  a.rope.ld_ids = ld_ids;
  return launched(launch_append_axes(a, is_q4(cfg), stream));
}

EPIKV_EXPORT int epikv_read(const epikv_cfg* cfg, const epikv_read_io* io, hipStream_t stream) {
  if (!cfg || !io) return EPIKV_EINVAL_NULL;
  int st = check_paged(cfg, &io->pool, io->layer, io->chunk, io->page_table, io->ld_pt);
  if (st) return st;
  if (!io->first || (!io->k.base && !io->v.base)) return EPIKV_EINVAL_NULL;
  const int B = cfg->batch, C = io->chunk, H = cfg->n_kv_heads, d = cfg->head_dim;
  for (const epikv_rows* x : {&io->k, &io->v}) {
    st = x->base ? check_out_rows(x, B, C, H, d) : EPIKV_OK;
    if (st) return st;
  }
  if (io->k.base && io->v.base && rows_meet(&io->k, H, &io->v, H, B, C, d, 2)) return EPIKV_EALIAS;
  if (!append_fits((int64_t)B * C, H, 0, d)) return EPIKV_EINVAL_SHAPE;
  ReadArgs a;
  a.pg = paged_args(cfg, &io->pool, io->layer, C, io->page_table, io->ld_pt, io->first, nullptr,
                    io->seq_status);
  a.k = rows_arg(&io->k);
  a.v = rows_arg(&io->v);
  return launched(launch_read(a, is_q4(cfg), stream));
}

namespace epikv {
namespace {

bool attend_fits(const epikv_cfg* cfg, int32_t chunk, int32_t n_heads) {
  return !check_cfg(cfg) && chunk >= 1 && chunk <= kMaxChunk && heads_fit(chunk, cfg->n_kv_heads, n_heads) &&
         (int64_t)cfg->batch * chunk <= INT32_MAX;
}

int32_t watched(int32_t watch, int32_t chunk) { return watch ? std::min(watch, chunk) : chunk; }

struct Span {
  const void* p;
  size_t n;
};

// What epikv_attend and epikv_attend_weigh check alike, and the arguments.
// `spans` receives six arguments that nothing written besides may overlap.
int prepare_attend(AttendArgs& a, const epikv_cfg* cfg, const epikv_attend_io* io, Span* spans) {
  int st = check_paged(cfg, &io->pool, io->layer, io->chunk, io->page_table, io->ld_pt);
  if (st) return st;
  if (!io->n_cached) return EPIKV_EINVAL_NULL;
  const int B = cfg->batch, C = io->chunk, H = cfg->n_kv_heads, d = cfg->head_dim;
  if (!heads_fit(C, H, io->n_heads)) return EPIKV_EINVAL_SHAPE;
  if (!(io->scale >= 0.f) || !isfinite(io->scale)) return EPIKV_EINVAL_PARAM;
  st = check_rows(&io->q);
  if (st) return st;
  st = check_out_rows(&io->out, B, C, io->n_heads, d);
  if (st) return st;
  if (rows_meet(&io->out, io->n_heads, &io->q, io->n_heads, B, C, d, 2)) return EPIKV_EALIAS;
  spans[0] = {io->q.base, rows_span(&io->q, B, C, io->n_heads, d, 2)};
  spans[1] = {io->out.base, rows_span(&io->out, B, C, io->n_heads, d, 2)};
  spans[2] = {io->lse, io->lse ? (size_t)B * io->n_heads * C * 4 : 0};
  spans[3] = {io->page_table, 4 * (size_t)B * (size_t)io->ld_pt};
  spans[4] = {io->n_cached, 4 * (size_t)B};
  spans[5] = {io->n_new, io->n_new ? 4 * (size_t)B : 0};
  memset(&a, 0, sizeof(a));
  a.pg = paged_args(cfg, &io->pool, io->layer, C, io->page_table, io->ld_pt, io->n_cached,
                    io->n_new, io->seq_status);
  a.q = rows_arg(&io->q);
  a.out = rows_arg(&io->out);
  a.lse = io->lse;
  a.heads = io->n_heads;
  a.G = io->n_heads / H;
  a.R = C * a.G;
  const float scale = io->scale > 0.f ? io->scale : 1.f / sqrtf((float)d);
  a.scale2 = scale * 1.4426950408889634f;
  return EPIKV_OK;
}

bool meets(const void* p, size_t n, const Span* spans, int n_spans) {
  for (int i = 0; i < n_spans; ++i)
    if (spans[i].n && overlap(p, n, spans[i].p, spans[i].n)) return true;
  return false;
}

int check_workspace(const epikv_attend_io* io, size_t need, const Span* spans, int n_spans) {
  if (!need) return EPIKV_OK;
  if (!io->workspace || io->workspace_bytes < need) return EPIKV_EWORKSPACE;
  if (!aligned16(io->workspace)) return EPIKV_EALIGN;
  return meets(io->workspace, need, spans, n_spans) ? EPIKV_EALIAS : EPIKV_OK;
}

}  // namespace
}  // namespace epikv

EPIKV_EXPORT size_t epikv_attend_workspace_bytes(const epikv_cfg* cfg, int32_t chunk,
                                                 int32_t n_heads) {
  if (!attend_fits(cfg, chunk, n_heads)) return 0;
  return attend_workspace(cfg->batch, chunk, cfg->n_kv_heads, n_heads, cfg->head_dim);
}

EPIKV_EXPORT int epikv_attend(const epikv_cfg* cfg, const epikv_attend_io* io,
                              hipStream_t stream) {
  if (!cfg || !io) return EPIKV_EINVAL_NULL;
  AttendArgs a;
  Span spans[6];
  int st = prepare_attend(a, cfg, io, spans);
  if (st) return st;
  const size_t need = attend_workspace(cfg->batch, io->chunk, cfg->n_kv_heads, io->n_heads, cfg->head_dim);
  st = check_workspace(io, need, spans, 5);
  if (st) return st;
  return launched(launch_attend(a, is_q4(cfg), io->workspace, stream));
}

EPIKV_EXPORT size_t epikv_attend_weigh_workspace_bytes(const epikv_cfg* cfg, int32_t chunk, int32_t n_heads,
                                                       int64_t ld_pt, int32_t watch) {
  if (!attend_fits(cfg, chunk, n_heads) || ld_pt < 1 || watch < 0) return 0;
  return attend_weigh_workspace(cfg->batch, chunk, cfg->n_kv_heads, n_heads, cfg->head_dim,
                                slots_of(cfg, ld_pt), watched(watch, chunk));
}

EPIKV_EXPORT int epikv_attend_weigh(const epikv_cfg* cfg, const epikv_attend_io* io,
                                    const epikv_weigh_io* weigh, hipStream_t stream) {
  if (!cfg || !io || !weigh) return EPIKV_EINVAL_NULL;
  AttendArgs a;
  Span spans[9];
  int st = prepare_attend(a, cfg, io, spans);
  if (st) return st;
  if (!weigh->weights) return EPIKV_EINVAL_NULL;
  if (weigh->ld_s < 1 || weigh->watch < 0) return EPIKV_EINVAL_SHAPE;
  if (!(weigh->keep_old >= 0.f && weigh->keep_old <= 1.f) || !(weigh->keep_new >= 0.f && weigh->keep_new <= 1.f) ||
      !(weigh->gain > 0.f) || !isfinite(weigh->gain))
    return EPIKV_EINVAL_PARAM;
  if ((uintptr_t)weigh->weights % 4 || (uintptr_t)weigh->old % 4) return EPIKV_EALIGN;
  const int B = cfg->batch;
  const size_t n_sums = 4 * (size_t)B * (size_t)weigh->ld_s;
  spans[6] = {io->seq_status, io->seq_status ? 4 * (size_t)B : 0};
  if (meets(weigh->weights, n_sums, spans, 7)) return EPIKV_EALIAS;
  if (weigh->old && weigh->old != weigh->weights) {
    if (overlap(weigh->weights, n_sums, weigh->old, n_sums)) return EPIKV_EALIAS;
    // (what the call writes before it reads them)
    if (overlap(spans[1].p, spans[1].n, weigh->old, n_sums) ||
        (spans[2].n && overlap(spans[2].p, spans[2].n, weigh->old, n_sums)))
      return EPIKV_EALIAS;
  }
  spans[7] = {weigh->weights, n_sums};
  spans[8] = {weigh->old, weigh->old ? n_sums : 0};
  const int watch = watched(weigh->watch, io->chunk);
  const size_t need = attend_weigh_workspace(B, io->chunk, cfg->n_kv_heads, io->n_heads, cfg->head_dim,
                                             a.pg.max_tokens, watch);
  st = check_workspace(io, need, spans, 9);
  if (st) return st;
  WeighArgs w;
  w.old = weigh->old;
  w.weights = weigh->weights;
  w.ld_s = weigh->ld_s;
  w.keep_old = weigh->old ? weigh->keep_old : 0.f;
  w.keep_new = weigh->old ? weigh->keep_new : 0.f;
  w.gain = weigh->gain;
  w.watch = watch;
  return launched(launch_attend_weigh(a, w, is_q4(cfg), io->workspace, stream));
}
