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
  a.max_tokens = (int32_t)std::min<int64_t>(std::min<int64_t>(ld_pt, INT32_MAX) * c->page_size,
                                            kMaxTokens);
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
  return launched(launch_rope_table(a, stream));
}

EPIKV_EXPORT int epikv_rope(const epikv_rope_cfg* rope, const float* table, int32_t dtype,
                            int32_t batch, int32_t chunk, int32_t n_heads, int32_t head_dim,
                            const epikv_rows* x, const epikv_rows* y, const int32_t* positions,
                            int64_t ld_pos, int32_t transpose, int32_t* seq_status,
                            hipStream_t stream) {
  int st = check_rope_cfg(rope);
  if (st) return st;
  if (!table || !x || !y) return EPIKV_EINVAL_NULL;
  if (dtype != EPIKV_DTYPE_BF16 && dtype != EPIKV_DTYPE_FP32) return EPIKV_EINVAL_PARAM;
  if (batch < 1 || chunk < 1 || (int64_t)batch * chunk > INT32_MAX) return EPIKV_EINVAL_SHAPE;
  if (n_heads < 1 || n_heads > kMaxHeads) return EPIKV_EINVAL_SHAPE;
  if (head_dim < 16 || head_dim > 1024 || head_dim % 16 || rope->rotary_dim > head_dim)
    return EPIKV_EINVAL_SHAPE;
  if (!rope_fits((int64_t)batch * chunk, n_heads, head_dim)) return EPIKV_EINVAL_SHAPE;
  if (!aligned16(table)) return EPIKV_EALIGN;
  st = check_rows(x);
  if (st) return st;
  st = check_out_rows(y, batch, chunk, n_heads, head_dim);
  if (st) return st;
  st = check_positions(positions, ld_pos, chunk);
  if (st) return st;
  st = check_alias(x, y, batch, chunk, n_heads, head_dim, dtype == EPIKV_DTYPE_FP32 ? 4 : 2);
  if (st) return st;
  RopeArgs a;
  a.x = rows_arg(x);
  a.y = rows_arg(y);
  a.rope = rope_arg(rope, table, positions, ld_pos, transpose);
  a.B = batch;
  a.C = chunk;
  a.heads = n_heads;
  a.d = head_dim;
  a.fp32 = dtype == EPIKV_DTYPE_FP32;
  a.status = seq_status;
  return launched(launch_rope(a, stream));
}

EPIKV_EXPORT int epikv_append(const epikv_cfg* cfg, const epikv_append_io* io,
                              hipStream_t stream) {
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
  AppendArgs a;
  memset(&a, 0, sizeof(a));
  a.pg = paged_args(cfg, &io->pool, io->layer, C, io->page_table, io->ld_pt, io->n_cached,
                    io->n_new, io->seq_status);
  a.rope = rope_arg(io->rope, io->rope_table, io->positions, io->ld_pos, 0);
  a.k = rows_arg(&io->k);
  a.v = rows_arg(&io->v);
  if (io->q.base) {
    a.q = rows_arg(&io->q);
    a.q_out = rows_arg(&io->q_out);
    a.heads = io->n_heads;
  }
  a.pos = io->pos;
  a.ld_s = io->ld_s;
  return launched(launch_append(a, is_q4(cfg), stream));
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

EPIKV_EXPORT size_t epikv_attend_workspace_bytes(const epikv_cfg* cfg, int32_t chunk,
                                                 int32_t n_heads) {
  if (check_cfg(cfg) || chunk < 1 || chunk > kMaxChunk ||
      !heads_fit(chunk, cfg->n_kv_heads, n_heads) || (int64_t)cfg->batch * chunk > INT32_MAX)
    return 0;
  return attend_workspace(cfg->batch, chunk, cfg->n_kv_heads, n_heads, cfg->head_dim);
}

EPIKV_EXPORT int epikv_attend(const epikv_cfg* cfg, const epikv_attend_io* io,
                              hipStream_t stream) {
  if (!cfg || !io) return EPIKV_EINVAL_NULL;
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
  const size_t n_out = rows_span(&io->out, B, C, io->n_heads, d, 2);
  const size_t n_q = rows_span(&io->q, B, C, io->n_heads, d, 2);
  const size_t need = attend_workspace(B, C, H, io->n_heads, d);
  if (need) {
    if (!io->workspace || io->workspace_bytes < need) return EPIKV_EWORKSPACE;
    if (!aligned16(io->workspace)) return EPIKV_EALIGN;
    const size_t n_lse = io->lse ? (size_t)B * io->n_heads * C * 4 : 0;
    if (overlap(io->workspace, need, io->q.base, n_q) ||
        overlap(io->workspace, need, io->out.base, n_out) ||
        (io->lse && overlap(io->workspace, need, io->lse, n_lse)) ||
        overlap(io->workspace, need, io->page_table, 4 * (size_t)B * (size_t)io->ld_pt) ||
        overlap(io->workspace, need, io->n_cached, 4 * (size_t)B))
      return EPIKV_EALIAS;
  }
  AttendArgs a;
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
  return launched(launch_attend(a, is_q4(cfg), io->workspace, stream));
}
