// What the entry points over a page pool check before they launch, and the kernels' view of
// their arguments (host side).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/crf.h"
#include "context.hpp"
#include "paged.hpp"

namespace crf {
namespace {

constexpr int64_t MAX_KEYS = (int64_t)1 << 30;  // tokens that a block table may hold; rows, sequences x query heads

bool aligned4(const void *p) { return ((uintptr_t)p & 3u) == 0; }

const char *zeros(const crf_context *ctx) { return ctx->paged_ws; }
int32_t *fork_state(const crf_context *ctx) { return (int32_t *)(ctx->paged_ws + PAGED_ZERO_BYTES); }
unsigned *tickets(const crf_context *ctx) { return (unsigned *)(fork_state(ctx) + PAGED_MAX_LIST); }

int64_t page_bytes(const crf_context *ctx, const crf_page_pool &p) {
  return (int64_t)ctx->dims.n_kv_heads * p.page_size * ctx->dims.head_dim * (int64_t)ctx->esz;
}

// The context and the device that its buffers are on.
crf_status check_context(crf_context *ctx, const char *what) {
  if (!ctx) return fail(nullptr, CRF_ERR_INVALID_ARG, "%s: context is NULL", what);
  int dev = -1;
  HIP_TRY(ctx, hipGetDevice(&dev));
  if (dev != ctx->device)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: the current device is %d, the context's %d", what, dev, ctx->device);
  return CRF_OK;
}

crf_status check_pool(crf_context *ctx, const crf_page_pool *p, const char *what) {
  if (!p) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: the page pool is NULL", what);
  const crf_model_dims &d = ctx->dims;
  if (p->page_size < 1 || p->n_pages < 0)
    return fail(ctx, CRF_ERR_SHAPE, "%s: page_size must be >= 1 and n_pages >= 0", what);
  if (page_bytes(ctx, *p) >= (int64_t)1 << 30)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: a page of 1 GiB or more", what);
  if (p->page_stride < (int64_t)d.n_kv_heads * p->page_size * d.head_dim)
    return fail(ctx, CRF_ERR_SHAPE, "%s: page_stride %lld < n_kv_heads*page_size*head_dim", what,
                (long long)p->page_stride);
  if (p->page_stride > INT64_MAX / 64 / (p->n_pages + 1) || p->layer_stride < p->n_pages * p->page_stride)
    return fail(ctx, CRF_ERR_SHAPE, "%s: layer_stride %lld < n_pages*page_stride", what, (long long)p->layer_stride);
  if (!p->k_pool || !p->v_pool) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: k_pool and v_pool must be non-NULL", what);
  if (!aligned16(p->k_pool) || !aligned16(p->v_pool) || p->page_stride % 8 || p->layer_stride % 8)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: pools must be 16-byte aligned with strides multiple of 8", what);
  return CRF_OK;
}

crf_status check_layers(crf_context *ctx, int32_t l0, int32_t h, const char *what) {
  if (l0 < 0 || h < 0 || (int64_t)l0 + h > ctx->dims.n_layers)
    return fail(ctx, CRF_ERR_RANGE, "%s: layers [%d, %d+%d) outside [0, %d)", what, l0, l0, h, ctx->dims.n_layers);
  return CRF_OK;
}

crf_status check_batch(crf_context *ctx, const crf_seq_batch *b, const crf_page_pool &pool, const char *what) {
  if (!b) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: the batch is NULL", what);
  if (b->n_seqs < 0 || b->n_rows < 0 || b->max_new < 0 || b->max_pages < 0 || b->table_stride < b->max_pages)
    return fail(ctx, CRF_ERR_SHAPE, "%s: n_seqs, n_rows, max_new, max_pages >= 0 and table_stride >= max_pages", what);
  if ((int64_t)b->max_pages * pool.page_size > MAX_KEYS)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: block tables of more than 2^30 tokens", what);
  if ((int64_t)b->n_rows * ctx->dims.n_q_heads > MAX_KEYS)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: more than 2^30 rows x query heads", what);
  if ((int64_t)b->n_seqs * ctx->dims.n_q_heads > MAX_KEYS)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: more than 2^30 sequences x query heads", what);
  if (b->n_seqs == 0 || b->n_rows == 0) return CRF_OK;
  if (!b->row_start || !b->length || !b->block_tables)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: row_start, length and block_tables must be non-NULL", what);
  if (!aligned4(b->row_start) || !aligned4(b->length) || !aligned4(b->block_tables))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: row_start, length or block_tables misaligned", what);
  return CRF_OK;
}

// A tensor of rows [n_rows][heads * head_dim], ld elements apart.
crf_status check_rows(crf_context *ctx, const void *t, int64_t ld, int heads, const char *name, const char *what) {
  if (!t || !aligned16(t)) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: %s NULL or misaligned", what, name);
  if (ld < (int64_t)heads * ctx->dims.head_dim)
    return fail(ctx, CRF_ERR_SHAPE, "%s: %s's rows overlap (stride %lld)", what, name, (long long)ld);
  if ((ld * (int64_t)ctx->esz) % 16)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: %s's row stride is no multiple of 16 bytes", what, name);
  return CRF_OK;
}

// In place means the same rows: with another stride a row of the output lies on rows of
// the queries that other workgroups have yet to read.
crf_status check_in_place(crf_context *ctx, const crf_seq_batch &b, const void *q, int64_t q_ld, const void *out,
                          int64_t out_ld, const char *what) {
  if (q == out && q_ld != out_ld && b.n_rows > 1)
    return fail(ctx, CRF_ERR_SHAPE, "%s: in place with two strides (%lld, %lld)", what, (long long)q_ld,
                (long long)out_ld);
  return CRF_OK;
}

PagedBatch device_batch(const crf_context *ctx, const crf_seq_batch &b, const crf_page_pool &pool, int layer) {
  PagedBatch d;
  d.row_start = b.row_start;
  d.length = b.length;
  d.tables = b.block_tables;
  d.table_stride = b.table_stride;
  d.n_seqs = b.n_seqs;
  d.n_rows = b.n_rows;
  d.max_new = b.max_new > 0 && b.max_new < b.n_rows ? b.max_new : b.n_rows;
  d.max_pages = b.max_pages;
  d.page_size = pool.page_size;
  d.n_pages = pool.n_pages;
  d.ps_div = fast_div(pool.page_size);
  d.page_bytes = pool.page_stride * (int64_t)ctx->esz;
  d.k = (char *)pool.k_pool + layer * pool.layer_stride * (int64_t)ctx->esz;
  d.v = (char *)pool.v_pool + layer * pool.layer_stride * (int64_t)ctx->esz;
  d.err = ctx->d_err;
  return d;
}

crf_status check_map(crf_context *ctx, const crf_page_map *m, const char *what) {
  if (!m) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: the page map is NULL", what);
  if (m->n_pages < 0 || m->page_size < 1 || m->n_seqs < 0 || m->max_pages < 0 || m->table_stride < m->max_pages)
    return fail(ctx, CRF_ERR_SHAPE,
                "%s: page_size >= 1, n_pages, n_seqs, max_pages >= 0 and table_stride >= max_pages", what);
  if (m->n_pages > PAGED_MAX_PAGES || m->n_seqs > PAGED_MAX_LIST || m->max_pages > PAGED_MAX_PAGES ||
      (int64_t)m->max_pages * m->page_size > MAX_KEYS)
    return fail(ctx, CRF_ERR_UNSUPPORTED,
                "%s: a page map holds at most %d pages, %d sequences and 2^30 tokens a sequence", what,
                PAGED_MAX_PAGES, PAGED_MAX_LIST);
  if (!m->refs || !m->block_tables || !m->lengths)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: refs, block_tables and lengths must be non-NULL", what);
  if (!aligned4(m->refs) || !aligned4(m->block_tables) || !aligned4(m->lengths))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: refs, block_tables or lengths misaligned", what);
  return CRF_OK;
}

crf_status check_map_pool(crf_context *ctx, const crf_page_map *m, const crf_page_pool *pool, const char *what) {
  crf_status st = check_map(ctx, m, what);
  if (st == CRF_OK) st = check_pool(ctx, pool, what);
  if (st != CRF_OK) return st;
  if (m->n_pages != pool->n_pages || m->page_size != pool->page_size)
    return fail(ctx, CRF_ERR_SHAPE, "%s: the map's pages are not the pool's", what);
  return CRF_OK;
}

// A list of n sequences or pages.
crf_status check_list(crf_context *ctx, int32_t n, const int32_t *a, const int32_t *b, int32_t most, const char *what) {
  if (n < 0) return fail(ctx, CRF_ERR_SHAPE, "%s: a negative count", what);
  if (n > most) return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: at most %d at a time", what, most);
  if (n > 0 && (!a || !b || !aligned4(a) || !aligned4(b)))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: a list is NULL or misaligned", what);
  return CRF_OK;
}

PageMap device_map(const crf_context *ctx, const crf_page_map &m) {
  return PageMap{m.refs,    m.block_tables, m.lengths, m.table_stride, m.n_pages, m.page_size,
                 m.n_seqs, m.max_pages,    ctx->d_err};
}

PagePools device_pools(const crf_context *ctx, const crf_page_pool &p, int layer) {
  const int64_t e = (int64_t)ctx->esz, at = layer * p.layer_stride * e;
  return PagePools{(char *)p.k_pool + at, (char *)p.v_pool + at, p.layer_stride * e, p.page_stride * e, p.n_pages};
}

// A pair's 16-byte chunks are counted in 31 bits.
crf_status check_copy(crf_context *ctx, const crf_page_pool &p, int layers, const char *what) {
  if (page_bytes(ctx, p) / 16 * 2 * layers >= (int64_t)1 << 30)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: a page of all layers reaches 16 GiB", what);
  return CRF_OK;
}

// The checks of an append and what its kernel is given; any: there is something to do.
crf_status prepare_append(crf_context *ctx, const char *what, const crf_rope *rope, const crf_seq_batch *batch,
                          const int32_t *positions, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                          const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride, const crf_page_pool *pool,
                          int32_t layer, RopeAppend &p, bool &any) {
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_pool(ctx, pool, what);
  if (st == CRF_OK) st = check_layers(ctx, layer, 1, what);
  if (st == CRF_OK) st = check_batch(ctx, batch, *pool, what);
  if (st != CRF_OK) return st;
  const crf_model_dims &d = ctx->dims;
  if (!rope) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: rope is NULL", what);
  if (rope->layout != CRF_ROPE_HALF && rope->layout != CRF_ROPE_INTERLEAVED)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: unknown layout %d", what, rope->layout);
  if (rope->rotary_dim < 0 || rope->rotary_dim > d.head_dim || rope->rotary_dim % 16)
    return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: rotary_dim %d is no multiple of 16 in [0, head_dim]", what,
                rope->rotary_dim);
  if (batch->n_seqs == 0 || batch->n_rows == 0) return CRF_OK;
  if ((q == nullptr) != (q_out == nullptr))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: q and q_out are given together or not at all", what);
  if (q) {
    if ((st = check_rows(ctx, q, q_stride, d.n_q_heads, "q", what)) != CRF_OK) return st;
    if ((st = check_rows(ctx, q_out, q_out_stride, d.n_q_heads, "q_out", what)) != CRF_OK) return st;
    if ((st = check_in_place(ctx, *batch, q, q_stride, q_out, q_out_stride, what)) != CRF_OK) return st;
  }
  if ((st = check_rows(ctx, k, k_stride, d.n_kv_heads, "k", what)) != CRF_OK) return st;
  if ((st = check_rows(ctx, v, v_stride, d.n_kv_heads, "v", what)) != CRF_OK) return st;
  if (!aligned4(positions)) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: positions misaligned", what);
  p.b = device_batch(ctx, *batch, *pool, layer);
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_out = q_out;
  p.q_ld = q_stride;
  p.k_ld = k_stride;
  p.v_ld = v_stride;
  p.qo_ld = q_out_stride;
  p.positions = positions;
  p.nq = q ? d.n_q_heads : 0;
  p.nkv = d.n_kv_heads;
  p.hd = d.head_dim;
  p.rotary_dim = rope->rotary_dim;
  p.interleaved = rope->layout == CRF_ROPE_INTERLEAVED;
  p.mscale = rope->mscale;
  for (int i = 0; i < rope->rotary_dim / 2; ++i) p.turns[i] = rope->freq[i] / (2 * M_PI);
  any = true;
  return CRF_OK;
}

// The same of attention over the pages.
crf_status prepare_attention(crf_context *ctx, const char *what, const crf_seq_batch *batch, const void *q,
                             int64_t q_stride, const crf_page_pool *pool, int32_t layer, float scale, int32_t window,
                             void *out, int64_t out_stride, float *lse, PagedAttn &p, bool &any) {
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_pool(ctx, pool, what);
  if (st == CRF_OK) st = check_layers(ctx, layer, 1, what);
  if (st == CRF_OK) st = check_batch(ctx, batch, *pool, what);
  if (st != CRF_OK) return st;
  const crf_model_dims &d = ctx->dims;
  if (!(scale >= 0.f) || !isfinite(1.45f * scale))
    return fail(ctx, CRF_ERR_SHAPE, "%s: scale must be finite and >= 0 (0: 1/sqrt(head_dim))", what);
  if (window < 0) return fail(ctx, CRF_ERR_SHAPE, "%s: window must be >= 0 (0: every key)", what);
  if (batch->n_seqs == 0 || batch->n_rows == 0) return CRF_OK;
  if ((st = check_rows(ctx, q, q_stride, d.n_q_heads, "q", what)) != CRF_OK) return st;
  if ((st = check_rows(ctx, out, out_stride, d.n_q_heads, "out", what)) != CRF_OK) return st;
  if ((st = check_in_place(ctx, *batch, q, q_stride, out, out_stride, what)) != CRF_OK) return st;
  if (!aligned4(lse)) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: lse misaligned", what);
  p.b = device_batch(ctx, *batch, *pool, layer);
  p.q = q;
  p.out = out;
  p.q_ld = q_stride;
  p.out_ld = out_stride;
  p.lse = lse;
  p.nq = d.n_q_heads;
  p.nkv = d.n_kv_heads;
  p.hd = d.head_dim;
  p.scale_log2 = (float)(1.4426950408889634 * (scale > 0.f ? (double)scale : 1.0 / sqrt((double)d.head_dim)));
  p.window = window;
  p.part = ctx->paged_part;
  p.part_floats = ctx->paged_part_floats;
  p.tickets = tickets(ctx);
  p.zeros = zeros(ctx);
  p.n_cu = ctx->n_cu;
  any = true;
  return CRF_OK;
}

}  // namespace
}  // namespace crf
