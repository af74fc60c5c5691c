// The C ABI's operators over a pool of pages that many sequences share
// (include/crf.h): validation and launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/crf.h"
#include "context.hpp"
#include "paged.hpp"
#include "paged_checks.hpp"

using namespace crf;

extern "C" {

crf_status crf_rope_init(crf_rope *out, int32_t layout, int32_t rotary_dim, double theta,
                         const crf_rope_scaling *scaling) {
  const char *what = "crf_rope_init";
  if (!out) return fail(nullptr, CRF_ERR_INVALID_ARG, "%s: out is NULL", what);
  if (layout != CRF_ROPE_HALF && layout != CRF_ROPE_INTERLEAVED)
    return fail(nullptr, CRF_ERR_INVALID_ARG, "%s: unknown layout %d", what, layout);
  if (rotary_dim < 0 || rotary_dim > 128 || rotary_dim % 16)
    return fail(nullptr, CRF_ERR_UNSUPPORTED, "%s: rotary_dim %d is no multiple of 16 in [0, 128]", what, rotary_dim);
  if (!(theta > 0) || !isfinite(theta)) return fail(nullptr, CRF_ERR_SHAPE, "%s: theta must be positive", what);
  const crf_rope_scaling none = {CRF_ROPE_NONE, 1.0, 0, 0, 0, 0};
  const crf_rope_scaling &sc = scaling ? *scaling : none;
  if (sc.kind < CRF_ROPE_NONE || sc.kind > CRF_ROPE_PARTS)
    return fail(nullptr, CRF_ERR_INVALID_ARG, "%s: unknown scaling %d", what, sc.kind);
  if (sc.kind != CRF_ROPE_NONE && (!(sc.factor > 0) || !isfinite(sc.factor)))
    return fail(nullptr, CRF_ERR_SHAPE, "%s: the scaling factor must be positive", what);
  if (!(sc.mscale >= 0) || !isfinite((float)sc.mscale))
    return fail(nullptr, CRF_ERR_SHAPE, "%s: mscale must be finite and >= 0", what);
  const double low = sc.low_turns > 0 ? sc.low_turns : 1.0, high = sc.high_turns > 0 ? sc.high_turns : 32.0;
  if (sc.kind == CRF_ROPE_PARTS && (!(sc.original_len >= 1) || !(high > low)))
    return fail(nullptr, CRF_ERR_SHAPE, "%s: original_len must be >= 1 and high_turns > low_turns", what);
  *out = crf_rope{};
  out->layout = layout;
  out->rotary_dim = rotary_dim;
  out->mscale = 1.f;
  if (sc.kind == CRF_ROPE_PARTS && sc.factor > 1) out->mscale = (float)(0.1 * log(sc.factor) + 1.0);
  if (sc.mscale > 0) out->mscale = (float)sc.mscale;
  const double r = rotary_dim;
  if (sc.kind == CRF_ROPE_BASE && rotary_dim > 0) theta *= pow(sc.factor, r / (r - 2));
  if (!isfinite(theta)) return fail(nullptr, CRF_ERR_SHAPE, "%s: the scaled theta is not finite", what);
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = pow(theta, -2.0 * i / r);
    if (sc.kind == CRF_ROPE_LINEAR) f /= sc.factor;
    if (sc.kind == CRF_ROPE_PARTS) {
      const double turns = f * sc.original_len / (2 * M_PI);
      const double keep = fmin(1.0, fmax(0.0, (turns - low) / (high - low)));
      f *= (1 - keep) / sc.factor + keep;
    }
    if (!isfinite(f)) return fail(nullptr, CRF_ERR_SHAPE, "%s: the frequency of pair %d is not finite", what, i);
    out->freq[i] = f;
  }
  return CRF_OK;
}

crf_status crf_rope_append(crf_context *ctx, const crf_rope *rope, const crf_seq_batch *batch,
                           const int32_t *positions, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride,
                           const crf_page_pool *pool, int32_t layer, void *stream) {
  RopeAppend p{};
  bool any = false;
  crf_status st = prepare_append(ctx, "crf_rope_append", rope, batch, positions, q, q_stride, k, k_stride, v, v_stride,
                                 q_out, q_out_stride, pool, layer, p, any);
  if (st != CRF_OK || !any) return st;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_rope_append((hipStream_t)stream, ctx->dims.dtype == CRF_F32, p));
  return CRF_OK;
}

crf_status crf_paged_attention(crf_context *ctx, const crf_seq_batch *batch, const void *q, int64_t q_stride,
                               const crf_page_pool *pool, int32_t layer, float scale, int32_t window, void *out,
                               int64_t out_stride, float *lse, void *stream) {
  PagedAttn p{};
  bool any = false;
  crf_status st = prepare_attention(ctx, "crf_paged_attention", batch, q, q_stride, pool, layer, scale, window, out,
                                    out_stride, lse, p, any);
  if (st != CRF_OK || !any) return st;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_ATTN,
         launch_paged_attn((hipStream_t)stream, ctx->dims.dtype == CRF_F32, p));
  return CRF_OK;
}

crf_status crf_pages_copy(crf_context *ctx, const crf_page_pool *from, int32_t from_l0, const crf_page_pool *to,
                          int32_t to_l0, int32_t h, int32_t n, const int32_t *src, const int32_t *dst, void *stream) {
  const char *what = "crf_pages_copy";
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_pool(ctx, from, what);
  if (st == CRF_OK) st = check_pool(ctx, to, what);
  if (st == CRF_OK) st = check_layers(ctx, from_l0, h, what);
  if (st == CRF_OK) st = check_layers(ctx, to_l0, h, what);
  if (st == CRF_OK) st = check_list(ctx, n, src, dst, INT32_MAX, what);
  if (st == CRF_OK) st = check_copy(ctx, *from, h, what);
  if (st != CRF_OK) return st;
  if (from->page_size != to->page_size) return fail(ctx, CRF_ERR_SHAPE, "%s: the pools' page sizes differ", what);
  if (n == 0 || h == 0) return CRF_OK;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_pages_copy((hipStream_t)stream, device_pools(ctx, *from, from_l0), device_pools(ctx, *to, to_l0), h,
                           (int)page_bytes(ctx, *from), n, src, dst, ctx->d_err));
  return CRF_OK;
}

crf_status crf_pages_fork(crf_context *ctx, const crf_page_pool *pool, const crf_page_map *map, int32_t n,
                          const int32_t *parents, const int32_t *children, void *stream) {
  const char *what = "crf_pages_fork";
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_map_pool(ctx, map, pool, what);
  if (st == CRF_OK) st = check_list(ctx, n, parents, children, PAGED_MAX_LIST, what);
  if (st == CRF_OK) st = check_copy(ctx, *pool, ctx->dims.n_layers, what);
  if (st != CRF_OK) return st;
  if (n == 0) return CRF_OK;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_pages_fork((hipStream_t)stream, device_map(ctx, *map), device_pools(ctx, *pool, 0), ctx->dims.n_layers,
                           (int)page_bytes(ctx, *pool), n, parents, children, fork_state(ctx)));
  return CRF_OK;
}

crf_status crf_pages_extend(crf_context *ctx, const crf_page_map *map, const int32_t *n_new, void *stream) {
  const char *what = "crf_pages_extend";
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_map(ctx, map, what);
  if (st == CRF_OK) st = check_list(ctx, map->n_seqs, n_new, n_new, PAGED_MAX_LIST, what);
  if (st != CRF_OK || map->n_seqs == 0) return st;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_pages_extend((hipStream_t)stream, device_map(ctx, *map), n_new));
  return CRF_OK;
}

crf_status crf_pages_free(crf_context *ctx, const crf_page_map *map, int32_t n, const int32_t *seqs, void *stream) {
  const char *what = "crf_pages_free";
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_map(ctx, map, what);
  if (st == CRF_OK) st = check_list(ctx, n, seqs, seqs, INT32_MAX, what);
  if (st != CRF_OK || n == 0) return st;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_pages_free((hipStream_t)stream, device_map(ctx, *map), n, seqs));
  return CRF_OK;
}

crf_status crf_pages_compact(crf_context *ctx, const crf_page_pool *pool, const crf_page_map *map,
                             const crf_page_map *map_out, int32_t *remap, int32_t *counts, void *stream) {
  const char *what = "crf_pages_compact";
  crf_status st = check_context(ctx, what);
  if (st == CRF_OK) st = check_map_pool(ctx, map, pool, what);
  if (st == CRF_OK) st = check_map(ctx, map_out, what);
  if (st == CRF_OK) st = check_copy(ctx, *pool, ctx->dims.n_layers, what);
  if (st != CRF_OK) return st;
  if (map_out->n_pages != map->n_pages || map_out->page_size != map->page_size || map_out->n_seqs != map->n_seqs ||
      map_out->max_pages < map->max_pages)
    return fail(ctx, CRF_ERR_SHAPE, "%s: the maps differ in pages, sequences or width", what);
  if (map_out->block_tables == map->block_tables && map_out->table_stride != map->table_stride)
    return fail(ctx, CRF_ERR_SHAPE, "%s: one table with two strides", what);
  if (!remap || !counts || !aligned4(remap) || !aligned4(counts))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: remap or counts NULL or misaligned", what);
  if (!ctx->paged_part || ctx->paged_part_floats < map->n_pages)
    return fail(ctx, CRF_ERR_WORKSPACE, "%s: no room for the moves of %d pages", what, map->n_pages);
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_pages_compact((hipStream_t)stream, device_map(ctx, *map), device_map(ctx, *map_out),
                              device_pools(ctx, *pool, 0), ctx->dims.n_layers, (int)page_bytes(ctx, *pool), remap,
                              (int32_t *)ctx->paged_part, counts));
  return CRF_OK;
}

}  // extern "C"
