// The C ABI's further operators of a server's step (include/crf.h): norms with the rotary
// append, attention with sinks, attention over shared prefixes, log probabilities.
#include <hip/hip_runtime.h>

#include "../../include/crf.h"
#include "context.hpp"
#include "paged.hpp"
#include "paged_checks.hpp"

using namespace crf;

extern "C" {

crf_status crf_norm_rope_append(crf_context *ctx, const crf_rope *rope, const crf_seq_batch *batch,
                                const int32_t *positions, const void *q, int64_t q_stride, const void *k,
                                int64_t k_stride, const void *v, int64_t v_stride, const void *q_norm,
                                const void *k_norm, void *q_out, int64_t q_out_stride, const crf_page_pool *pool,
                                int32_t layer, void *stream) {
  const char *what = "crf_norm_rope_append";
  RopeAppend p{};
  bool any = false;
  crf_status st = prepare_append(ctx, what, rope, batch, positions, q, q_stride, k, k_stride, v, v_stride, q_out,
                                 q_out_stride, pool, layer, p, any);
  if (st != CRF_OK || !any) return st;
  if (!k_norm || !aligned16(k_norm) || (q && !q_norm) || !aligned16(q_norm))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: k_norm, or q_norm beside q, NULL or misaligned", what);
  p.q_norm = q_norm;
  p.k_norm = k_norm;
  p.eps = ctx->dims.rms_eps;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER,
         launch_rope_append((hipStream_t)stream, ctx->dims.dtype == CRF_F32, p));
  return CRF_OK;
}

crf_status crf_sink_attention(crf_context *ctx, const crf_seq_batch *batch, const void *q, int64_t q_stride,
                              const crf_page_pool *pool, int32_t layer, float scale, int32_t window, int32_t sinks,
                              void *out, int64_t out_stride, float *lse, void *stream) {
  const char *what = "crf_sink_attention";
  PagedAttn p{};
  bool any = false;
  crf_status st = prepare_attention(ctx, what, batch, q, q_stride, pool, layer, scale, window, out, out_stride, lse, p,
                                    any);
  if (st != CRF_OK) return st;
  if (sinks < 0) return fail(ctx, CRF_ERR_SHAPE, "%s: sinks must be >= 0", what);
  if (!any) return CRF_OK;
  p.sinks = sinks;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_ATTN,
         launch_paged_attn((hipStream_t)stream, ctx->dims.dtype == CRF_F32, p));
  return CRF_OK;
}

}  // extern "C"
