// The C ABI's further operators of a server's step (include/crf.h): norms with the rotary
// append, attention with sinks, attention over shared prefixes, log probabilities.
#include <hip/hip_runtime.h>

#include "../../include/crf.h"
#include "context.hpp"
#include "paged.hpp"
#include "paged_checks.hpp"
#include "serving.hpp"

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

crf_status crf_shared_attention(crf_context *ctx, const crf_seq_batch *batch, const crf_seq_groups *groups,
                                const void *q, int64_t q_stride, const crf_page_pool *pool, int32_t layer, float scale,
                                void *out, int64_t out_stride, float *lse, void *stream) {
  const char *what = "crf_shared_attention";
  SharedAttn p{};
  bool any = false;
  crf_status st = prepare_attention(ctx, what, batch, q, q_stride, pool, layer, scale, 0, out, out_stride, lse, p.a,
                                    any);
  if (st != CRF_OK) return st;
  if (!groups) return fail(ctx, CRF_ERR_INVALID_ARG, "%s: the groups are NULL", what);
  if (groups->n_groups < 0) return fail(ctx, CRF_ERR_SHAPE, "%s: n_groups must be >= 0", what);
  if (groups->n_groups > batch->n_seqs)
    return fail(ctx, CRF_ERR_SHAPE, "%s: %d groups of %d sequences", what, groups->n_groups, batch->n_seqs);
  if (!any) return CRF_OK;
  if (groups->n_groups > 0 && (!groups->seq_start || !groups->shared_len || !aligned4(groups->seq_start) ||
                               !aligned4(groups->shared_len)))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: seq_start or shared_len NULL or misaligned", what);
  p.max_new = batch->max_new;
  p.n_groups = groups->n_groups;
  p.seq_start = groups->seq_start;
  p.shared_len = groups->shared_len;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_ATTN,
         launch_shared_attn((hipStream_t)stream, ctx->dims.dtype == CRF_F32, p));
  return CRF_OK;
}

crf_status crf_token_logprobs(crf_context *ctx, int32_t dtype, const void *logits, int64_t row_stride, int32_t n_rows,
                              int32_t vocab, const int32_t *tokens, int32_t n_tokens, float *logprob, float *entropy,
                              float *lse, int32_t top, int32_t *top_token, float *top_logprob, void *stream) {
  const char *what = "crf_token_logprobs";
  crf_status st = check_context(ctx, what);
  if (st != CRF_OK) return st;
  if (dtype != CRF_F32 && dtype != CRF_BF16)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: unknown dtype %d", what, dtype);
  if (n_rows < 0 || vocab < 1 || n_tokens < 0 || top < 0 || top > vocab)
    return fail(ctx, CRF_ERR_SHAPE, "%s: n_rows, n_tokens and top >= 0, vocab >= 1 and top <= vocab", what);
  if (top > LOGP_MAX_TOP) return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: top %d above %d", what, top, LOGP_MAX_TOP);
  if (vocab > 1 << 30) return fail(ctx, CRF_ERR_UNSUPPORTED, "%s: more than 2^30 logits a row", what);
  if (row_stride < vocab && n_rows > 1)
    return fail(ctx, CRF_ERR_SHAPE, "%s: the rows of logits overlap (stride %lld)", what, (long long)row_stride);
  if (n_rows == 0) return CRF_OK;
  const uintptr_t esz = dtype == CRF_F32 ? 4 : 2;
  if (!logits || (uintptr_t)logits % esz)
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: logits NULL or misaligned", what);
  if (n_tokens > 0 && (!tokens || !logprob || !aligned4(tokens) || !aligned4(logprob)))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: tokens or logprob NULL or misaligned", what);
  if (top > 0 && (!top_token || !top_logprob || !aligned4(top_token) || !aligned4(top_logprob)))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: top_token or top_logprob NULL or misaligned", what);
  if (!aligned4(entropy) || !aligned4(lse))
    return fail(ctx, CRF_ERR_INVALID_ARG, "%s: entropy or lse misaligned", what);
  TokenLogprobs p{};
  p.logits = logits;
  p.ld = row_stride;
  p.n_rows = n_rows;
  p.vocab = vocab;
  p.tokens = tokens;
  p.n_tokens = n_tokens;
  p.top = top;
  p.logprob = logprob;
  p.entropy = entropy;
  p.lse = lse;
  p.top_token = top_token;
  p.top_logprob = top_logprob;
  p.part = ctx->paged_part;
  p.part_floats = ctx->paged_part ? ctx->paged_part_floats : 0;
  p.tickets = tickets(ctx);
  p.n_tickets = PAGED_TICKETS;
  p.err = ctx->d_err;
  LAUNCH(ctx, (hipStream_t)stream, CRF_KK_OTHER, launch_token_logprobs((hipStream_t)stream, dtype == CRF_F32, p));
  return CRF_OK;
}

}  // extern "C"
