/*
 * crf.h — C ABI of the bounded stale-KV recomputation library (libcrf.so).
 *
 * The library implements the recovery executor of CacheReforge
 * (arxiv 2609.30884): when an evolving LoRA adapter has moved on from the
 * version that produced a KV cache, a contiguous window of decoder layers
 * [l0, l0+h) is re-run over the complete cached prefix under the current
 * adapter, starting from the hidden state retained at the restart boundary,
 * and the refreshed K/V overwrite those layers' slots of the cache
 * (paper Sec. 4.2 "Executable restart"; supplementary Sec. S1.1, definition of
 * the operation R_{r,h}).  It also scores the per-layer adapter drift and risk
 * that feed the reuse / bounded / full-suffix choice (Sec. 4.1, Eq. 8); that
 * choice itself stays with the caller.
 *
 * General conventions
 *   - Every tensor pointer is a DEVICE pointer on the current HIP device,
 *     allocated and owned by the caller.  The library owns only the workspace
 *     inside a crf_context.  Host arrays (per-layer descriptor arrays, the
 *     anchor index array) are read during the call only.
 *   - Tensors are dense row-major.  Weights use the nn.Linear layout
 *     [d_out, d_in].  The storage type of every floating-point tensor is
 *     crf_model_dims.dtype (fp32 or bf16); accumulation is always fp32.
 *   - bf16 tensors must be 16-byte aligned; fp32 tensors 16-byte aligned.
 *   - Work is enqueued asynchronously on `stream` (a hipStream_t; NULL is the
 *     default stream).  No call synchronises the device except where stated.
 *   - Errors are returned as crf_status codes, never by aborting.  Shape,
 *     range and pointer checks happen on the host before anything is
 *     launched; a failed check launches nothing.  The message of the last
 *     failure is available from crf_last_error().
 *   - A context is not thread-safe; use one context per stream.  Calls that
 *     overlap on one context race on its workspace.
 */
#ifndef CRF_H
#define CRF_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CRF_ABI_VERSION 1

typedef enum {
  CRF_OK = 0,
  CRF_ERR_INVALID_ARG = 1,  /* null pointer, misaligned pointer, bad enum      */
  CRF_ERR_SHAPE = 2,        /* tensor/cache sizes inconsistent                  */
  CRF_ERR_RANGE = 3,        /* layer window outside [0, n_layers)              */
  CRF_ERR_UNSUPPORTED = 4,  /* valid model but not a shape this build handles   */
  CRF_ERR_WORKSPACE = 5,    /* exceeds the context's max_tokens / max rank     */
  CRF_ERR_HIP = 6,          /* a HIP runtime call failed                        */
  CRF_ERR_DEVICE = 7        /* a kernel's own bounds check fired (see below)   */
} crf_status;

typedef enum { CRF_F32 = 0, CRF_BF16 = 1 } crf_dtype;

/* Projection targets of one decoder layer (supplementary Eq. sup-qkv-current-layer
 * names Q, K, V; the output and MLP projections are the remaining update
 * targets of supplementary Eq. sup-first-invalid-cache-layer). */
enum { CRF_Q = 0, CRF_K, CRF_V, CRF_O, CRF_GATE, CRF_UP, CRF_DOWN, CRF_NUM_TARGETS };

/* Decoder shape.  Layers are indexed 0..n_layers-1 (Sec. 2.2, Eq. 1).
 * Target shapes: q [n_q_heads*head_dim, d_model], k and v
 * [n_kv_heads*head_dim, d_model], o [d_model, n_q_heads*head_dim],
 * gate and up [d_ffn, d_model], down [d_model, d_ffn]. */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn;
  float rms_eps;      /* RMSNorm epsilon, inside the square root          */
  float rope_theta;   /* rotary base: angle(p, i) = p * theta^(-2i/hd)     */
  int32_t dtype;      /* crf_dtype: storage type of every tensor          */
} crf_model_dims;

/* Frozen base weights of one layer.  attn_norm, mlp_norm: RMSNorm gains [d_model].
 * w[t]: [d_out, d_in] of target t.  bias_q/k/v: optional [d_out] (NULL = none). */
typedef struct {
  const void *attn_norm, *mlp_norm;
  const void *w[CRF_NUM_TARGETS];
  const void *bias_q, *bias_k, *bias_v;
} crf_layer_weights;

/* Current LoRA adapter state of one layer: delta_t(x) = scale * (x A_t^T) B_t^T
 * with A_t [rank, d_in] and B_t [d_out, rank].  A[t] == NULL (with B[t] == NULL)
 * means target t carries no adapter.  rank 0 means the layer has no adapter. */
typedef struct {
  int32_t rank;
  float scale;
  const void *A[CRF_NUM_TARGETS];
  const void *B[CRF_NUM_TARGETS];
} crf_lora_layer;

/* Paged layerwise KV cache C = {K_l, V_l} (Sec. 2.2, Eq. 1).
 * k_pool / v_pool element (layer, page, kv_head, slot, e) lives at
 *   layer*layer_stride + page*page_stride + (kv_head*page_size + slot)*head_dim + e
 * (strides in elements).  Logical token t lives in physical page
 * block_table[t / page_size] (a DEVICE int32 array of ceil(n_tokens/page_size)
 * entries, shared by all layers), slot t % page_size.  K is stored after the
 * rotary rotation, V unrotated.  Pages not named by the block table, slots
 * past n_tokens and layers outside the window are never written.  A block
 * table entry outside [0, n_pages) is caught by the kernels: they skip that
 * page (treating its keys/values as zero) and raise the context's device
 * error flag (crf_context_device_errors). */
typedef struct {
  void *k_pool, *v_pool;
  int64_t layer_stride, page_stride;
  const int32_t *block_table;
  int32_t n_pages, page_size, n_tokens;
} crf_kv_cache;

typedef struct crf_context crf_context;

/* Kernel classes for the optional event timing (crf_context_set_timing). */
enum {
  CRF_KK_NORM = 0, CRF_KK_LORA_DOWN, CRF_KK_GEMM_QKV, CRF_KK_ATTN, CRF_KK_GEMM_O,
  CRF_KK_GEMM_GATEUP, CRF_KK_GEMM_DOWN, CRF_KK_DRIFT, CRF_KK_OTHER, CRF_KK_COUNT
};

/* Human-readable name of a status code (static string). */
const char *crf_status_string(crf_status s);

/* ABI version of the loaded library (CRF_ABI_VERSION at build time). */
int32_t crf_abi_version(void);

/* Create a context for `dims` on the current HIP device.  Allocates the
 * workspace for windows of up to max_tokens prefix tokens and LoRA ranks up
 * to max_lora_rank, and the rotary angle table for positions
 * 0..max_tokens-1.  Besides the per-token buffers (fp32 residual stream,
 * normalised input, queries, attention output, SwiGLU output, LoRA
 * down-projections), a bf16 context holds fixed-size scratch for split
 * work: one or, for prefixes of more 256x256 tiles of d_model than half the
 * compute units, two such fp32 tiles per compute unit for the K-parts of the QKV
 * and residual GEMMs (64 or 128 MiB on 256 CUs), key-split attention partials
 * (ceil(max_tokens/64) x n_q_heads x 16 x (head_dim+4) floats, 61 MB for 16384
 * tokens of 28 heads of 128; from max_tokens = 2048 on at least 512 x 128 x
 * (head_dim+4), 35 MB at head_dim 128), K-split LoRA partials and, when max_lora_rank > 0, the down projection's
 * adapter sums formed inside the gate/up projection (4 x 2 x 256 x 16 floats
 * per compute unit, 32 MiB on 256 CUs, plus one int per gate/up tile), and 2 KiB
 * of arrival counters.  An fp32 context holds 64 MiB of partials for
 * crf_paged_attention (a bf16 one uses the K-parts' scratch), and every context
 * 21 KiB of counters for the operators over a page pool.  All of
 * it is freed by crf_context_destroy.  On success *out
 * receives the context.  Errors: INVALID_ARG (null), UNSUPPORTED (see
 * crf_validate_dims), HIP (allocation failed). */
crf_status crf_context_create(const crf_model_dims *dims, int32_t max_tokens, int32_t max_lora_rank,
                              crf_context **out);
void crf_context_destroy(crf_context *ctx);

/* Message of the last failure on this context ("" if none).  With ctx == NULL,
 * the message of the last failure of a call made without a context. */
const char *crf_last_error(const crf_context *ctx);

/* Host-only check of a decoder shape: every dimension positive,
 * n_q_heads % n_kv_heads == 0, head_dim in {64, 128}, and for bf16 the
 * projection widths multiples of 128, d_ffn a multiple of 64 and every
 * projection weight matrix smaller than 2 GiB.  Touches no device.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED. */
crf_status crf_validate_dims(const crf_model_dims *dims);

/* Host-only check of a recomputation request (Sec. 4.1: the candidate window
 * min(h, N - r) never passes the last layer; supplementary terminology table:
 * ranges are half-open).  Checks dims as above, 0 <= l0, 0 <= h,
 * l0 + h <= n_layers (else RANGE), and the cache geometry: page_size >= 1,
 * n_tokens >= 0, n_tokens <= n_pages * page_size, page_stride >=
 * n_kv_heads*page_size*head_dim, layer_stride >= n_pages*page_stride (else
 * SHAPE), one layer of a pool (n_pages*page_stride elements) under 2 GiB
 * (else UNSUPPORTED), on the bf16 path with h > 0 and more than 16 tokens a
 * projection input of n_tokens x max(d_model, n_q_heads*head_dim, d_ffn)
 * elements under 2 GiB (else UNSUPPORTED: 56,679 tokens at most at
 * Qwen2.5-7B shapes), non-null pools and block table when h > 0 and
 * n_tokens > 0 (else INVALID_ARG).  Touches no device. */
crf_status crf_validate_window(const crf_model_dims *dims, int32_t l0, int32_t h, const crf_kv_cache *kv);

/* Bounded recomputation R_{l0,h} (Sec. 4.2 "Executable restart"; supplementary
 * Sec. S1.1): starting from hidden_at_boundary = H_{l0-1} [n_tokens, d_model]
 * (the residual-stream output of layer l0-1, or the embedding state H_{-1}
 * when l0 == 0), run decoder layers l0..l0+h-1 over all n_tokens prefix
 * tokens under the current adapter `lora`, and overwrite layer l's K/V slots
 * of `kv_cache` for every l in the window with the recomputed, rotated K and
 * V.  Each layer: RMSNorm, Q/K/V projections with the LoRA delta, rotary
 * rotation of Q and K at positions 0..n_tokens-1, causal grouped-query
 * softmax attention (query head j reads K/V head j / (n_q_heads/n_kv_heads),
 * scale 1/sqrt(head_dim)), output projection with LoRA delta and residual,
 * RMSNorm, SwiGLU MLP down(silu(gate x) * up x) with LoRA deltas and residual.
 *   base_weights: host array [n_layers]; only the window's entries are read.
 *   lora:         host array [n_layers] of the current adapter, or NULL (no adapter).
 *   hidden_out:   [n_tokens, d_model] receives H_{l0+h-1}; may be NULL; may alias
 *                 hidden_at_boundary.  When NULL, nothing reads the last
 *                 window layer's output, and that layer's cache entry depends
 *                 on its input only through the K and V projections
 *                 (supplementary Eq. sup-layer-cache-dependency:
 *                 C_l = G_l(H_{l-1})), so it runs RMSNorm and the K/V
 *                 projections (LoRA, bias, rotary, page write) only.
 *                 The K/V written are the same either way: to the bit in an
 *                 fp32 context, in a bf16 one up to the order in which a
 *                 projection's products are summed (which follows from how
 *                 many rows are projected together).
 * h == 0 is direct reuse: nothing is launched and hidden_out (if given and
 * distinct) is not written.  Layers outside the window and pages outside the
 * block table are never touched.  n_tokens comes from kv_cache->n_tokens and
 * must not exceed the context's max_tokens (else WORKSPACE).
 * Errors: as crf_validate_window, plus INVALID_ARG (null or misaligned
 * weights/boundary, dims differing from the context's), WORKSPACE, HIP. */
crf_status crf_recompute_window(crf_context *ctx, const crf_model_dims *dims, const void *hidden_at_boundary,
                                const crf_layer_weights *base_weights, const crf_lora_layer *lora, int32_t l0,
                                int32_t h, const crf_kv_cache *kv_cache, void *hidden_out, void *stream);

/* One stale cache of a batched request. */
typedef struct {
  const void *hidden_at_boundary;   /* [kv.n_tokens, d_model] = H_{l0-1}          */
  const crf_lora_layer *lora;       /* host array [n_layers] or NULL              */
  int32_t l0, h;
  crf_kv_cache kv;
  void *hidden_out;                 /* [kv.n_tokens, d_model] or NULL             */
} crf_window_item;

/* crf_recompute_window over several independent stale caches of one base
 * model, each with its own boundary state, window and adapter version (the
 * per-cache decision of Sec. 4.1 applied to many caches at once).  Every item
 * is validated before anything is launched.  When the items are independent
 * and event timing is off, they run
 * on two internal streams that wait for `stream` and that `stream` then waits
 * for, longest windows first, each on the lane with less work so far; the
 * first such call allocates a second workspace as large as the context's own
 * (what crf_context_create allocates, but for the page-pool operators' partials
 * and counters) and two streams, kept until crf_context_destroy.  Otherwise items run in order on `stream`.  Items are
 * independent when no byte one item may write lies in a range another item
 * may read or write: an item writes the layers [l0, l0+h) of both pools (each
 * layer's whole n_pages*page_stride span, since the pages are chosen by the
 * device-side block table) and its hidden_out, and reads those pool spans,
 * its hidden_at_boundary and its block table.  Items with h == 0 or no tokens
 * take part in no conflict.  Results are the same either way, and to the bit
 * those of the items' windows as separate calls on this context (each item's
 * arithmetic depends on the item alone).
 * Errors: as crf_recompute_window; the failing item's index is in the message;
 * WORKSPACE if the second workspace cannot be allocated. */
crf_status crf_recompute_window_batched(crf_context *ctx, const crf_model_dims *dims,
                                        const crf_layer_weights *base_weights, int32_t n_items,
                                        const crf_window_item *items, void *stream);

/* First decoding step over a cached prefix (Sec. 3.2 "Tail Influence": the
 * first-step next-token logits z, fresh or with a hybrid cache): the embedding
 * states of n_new tokens [n_new, d_model] run through every layer 0..N-1 under
 * `lora`, at positions kv_cache->n_tokens .. kv_cache->n_tokens + n_new - 1.
 * At each layer they attend to that layer's cached K/V of the prefix (whatever
 * adapter version produced each layer: a hybrid cache is just a pool whose
 * layers come from different versions) and causally to each other; their own
 * rotated K and V are written into the slots after the prefix.  Then the final
 * RMSNorm (final_norm [d_model]) and the LM head (lm_head [vocab, d_model],
 * nn.Linear layout) give the logits of the last new token:
 * logits_out[vocab] (fp32, device).  The block table must cover
 * kv_cache->n_tokens + n_new tokens.  bf16 contexts only.
 * Errors: as crf_recompute_window over the window [0, N) of a prefix of
 * n_tokens + n_new tokens, plus SHAPE (n_new < 1), UNSUPPORTED (fp32 context,
 * vocab not a positive multiple of 8, LM head of 2 GiB or more), WORKSPACE
 * (n_new or n_tokens + n_new above max_tokens), INVALID_ARG (NULL or
 * misaligned final_norm, lm_head, logits_out). */
crf_status crf_decode_logits(crf_context *ctx, const crf_model_dims *dims, const void *new_tokens, int32_t n_new,
                             const crf_layer_weights *base_weights, const crf_lora_layer *lora,
                             const crf_kv_cache *kv_cache, const void *final_norm, const void *lm_head,
                             int32_t vocab, float *logits_out, void *stream);

/* Runtime drift and risk (Sec. 4.1 "Runtime risk and range selection", Eq. 8):
 *   d_l = || theta_t - theta_l^anchor ||_2,   q_l = s_l * d_l.
 * theta is the whole adapter: every A and B entry of every target of every
 * layer.  current: host array [n_layers] (theta_t).  versions: host array of
 * n_versions pointers, each to a host array [n_layers] of stored adapter
 * states; anchor_version: host int32 [n_layers], index of the version that
 * produced layer l's cache.  Targets present in `current` must be present
 * with the same rank in every version.  sensitivity: device fp32 [n_layers]
 * (s_l) or NULL for s = 1.  per_layer_only != 0 restricts the norm to layer
 * l's own slice.  Outputs (device fp32): drift_out [n_layers], risk_out
 * [n_layers], sq_partial_out [n_versions * n_layers] (squared distance of
 * layer l's slice to version v at index v*n_layers + l; may be NULL).
 * Errors: INVALID_ARG (null, anchor index out of range, target missing in a
 * version), SHAPE, HIP. */
crf_status crf_layer_drift(crf_context *ctx, const crf_model_dims *dims, const crf_lora_layer *current,
                           int32_t n_versions, const crf_lora_layer *const *versions,
                           const int32_t *anchor_version, const float *sensitivity, int32_t per_layer_only,
                           float *drift_out, float *risk_out, float *sq_partial_out, void *stream);

/* crf_layer_drift for callers that cannot allocate device memory (tight
 * serving loops, harnesses that forbid hipMalloc).  Not for stream capture:
 * the tables are uploaded from a host buffer that the next call on the same
 * thread overwrites, so a captured copy would read whatever it holds then.
 * Same arguments and results as crf_layer_drift (bitwise: the same kernels in
 * the same order) without a context: the segment tables and the partial sums
 * live in a fixed device scratch of CRF_DRIFT_NOALLOC_MAX_BYTES that the
 * library holds on each device it runs on until the process ends, and the
 * tables are staged on the host in a fixed per-thread buffer of the same size.
 * Nothing is allocated on the device and no allocating library routine is
 * called; the tables reach the scratch by one hipMemcpyAsync from pageable host
 * memory on `stream` (so the call returns once they are copied).  Calls that
 * overlap on one device race on its scratch: serialise them (one stream, or
 * the caller's own ordering).  A request whose tables and partials exceed the
 * scratch (segments: two per adapter target, layer and version; chunks of 2^16
 * elements each; about 64 bytes per chunk and segment) is rejected with
 * WORKSPACE before anything is copied or launched.  Errors are reported through
 * crf_last_error(NULL): INVALID_ARG, SHAPE, UNSUPPORTED (as crf_validate_dims),
 * WORKSPACE, HIP. */
#define CRF_DRIFT_NOALLOC_MAX_BYTES (4 << 20)
crf_status crf_layer_drift_noalloc(const crf_model_dims *dims, const crf_lora_layer *current, int32_t n_versions,
                                   const crf_lora_layer *const *versions, const int32_t *anchor_version,
                                   const float *sensitivity, int32_t per_layer_only, float *drift_out,
                                   float *risk_out, float *sq_partial_out, void *stream);

/* ------------------------------------------------------------------------
 * Many sequences in one cache: operators of a server that keeps the caches of
 * many sequences, each perhaps of another adapter version, in one pool of pages.
 *
 * They take the pool's layout and the head layout of crf_kv_cache and of the
 * context's dims, in both storage types.  Everything about a sequence (its
 * length, its new tokens, its pages) is read on the device, so a captured call
 * follows the values at each replay; the host gives bounds.  Conventions as
 * above: asynchronous on `stream`, nothing allocated, checks on the host before
 * any launch, the kernels' own checks reported by crf_context_device_errors.
 * The current device must be the context's (else INVALID_ARG).  Calls on one
 * context share its workspace: they run one after the other, on one stream or
 * ordered by the caller, captured ones and their replays too. */

/* The pages of all layers.  Element (layer, page, kv_head, slot, e) of a pool is
 * where crf_kv_cache has it; a layer of a pool may pass 2 GiB.  Pools 16-byte
 * aligned, strides (elements) multiples of 8. */
typedef struct {
  void *k_pool, *v_pool;
  int64_t layer_stride, page_stride;
  int32_t n_pages, page_size;
} crf_page_pool;

/* The new tokens of many sequences.  Rows row_start[s] .. row_start[s+1]-1 of the
 * call's tensors are the last tokens of sequence s, which has length[s] tokens
 * with them: row r sits at position length[s] - row_start[s+1] + r, in page
 * block_tables[s][position / page_size].  A sequence may have no new token.
 * Rows past row_start[n_seqs] belong to nobody and are left as they are.
 * row_start [n_seqs+1] (not descending), length [n_seqs] and block_tables
 * [n_seqs][table_stride] are DEVICE int32.  A sequence whose rows or length
 * contradict the bounds below raises error bit 1 and has no new tokens.
 *
 * max_new and max_pages are all that the host knows of the lengths, and
 * crf_paged_attention chooses its kernel by them: tiles of 32 rows where
 * max_new x (n_q_heads/n_kv_heads) is at most 32, or where n_rows and
 * max_pages x page_size keep the reads of K and V small, else tiles of 128.
 * Results are right either way, in other last bits; bounds far above what the
 * batch holds cost time (64 single tokens of 28/4 heads: 154 us with max_new 1,
 * 196 with 0).  A batch of single tokens should say so. */
typedef struct {
  int32_t n_seqs;
  int32_t n_rows;       /* rows of the call's tensors                            */
  int32_t max_new;      /* no sequence has more new tokens (0: n_rows), see above */
  int32_t max_pages;    /* no sequence has more pages, see above                  */
  int64_t table_stride; /* entries between the rows of block_tables              */
  const int32_t *row_start, *length, *block_tables;
} crf_seq_batch;

/* Rotary positions: which elements of a head pair up, how much of the head
 * rotates (the rest passes) and by what angle.  freq[i]: radians per position of
 * pair i; mscale: factor on every cosine and sine.  Made by crf_rope_init, or by
 * the caller for frequencies of its own. */
enum { CRF_ROPE_HALF = 0,         /* pairs (i, i + rotary_dim/2), as the windows use */
       CRF_ROPE_INTERLEAVED = 1   /* pairs (2i, 2i + 1)                              */ };
typedef struct {
  int32_t layout, rotary_dim;
  float mscale;
  double freq[64];
} crf_rope;

/* Scaling of the frequencies f_i = theta^(-2i/rotary_dim) for contexts longer
 * than the trained ones:
 *   NONE    f_i;
 *   LINEAR  f_i / factor (positions interpolated);
 *   BASE    of theta * factor^(rotary_dim / (rotary_dim - 2)) instead of theta;
 *   PARTS   f_i (g_i + (1 - g_i) / factor), g_i the turns f_i original_len / 2 pi of
 *           a pair over the trained length, put on [0, 1] between low_turns and
 *           high_turns (0: 1 and 32).
 * mscale 0: 0.1 ln(factor) + 1 for PARTS with factor > 1, else 1. */
enum { CRF_ROPE_NONE = 0, CRF_ROPE_LINEAR, CRF_ROPE_BASE, CRF_ROPE_PARTS };
typedef struct {
  int32_t kind;
  double factor;
  double original_len;
  double low_turns, high_turns;
  double mscale;
} crf_rope_scaling;

/* Host only.  scaling NULL: none.  Errors: INVALID_ARG (NULL, unknown layout or
 * scaling), UNSUPPORTED (rotary_dim no multiple of 16 in [0, 128]), SHAPE
 * (theta, factor, mscale, original_len or turns out of range, a frequency that is
 * not finite). */
crf_status crf_rope_init(crf_rope *out, int32_t layout, int32_t rotary_dim, double theta,
                         const crf_rope_scaling *scaling);

/* Rotates q into q_out, and appends the new tokens to the cache: k rotated, v as
 * it is, into layer `layer` of the pages at the tokens' positions (which the
 * block tables must already cover, see crf_pages_extend).
 *   q [n_rows][n_q_heads][head_dim], k, v [n_rows][n_kv_heads][head_dim], rows
 *   *_stride elements apart (slices of one fused projection), 16-byte aligned;
 *   q_out may be q with q's stride (else it must not overlap the inputs); both
 *   NULL: keys and values only.
 *   positions: DEVICE int32 [n_rows], rotary positions other than the cache's
 *   (NULL: the cache's).  Angles are reduced in 64 bits (3e-16 of the angle lost
 *   at most); cosine, sine and the products are fp32.
 * A token on a page out of range raises error bit 0 and is not appended (its q is
 * still rotated).
 * Errors: INVALID_ARG, SHAPE, RANGE (layer), UNSUPPORTED (rotary_dim above
 * head_dim or no multiple of 16, more than 2^30 tokens a table, rows x query heads
 * or sequences x query heads). */
crf_status crf_rope_append(crf_context *ctx, const crf_rope *rope, const crf_seq_batch *batch,
                           const int32_t *positions, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride,
                           const crf_page_pool *pool, int32_t layer, void *stream);

/* Softmax attention of every new token over its sequence's pages in layer
 * `layer`: a row at position p sees the keys j <= p, and with window > 0 only
 * those with j > p - window; query head i reads K/V head i / (n_q_heads/n_kv_heads).
 *   q, out [n_rows][n_q_heads][head_dim] as above; out may be q with q's stride
 *   (else it must not overlap q).
 *   scale: of the scores (0: 1/sqrt(head_dim)).
 *   lse (nullable): fp32 [n_rows][n_q_heads], the natural logarithm of each row's
 *   sum of exponentials, by which results over parts of a cache can be joined.
 * Keys on pages out of range are seen by nobody (error bit 0); a row that sees no
 * key gets zeros and lse -inf.  What lies in slots past a sequence's length, or in
 * keys that a row does not see, has no influence on it, numbers or not; a value
 * that is no number counts at every key that the row sees, whatever it weighs.  The
 * result is the same to the bit for every call with the same inputs.
 * Errors: INVALID_ARG, SHAPE (negative or non-finite scale, negative window,
 * strides), RANGE (layer), UNSUPPORTED (as crf_rope_append). */
crf_status crf_paged_attention(crf_context *ctx, const crf_seq_batch *batch, const void *q, int64_t q_stride,
                               const crf_page_pool *pool, int32_t layer, float scale, int32_t window, void *out,
                               int64_t out_stride, float *lse, void *stream);

/* Copies pages src[i] of `from` to pages dst[i] of `to` for i < n, in h layers
 * from from_l0 and to_l0 on: a window's layers saved before a refresh overwrites
 * them, or a cache duplicated for another adapter version.  src, dst: DEVICE
 * int32.  The dst pages must differ from each other and, within one pool, from
 * every src page; else what they hold is one of the sources, in pieces.  A page
 * out of range raises error bit 0 and is skipped.
 * Errors: INVALID_ARG, SHAPE (page sizes differ), RANGE (layers), UNSUPPORTED. */
crf_status crf_pages_copy(crf_context *ctx, const crf_page_pool *from, int32_t from_l0, const crf_page_pool *to,
                          int32_t to_l0, int32_t h, int32_t n, const int32_t *src, const int32_t *dst, void *stream);

/* Who holds which pages, all DEVICE int32: refs [n_pages], how many sequences
 * hold each page (0: free); block_tables [n_seqs][table_stride], of which a
 * sequence's first ceil(length / page_size) entries are in use; lengths [n_seqs]
 * (0: no sequence).  At most 2^19 pages, 4096 sequences and 2^30 tokens a
 * sequence (else UNSUPPORTED).  Free pages are always taken lowest first, in the
 * order of the sequences (or forks) that need them. */
typedef struct {
  int32_t *refs, *block_tables, *lengths;
  int64_t table_stride;
  int32_t n_pages, page_size, n_seqs, max_pages;
} crf_page_map;

/* Makes children[i], which must be empty, a copy of parents[i] for i < n <= 4096
 * (DEVICE int32): it shares the parent's full pages and gets a copy of a page
 * that the parent has begun, in every layer of the context's dims, so that both
 * can be extended.  Parents are taken as they are before the call.  A fork that
 * names a sequence out of range, a child that is not empty or a child that an
 * earlier fork of the call names is skipped (error bit 1), and one for whose page
 * no free page is left (error bit 2); its child stays empty.
 * A table entry of the parent's that is out of range raises error bit 0: it is
 * passed on as it is, or (the begun page) not copied.
 * Errors: INVALID_ARG, SHAPE (map and pool differ), UNSUPPORTED. */
crf_status crf_pages_fork(crf_context *ctx, const crf_page_pool *pool, const crf_page_map *map, int32_t n,
                          const int32_t *parents, const int32_t *children, void *stream);

/* Makes every sequence n_new[s] tokens longer (DEVICE int32 [n_seqs]), with the
 * pages that this takes.  A sequence for which n_new is negative or which would
 * pass max_pages keeps its length (error bit 1); once too few pages are free for
 * one, it and every later one that needs any keep theirs (error bit 2).
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED. */
crf_status crf_pages_extend(crf_context *ctx, const crf_page_map *map, const int32_t *n_new, void *stream);

/* Ends n sequences (DEVICE int32): their pages are held by one fewer, their
 * length is 0, their table rows are left.  A sequence that is empty or named
 * twice is freed once; one out of range, or a page that nobody holds, raises
 * error bit 1, a table entry out of range bit 0.  Errors: INVALID_ARG, SHAPE, UNSUPPORTED. */
crf_status crf_pages_free(crf_context *ctx, const crf_page_map *map, int32_t n, const int32_t *seqs, void *stream);

/* Moves the pages in use to the front of the pool, in every layer: with L of
 * them, the k-th at or past L goes to the k-th free one below L.  map_out, which
 * may be map or any of its arrays, receives the new counts, tables and lengths;
 * remap [n_pages] the new place of every page (-1: it was free); counts [2] L and
 * the number of pages moved (all DEVICE int32).  The pages moved keep their bytes
 * in their old places, so readers through the old map are right until those are
 * used again.  A table entry that names no page in use becomes -1 (error bit 0).
 * A sequence whose length passes max_pages or is negative keeps its table row as
 * it is (error bit 1); map_out's length and row of it are not written.
 * Errors: INVALID_ARG, SHAPE (maps or pool differ), UNSUPPORTED, WORKSPACE. */
crf_status crf_pages_compact(crf_context *ctx, const crf_page_pool *pool, const crf_page_map *map,
                             const crf_page_map *map_out, int32_t *remap, int32_t *counts, void *stream);

/* Device-side error flags raised by kernels' own bounds checks since the last
 * call (bit 0: a block table entry outside [0, n_pages); bit 1: a sequence of a
 * batch or page map that contradicts it; bit 2: too few free pages).
 * Synchronises the device, then clears the flags. */
crf_status crf_context_device_errors(crf_context *ctx, int32_t *flags_out);

/* Optional per-kernel-class event timing.  While enabled, each launch is
 * bracketed by HIP events on its stream.  crf_context_read_timing
 * synchronises those events and returns, per kernel class (CRF_KK_*), the
 * summed milliseconds and launch counts since the last read, then resets. */
crf_status crf_context_set_timing(crf_context *ctx, int32_t enable);
/* The same for a subset of kernel classes: bit k of class_mask enables class
 * k (CRF_KK_*), 0 disables timing; enable != 0 above is the mask of every
 * class.  Each bracketed launch costs two event records on its stream, so a
 * measurement that needs one class's launch times only brackets that class.
 * Errors: INVALID_ARG (null context, bits at or past CRF_KK_COUNT). */
crf_status crf_context_set_timing_classes(crf_context *ctx, uint32_t class_mask);
crf_status crf_context_read_timing(crf_context *ctx, float *ms_out, int32_t *count_out, int32_t n_kinds);

/* Device facts for reporting measurements against the hardware's peak:
 * compute-unit count, peak engine clock (MHz) and the architecture name
 * (written NUL-terminated into name, at most name_len bytes; name may be NULL).
 * Errors: INVALID_ARG (null outputs), HIP. */
crf_status crf_device_info(int32_t device, int32_t *n_cu_out, int32_t *max_sclk_mhz_out, char *name,
                           int32_t name_len);

#ifdef __cplusplus
}
#endif
#endif /* CRF_H */
