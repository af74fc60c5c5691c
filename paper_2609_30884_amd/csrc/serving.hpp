// Launchers of a server step's operators beside those over its pages (paged.hpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "paged.hpp"

namespace crf {

// Device error flag bit of a token past the vocabulary (mirrors crf_context_device_errors).
enum { CRF_DEVERR_TOKEN = 8 };

// ---------------------------------------------------------------- log probabilities
constexpr int LOGP_MAX_TOP = 32;
constexpr int LOGP_PARTS = 64;  // workgroups that a row is shared out to, at most: a lane to each
constexpr int LOGP_MOST_GROUPS = MOST_GROUPS;

struct TokenLogprobs {
  const void *logits;
  int64_t ld;  // elements between rows
  int n_rows, vocab;
  const int32_t *tokens;  // [n_rows][n_tokens]
  int n_tokens, top;
  float *logprob, *entropy, *lse;  // [n_rows][n_tokens], [n_rows], [n_rows] (the last two nullable)
  int32_t *top_token;              // [n_rows][top]
  float *top_logprob;
  float *part;  // parts of rows that several workgroups share
  int64_t part_floats;
  unsigned *tickets;  // n_tickets, zero between launches
  int n_tickets;
  int *err;
};
hipError_t launch_token_logprobs(hipStream_t s, bool f32, const TokenLogprobs &p);

// ---------------------------------------------------------------- attention over shared prefixes
constexpr int SHARED_MAX_GROUPS = 1023;

struct SharedAttn {
  PagedAttn a;  // the batch (no window)
  int max_new;   // as the caller bounds it (0: not at all)
  int n_groups;
  const int32_t *seq_start, *shared_len;  // [n_groups + 1], [n_groups]
  // set by the launcher: the items' table, and the parts' O [part_rows][hd] and (reference, sum)
  void *info;
  float *o;
  float2 *ml;
  int part_rows, slots;
};
hipError_t launch_shared_attn(hipStream_t s, bool f32, SharedAttn p);

}  // namespace crf
