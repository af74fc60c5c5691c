// The context behind the C ABI and what its entry points share (host side).
#pragma once
#include <hip/hip_runtime.h>

#include <string>
#include <vector>

#include "../../include/crf.h"
#include "kernels.hpp"

namespace crf {

struct Timer {
  uint32_t mask = 0;            // bit k: launches of class k are bracketed by events
  std::vector<hipEvent_t> ev;   // pairs (start, stop)
  std::vector<int> kind;        // per pair
  size_t used = 0;              // pairs recorded since last read
};

// Pinned host staging of the drift tables of one call; `ev` marks their copy.
struct DriftStage {
  void *host = nullptr;
  size_t bytes = 0;
  hipEvent_t ev = nullptr;
  bool recorded = false;
};

}  // namespace crf

struct crf_context {
  crf_model_dims dims;
  int32_t max_tokens = 0, max_rank = 0, rank_pad = 0;
  int device = 0;
  size_t esz = 2;
  // workspace
  float *hres = nullptr;   // [T, d] residual stream, fp32
  void *xn = nullptr;      // [T, d] normalised input
  void *q = nullptr;       // [T, dq] rotated queries
  void *attn = nullptr;    // [T, dq] attention output
  void *act = nullptr;     // [T, f] SwiGLU output
  void *u = nullptr;       // bf16: [T, 3*rank_pad] LoRA down-projections; fp32: [T, 3*max_rank] past the fused ranks
  float2 *rope_cs = nullptr;
  int *d_err = nullptr;
  float *attn_part = nullptr;  // bf16 path: key-split attention partials
  int64_t attn_part_floats = 0;
  float *lora_part = nullptr;  // bf16 path, <= 16 token rows: parts of the LoRA down-projections
  int64_t lora_part_floats = 0;
  // bf16 path: K-part partials of the projections (gemm_part_floats), of which
  // the 256x256 tiles' last round may fill more (gemm_split_floats)
  float *gemm_part = nullptr;
  int64_t gemm_part_floats = 0, gemm_split_floats = 0;
  float *dn_part = nullptr;    // bf16 path: down-projection adapter sums fused into gate/up
  int *dn_head = nullptr;      //   and the table of their first tiles
  unsigned *tickets = nullptr; // bf16 path: arrival counters of K-split workgroups, zero between launches
  int n_tickets = 0;
  int n_cu = 0;
  // the paged operators: a block of zeros (loads of keys that no row sees), the
  // outcome of each fork of a call, arrival counters (zero between launches) and
  // the partials of keys split over workgroups (bf16: the K-part buffer above)
  char *paged_ws = nullptr;
  float *paged_part = nullptr;
  int64_t paged_part_floats = 0;
  // drift staging
  crf::DriftStage drift_stage[4];
  unsigned drift_next = 0;  // stage of the next call
  void *drift_dev = nullptr;
  size_t drift_dev_bytes = 0;
  std::string last_error;
  crf::Timer timer;
  // batched calls over independent caches: a second workspace (a context of
  // the same shape, made by the first such call) and two lane streams forked
  // from the caller's stream
  crf_context *lane2 = nullptr;
  hipStream_t lane_s[2] = {nullptr, nullptr};
  hipEvent_t fork_ev = nullptr, join_ev[2] = {nullptr, nullptr};
};

namespace crf {

// Records the message of a failed call (ctx NULL: for crf_last_error(NULL)).
crf_status fail(crf_context *ctx, crf_status st, const char *fmt, ...);

#define HIP_TRY(ctx, expr)                                                                       \
  do {                                                                                           \
    hipError_t e_ = (expr);                                                                      \
    if (e_ != hipSuccess) return fail(ctx, CRF_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// Event timing of one launch of kernel class k, when it is enabled.
struct Launch {
  crf_context *ctx;
  hipStream_t s;
  int kind;
  size_t idx = 0;
  bool on;
  Launch(crf_context *c, hipStream_t st, int k) : ctx(c), s(st), kind(k), on(((c->timer.mask >> k) & 1u) != 0) {
    Timer &t = ctx->timer;
    if (!on) return;
    idx = t.used;
    if (2 * idx + 2 > t.ev.size()) {
      hipEvent_t a, b;
      if (hipEventCreate(&a) != hipSuccess || hipEventCreate(&b) != hipSuccess) return;
      t.ev.push_back(a);
      t.ev.push_back(b);
      t.kind.push_back(k);
    }
    t.kind[idx] = k;
    (void)hipEventRecord(t.ev[2 * idx], s);
  }
  ~Launch() {
    Timer &t = ctx->timer;
    if (!on || 2 * idx + 2 > t.ev.size()) return;
    (void)hipEventRecord(t.ev[2 * idx + 1], s);
    t.used = idx + 1;
  }
};

#define LAUNCH(ctx, s, kind, expr)                                                                     \
  do {                                                                                                 \
    Launch lt_(ctx, s, kind);                                                                          \
    hipError_t e_ = (expr);                                                                            \
    if (e_ != hipSuccess) return fail(ctx, CRF_ERR_HIP, "launch %s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

}  // namespace crf
