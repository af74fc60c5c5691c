// Launchers of the operators over a pool of pages that many sequences share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "common.hpp"

namespace crf {

// Device error flag bits of these operators, next to CRF_DEVERR_BLOCK_TABLE
// (mirrors crf_context_device_errors).
enum { CRF_DEVERR_BATCH = 2, CRF_DEVERR_PAGES = 4 };

// The context's block for these operators: zeros, one int per fork of a call,
// arrival counters.
constexpr int PAGED_ZERO_BYTES = 1024;
constexpr int PAGED_MAX_LIST = 4096;   // forks of a call; sequences of a page map
constexpr int PAGED_MAX_PAGES = 1 << 19;  // pages of a page map
constexpr int PAGED_TICKETS = 1024;
// Workgroups of a launch (a grid holds fewer than 2^32 threads); past them the kernels loop.
constexpr int MOST_GROUPS = 1 << 20;
constexpr size_t PAGED_WS_BYTES = PAGED_ZERO_BYTES + sizeof(int) * (PAGED_MAX_LIST + PAGED_TICKETS);
constexpr int64_t PAGED_PART_FLOATS = (int64_t)1 << 24;  // fp32 contexts: 64 MiB of attention partials

// n / d for 0 <= n < 2^31 as (n * mul) >> shift (exact: shift = 31 + ceil(log2 d),
// mul = ceil(2^shift / d) < 2^32, and n * (mul * d - 2^shift) < 2^shift).
struct FastDiv {
  uint32_t mul;
  int shift;
};
inline FastDiv fast_div(int d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  return FastDiv{(uint32_t)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
}
CRF_DEV int div_by(int n, FastDiv f) { return (int)(((uint64_t)(uint32_t)n * f.mul) >> f.shift); }

// Inclusive prefix over the wave by data-parallel primitives: within rows of 16 lanes,
// then across them.
template <typename F>
CRF_DEV void wave_prefix(F step) {
  step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());  // row_shr:1
  step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());  // row_bcast:15
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());  // row_bcast:31
}
// The value of the lane that step C names, zero where it names none.
template <int C, int ROWS>
CRF_DEV int from_lane(int v) {
  return __builtin_amdgcn_update_dpp(0, v, C, ROWS, 0xf, false);
}
template <int C, int ROWS>
CRF_DEV double from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)from_lane<C, ROWS>((int)(u >> 32)) << 32 |
                                        (uint32_t)from_lane<C, ROWS>((int)u));
}

// Sequences with their new tokens and the pages they own, in one layer's pools.
struct PagedBatch {
  const int32_t *row_start, *length, *tables;  // [n_seqs + 1], [n_seqs], [n_seqs][table_stride]
  int64_t table_stride;
  int n_seqs, n_rows, max_new, max_pages;
  int page_size, n_pages;
  FastDiv ps_div;
  int64_t page_bytes;  // stride of a page in the pool
  char *k, *v;         // layer bases
  int *err;
};

// New tokens of sequence s (the rows from `start` on) and its whole length; a
// sequence that contradicts the batch is flagged and has none.
CRF_DEV int seq_new(const PagedBatch &b, int s, int &start, int &len) {
  start = b.row_start[s];
  const int end = b.row_start[s + 1];
  len = b.length[s];
  const int n = end - start;
  if (start < 0 || end < start || end > b.n_rows || n > b.max_new || len < n ||
      (int64_t)len > (int64_t)b.max_pages * b.page_size) {
    atomicOr(b.err, (int)CRF_DEVERR_BATCH);
    return 0;
  }
  return n;
}

// ---------------------------------------------------------------- rotary positions and append
struct RopeAppend {
  PagedBatch b;
  const void *q, *k, *v;
  void *q_out;                      // q and q_out null: keys and values only
  int64_t q_ld, k_ld, v_ld, qo_ld;  // elements between rows
  const int32_t *positions;         // nullable
  int nq, nkv, hd;
  int rotary_dim, interleaved;
  float mscale;
  double turns[64];                 // revolutions per position of each pair
  const void *q_norm, *k_norm;      // gains [hd] of the heads' norms (k_norm null: no norms)
  float eps;
};
hipError_t launch_rope_append(hipStream_t s, bool f32, const RopeAppend &p);

// ---------------------------------------------------------------- attention
struct PagedAttn {
  PagedBatch b;
  const void *q;
  void *out;
  int64_t q_ld, out_ld;
  float *lse;          // [n_rows, nq], nullable
  int nq, nkv, hd;
  float scale_log2;    // log2(e) * scale
  int window;          // 0: every key
  int sinks;           // first keys that every later row sees besides its window
  float *part;         // partials of split units
  int64_t part_floats;
  unsigned *tickets;   // PAGED_TICKETS, zero between launches
  const char *zeros;   // PAGED_ZERO_BYTES
  int n_cu;
  // set by the launcher
  FastDiv g_div;       // by nq / nkv
  double per_wg;       // workgroups that a unit of work is worth (tiles of 32 rows)
};
hipError_t launch_paged_attn(hipStream_t s, bool f32, const PagedAttn &p);

// ---------------------------------------------------------------- pages
struct PagePools {  // the layers [0, n_layers) from the bases on
  char *k, *v;
  int64_t layer_bytes, page_bytes;
  int n_pages;
};
// pages src[i] of `from` to pages dst[i] of `to`, `bytes` of each in `layers` layers
hipError_t launch_pages_copy(hipStream_t s, const PagePools &from, const PagePools &to, int layers, int bytes, int n,
                             const int32_t *src, const int32_t *dst, int *err);

struct PageMap {
  int32_t *refs, *tables, *lengths;  // [n_pages], [n_seqs][table_stride], [n_seqs]
  int64_t table_stride;
  int n_pages, page_size, n_seqs, max_pages;
  int *err;
};
hipError_t launch_pages_fork(hipStream_t s, const PageMap &m, const PagePools &pool, int layers, int bytes, int n,
                             const int32_t *parents, const int32_t *children, int32_t *state);
hipError_t launch_pages_extend(hipStream_t s, const PageMap &m, const int32_t *n_new);
hipError_t launch_pages_free(hipStream_t s, const PageMap &m, int n, const int32_t *seqs);
hipError_t launch_pages_compact(hipStream_t s, const PageMap &in, const PageMap &out, const PagePools &pool, int layers,
                                int bytes, int32_t *remap, int32_t *moves, int32_t *counts);

}  // namespace crf
