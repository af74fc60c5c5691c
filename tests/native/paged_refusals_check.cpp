// What the entry points over a page pool refuse, on the host: their sources with
// launches that only count.  A refused call launches nothing; a right one once.
// Prints the number of calls checked.
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <functional>
#include <limits>

static int g_device = 0;
static hipError_t fake_device(int *d) {
  *d = g_device;
  return hipSuccess;
}
#define hipGetDevice fake_device
#include "../../paper_2609_30884_amd/csrc/paged_api.cpp"

static int g_launches = 0;
static RopeAppend g_rope;
static PagedAttn g_attn;

namespace crf {
static std::string g_message;
crf_status fail(crf_context *, crf_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_message = buf;
  return st;
}
static hipError_t count() {
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_rope_append(hipStream_t, bool, const RopeAppend &p) {
  g_rope = p;
  return count();
}
hipError_t launch_paged_attn(hipStream_t, bool, const PagedAttn &p) {
  g_attn = p;
  return count();
}
hipError_t launch_pages_copy(hipStream_t, const PagePools &, const PagePools &, int, int, int, const int32_t *,
                             const int32_t *, int *) {
  return count();
}
hipError_t launch_pages_fork(hipStream_t, const PageMap &, const PagePools &, int, int, int, const int32_t *,
                             const int32_t *, int32_t *) {
  return count();
}
hipError_t launch_pages_extend(hipStream_t, const PageMap &, const int32_t *) { return count(); }
hipError_t launch_pages_free(hipStream_t, const PageMap &, int, const int32_t *) { return count(); }
hipError_t launch_pages_compact(hipStream_t, const PageMap &, const PageMap &, const PagePools &, int, int, int32_t *,
                                int32_t *, int32_t *) {
  return count();
}
}  // namespace crf

struct Call {  // a right call of every entry point, before something is made wrong
  crf_context ctx;
  crf_rope rope;
  crf_seq_batch batch;
  crf_page_pool pool, to;
  crf_page_map map, map_out;
  int32_t layer = 1, from_l0 = 0, to_l0 = 1, h = 2, n = 3, window = 0;
  float scale = 0.f;
  char *at = (char *)4096;
  const void *q, *k, *v;
  void *q_out, *out;
  int64_t q_ld, k_ld, v_ld, o_ld;
  float *lse;
  const int32_t *positions, *list_a, *list_b;
  int32_t *remap, *counts;
  Call() {
    ctx.dims = crf_model_dims{3, 256, 4, 2, 64, 128, 1e-6f, 1e6f, CRF_BF16};
    ctx.esz = 2;
    ctx.paged_ws = (char *)4096;
    ctx.paged_part = (float *)4096;
    ctx.paged_part_floats = 1 << 20;
    crf_rope_init(&rope, CRF_ROPE_HALF, 64, 1e6, nullptr);
    pool = crf_page_pool{at, at, 100 * 2048, 2048, 100, 16};
    to = pool;
    batch = crf_seq_batch{5, 20, 4, 10, 10, (int32_t *)at, (int32_t *)at, (int32_t *)at};
    map = crf_page_map{(int32_t *)at, (int32_t *)at, (int32_t *)at, 10, 100, 16, 5, 10};
    map_out = map;
    q = k = v = q_out = out = at;
    q_ld = o_ld = 256;
    k_ld = v_ld = 128;
    lse = (float *)at;
    positions = nullptr;
    list_a = list_b = (int32_t *)at;
    remap = counts = (int32_t *)at;
  }
  crf_status append() {
    return crf_rope_append(&ctx, &rope, &batch, positions, q, q_ld, k, k_ld, v, v_ld, q_out, o_ld, &pool, layer, nullptr);
  }
  crf_status attend() {
    return crf_paged_attention(&ctx, &batch, q, q_ld, &pool, layer, scale, window, out, o_ld, lse, nullptr);
  }
  crf_status copy() { return crf_pages_copy(&ctx, &pool, from_l0, &to, to_l0, h, n, list_a, list_b, nullptr); }
  crf_status fork() { return crf_pages_fork(&ctx, &pool, &map, n, list_a, list_b, nullptr); }
  crf_status extend() { return crf_pages_extend(&ctx, &map, list_a, nullptr); }
  crf_status drop() { return crf_pages_free(&ctx, &map, n, list_a, nullptr); }
  crf_status compact() { return crf_pages_compact(&ctx, &pool, &map, &map_out, remap, counts, nullptr); }
};

static int g_checked = 0, g_wrong = 0;
typedef crf_status (Call::*Entry)();
static void expect(const char *name, Entry e, crf_status st, int launches, std::function<void(Call &)> change) {
  Call c;
  change(c);
  g_launches = 0;
  g_device = 0;
  const crf_status got = (c.*e)();
  ++g_checked;
  if (got != st || g_launches != launches) {
    ++g_wrong;
    printf("%s: status %d, %d launches; wanted %d, %d (%s)\n", name, got, g_launches, st, launches, g_message.c_str());
  }
}
#define REFUSED(entry, st, ...) expect(#__VA_ARGS__, &Call::entry, st, 0, [](Call &c) { __VA_ARGS__; })
#define TAKEN(entry, n, ...) expect(#__VA_ARGS__, &Call::entry, CRF_OK, n, [](Call &c) { __VA_ARGS__; })

int main() {
  const auto ARG = CRF_ERR_INVALID_ARG, SHAPE = CRF_ERR_SHAPE, RANGE = CRF_ERR_RANGE, UNS = CRF_ERR_UNSUPPORTED;
  const float inf = std::numeric_limits<float>::infinity();
  (void)inf;
  for (Entry e : {&Call::append, &Call::attend, &Call::copy, &Call::fork, &Call::extend, &Call::drop, &Call::compact}) {
    expect("right", e, CRF_OK, 1, [](Call &) {});
    expect("another device", e, ARG, 0, [](Call &c) { c.ctx.device = 1; });
  }
  for (Entry e : {&Call::append, &Call::attend, &Call::copy, &Call::fork, &Call::compact}) {
    expect("k_pool", e, ARG, 0, [](Call &c) { c.pool.k_pool = nullptr; });
    expect("v_pool", e, ARG, 0, [](Call &c) { c.pool.v_pool = c.at + 8; });
    expect("page_size", e, SHAPE, 0, [](Call &c) { c.pool.page_size = 0; });
    expect("n_pages", e, SHAPE, 0, [](Call &c) { c.pool.n_pages = -1; });
    expect("page_stride", e, SHAPE, 0, [](Call &c) { c.pool.page_stride = 2040; });
    expect("layer_stride", e, SHAPE, 0, [](Call &c) { c.pool.layer_stride = 99 * 2048; });
    expect("overflow", e, SHAPE, 0, [](Call &c) { c.pool.page_stride = INT64_MAX / 8 * 8; });
    expect("odd stride", e, ARG, 0, [](Call &c) { c.pool.layer_stride += 4; });
    expect("a page of 1 GiB", e, UNS, 0, [](Call &c) {
      c.pool.page_size = 1 << 22;
      c.pool.page_stride = (int64_t)1 << 29;
    });
  }
  for (Entry e : {&Call::append, &Call::attend}) {
    expect("layer", e, RANGE, 0, [](Call &c) { c.layer = 3; });
    expect("layer", e, RANGE, 0, [](Call &c) { c.layer = -1; });
    expect("n_seqs", e, SHAPE, 0, [](Call &c) { c.batch.n_seqs = -1; });
    expect("n_rows", e, SHAPE, 0, [](Call &c) { c.batch.n_rows = -1; });
    expect("table_stride", e, SHAPE, 0, [](Call &c) { c.batch.table_stride = 9; });
    expect("2^30 tokens", e, UNS, 0, [](Call &c) { c.batch.table_stride = c.batch.max_pages = (1 << 26) + 1; });
    expect("2^30 tokens", e, CRF_OK, 1, [](Call &c) { c.batch.table_stride = c.batch.max_pages = 1 << 26; });
    expect("2^30 rows", e, UNS, 0, [](Call &c) { c.batch.n_rows = (1 << 28) + 1; });
    expect("row_start", e, ARG, 0, [](Call &c) { c.batch.row_start = nullptr; });
    expect("length", e, ARG, 0, [](Call &c) { c.batch.length = (int32_t *)(c.at + 2); });
    expect("tables", e, ARG, 0, [](Call &c) { c.batch.block_tables = nullptr; });
    expect("q", e, ARG, 0, [](Call &c) { c.q = nullptr; });
    expect("q misaligned", e, ARG, 0, [](Call &c) { c.q = c.at + 2; });
    expect("q rows overlap", e, SHAPE, 0, [](Call &c) { c.q_ld = 248; });
    expect("q row stride", e, ARG, 0, [](Call &c) { c.q_ld = 260; });
    expect("output rows overlap", e, SHAPE, 0, [](Call &c) { c.o_ld = 0; });
    expect("no sequence", e, CRF_OK, 0, [](Call &c) { c.batch.n_seqs = 0; c.batch.row_start = nullptr; });
    expect("no row", e, CRF_OK, 0, [](Call &c) { c.batch.n_rows = 0; c.q = nullptr; });
  }
  REFUSED(append, ARG, c.k = nullptr);
  REFUSED(append, ARG, c.v = c.at + 8);
  REFUSED(append, SHAPE, c.k_ld = 64);
  REFUSED(append, ARG, c.v_ld = 132);
  REFUSED(append, ARG, c.q_out = nullptr);
  REFUSED(append, ARG, c.positions = (int32_t *)(c.at + 1));
  REFUSED(append, ARG, c.rope.layout = 2);
  REFUSED(append, UNS, c.rope.rotary_dim = 128);
  REFUSED(append, UNS, c.rope.rotary_dim = 24);
  REFUSED(append, UNS, c.rope.rotary_dim = -16);
  TAKEN(append, 1, c.rope.rotary_dim = 0);
  TAKEN(append, 1, c.q = c.q_out = nullptr; c.q_ld = c.o_ld = 0);
  REFUSED(attend, ARG, c.out = c.at + 4);
  REFUSED(attend, ARG, c.lse = (float *)(c.at + 2));
  TAKEN(attend, 1, c.lse = nullptr);
  REFUSED(attend, SHAPE, c.scale = -1.f);
  REFUSED(attend, SHAPE, c.scale = std::numeric_limits<float>::infinity());
  REFUSED(attend, SHAPE, c.scale = std::numeric_limits<float>::quiet_NaN());
  REFUSED(attend, SHAPE, c.window = -1);
  REFUSED(copy, RANGE, c.from_l0 = 2);
  REFUSED(copy, RANGE, c.to_l0 = 2);
  REFUSED(copy, RANGE, c.h = -1);
  REFUSED(copy, SHAPE, c.n = -1);
  REFUSED(copy, SHAPE, c.to.page_size = 8);
  REFUSED(copy, ARG, c.list_b = nullptr);
  TAKEN(copy, 0, c.n = 0; c.list_a = nullptr);
  TAKEN(copy, 0, c.h = 0);
  for (Entry e : {&Call::fork, &Call::extend, &Call::drop, &Call::compact}) {
    expect("map n_pages", e, UNS, 0, [](Call &c) { c.map.n_pages = (1 << 19) + 1; });
    expect("map n_seqs", e, UNS, 0, [](Call &c) { c.map.n_seqs = 4097; });
    expect("map max_pages", e, UNS, 0, [](Call &c) { c.map.table_stride = c.map.max_pages = (1 << 19) + 1; });
    expect("map tokens", e, UNS, 0, [](Call &c) { c.map.page_size = 1 << 28; });
    expect("map page_size", e, SHAPE, 0, [](Call &c) { c.map.page_size = 0; });
    expect("map stride", e, SHAPE, 0, [](Call &c) { c.map.table_stride = 9; });
    expect("map refs", e, ARG, 0, [](Call &c) { c.map.refs = nullptr; });
    expect("map tables", e, ARG, 0, [](Call &c) { c.map.block_tables = (int32_t *)(c.at + 1); });
    expect("map lengths", e, ARG, 0, [](Call &c) { c.map.lengths = nullptr; });
  }
  REFUSED(fork, SHAPE, c.map.n_pages = 99);
  REFUSED(fork, SHAPE, c.map.page_size = 8);
  REFUSED(fork, UNS, c.n = 4097);
  REFUSED(fork, ARG, c.list_a = nullptr);
  REFUSED(extend, ARG, c.list_a = nullptr);
  TAKEN(extend, 0, c.map.n_seqs = 0);
  REFUSED(drop, ARG, c.list_a = (int32_t *)(c.at + 2));
  TAKEN(drop, 0, c.n = 0);
  REFUSED(compact, SHAPE, c.map_out.n_seqs = 4);
  REFUSED(compact, SHAPE, c.map_out.max_pages = 9);
  REFUSED(compact, SHAPE, c.map_out.table_stride = 12);
  TAKEN(compact, 1, c.map_out.table_stride = 12; c.map_out.block_tables = (int32_t *)(c.at + 64));
  REFUSED(compact, ARG, c.remap = nullptr);
  REFUSED(compact, ARG, c.counts = nullptr);
  REFUSED(compact, CRF_ERR_WORKSPACE, c.ctx.paged_part_floats = 99);
  // rotary plans
  crf_rope r;
  const crf_rope_scaling parts = {CRF_ROPE_PARTS, 4.0, 4096, 0, 0, 0};
  auto init = [&](crf_status st, crf_rope *o, int layout, int dim, double theta, crf_rope_scaling s) {
    ++g_checked;
    const crf_status got = crf_rope_init(o, layout, dim, theta, &s);
    if (got != st) {
      ++g_wrong;
      printf("crf_rope_init: %d, wanted %d\n", got, st);
    }
  };
  init(CRF_OK, &r, 0, 128, 1e4, parts);
  init(CRF_OK, &r, 1, 0, 1e4, parts);
  init(ARG, nullptr, 0, 64, 1e4, parts);
  init(ARG, &r, 2, 64, 1e4, parts);
  init(UNS, &r, 0, 144, 1e4, parts);
  init(UNS, &r, 0, 72, 1e4, parts);
  init(UNS, &r, 0, -16, 1e4, parts);
  init(SHAPE, &r, 0, 64, 0, parts);
  init(SHAPE, &r, 0, 64, std::numeric_limits<double>::quiet_NaN(), parts);
  init(ARG, &r, 0, 64, 1e4, {4, 4.0, 4096, 0, 0, 0});
  init(SHAPE, &r, 0, 64, 1e4, {CRF_ROPE_LINEAR, 0, 0, 0, 0, 0});
  init(SHAPE, &r, 0, 64, 1e4, {CRF_ROPE_PARTS, 4.0, 0, 0, 0, 0});
  init(SHAPE, &r, 0, 64, 1e4, {CRF_ROPE_PARTS, 4.0, 4096, 40, 32, 0});
  init(SHAPE, &r, 0, 64, 1e4, {CRF_ROPE_NONE, 1.0, 0, 0, 0, -1});
  // what a right call hands to the kernels
  Call c;
  c.batch.max_new = 0;
  c.ctx.dims.dtype = CRF_F32;
  c.ctx.esz = 4;
  if (c.attend() != CRF_OK || g_attn.b.max_new != 20 || g_attn.b.k != c.at + 4 * 100 * 2048 ||
      g_attn.b.page_bytes != 4 * 2048)
    ++g_wrong, printf("attention's arguments\n");
  if (c.append() != CRF_OK || g_rope.b.v != c.at + 4 * 100 * 2048 || g_rope.nq != 4) ++g_wrong, printf("append's arguments\n");
  if (g_wrong) return 1;
  printf("ok %d\n", g_checked);
  return 0;
}
