// What the entry points of norms with the rotary append, attention with sinks and over shared
// prefixes and log probabilities refuse, on the host: their sources with launches that only
// count.  Prints the number of calls checked.
#define main refusals_main
#include "paged_refusals_check.cpp"
#undef main

#include "../../paper_2609_30884_amd/csrc/serving_api.cpp"

static SharedAttn g_shared;
static TokenLogprobs g_logp;
namespace crf {
hipError_t launch_shared_attn(hipStream_t, bool, SharedAttn p) {
  g_shared = p;
  return count();
}
hipError_t launch_token_logprobs(hipStream_t, bool, const TokenLogprobs &p) {
  g_logp = p;
  return count();
}
}  // namespace crf

struct More : Call {
  const void *q_norm, *k_norm, *logits;
  int32_t sinks = 4, dtype = CRF_BF16, n_rows = 6, vocab = 100, n_tokens = 2, top = 5;
  int64_t ld = 100;
  crf_seq_groups groups;
  const int32_t *tokens;
  float *logprob, *entropy, *lsum, *top_logprob;
  int32_t *top_token;
  More() {
    q_norm = k_norm = logits = at;
    groups = crf_seq_groups{2, (int32_t *)at, (int32_t *)at};
    tokens = top_token = (int32_t *)at;
    logprob = entropy = lsum = top_logprob = (float *)at;
    ctx.dims.rms_eps = 1e-5f;
  }
  crf_status norm() {
    return crf_norm_rope_append(&ctx, &rope, &batch, positions, q, q_ld, k, k_ld, v, v_ld, q_norm, k_norm, q_out, o_ld,
                                &pool, layer, nullptr);
  }
  crf_status sink() {
    return crf_sink_attention(&ctx, &batch, q, q_ld, &pool, layer, scale, window, sinks, out, o_ld, lse, nullptr);
  }
  crf_status shared() {
    return crf_shared_attention(&ctx, &batch, &groups, q, q_ld, &pool, layer, scale, out, o_ld, lse, nullptr);
  }
  crf_status no_groups() {
    return crf_shared_attention(&ctx, &batch, nullptr, q, q_ld, &pool, layer, scale, out, o_ld, lse, nullptr);
  }
  crf_status logp() {
    return crf_token_logprobs(&ctx, dtype, logits, ld, n_rows, vocab, tokens, n_tokens, logprob, entropy, lsum, top,
                              top_token, top_logprob, nullptr);
  }
};

typedef crf_status (More::*Entry2)();
static void expect2(const char *name, Entry2 e, crf_status st, int launches, std::function<void(More &)> change) {
  More c;
  change(c);
  g_launches = 0;
  const crf_status got = (c.*e)();
  ++g_checked;
  if (got != st || g_launches != launches) {
    ++g_wrong;
    printf("%s: status %d, %d launches; wanted %d, %d (%s)\n", name, got, g_launches, st, launches, g_message.c_str());
  }
}
#define NOT(entry, st, ...) expect2(#entry " " #__VA_ARGS__, &More::entry, st, 0, [](More &c) { __VA_ARGS__; })
#define DONE(entry, n, ...) expect2(#entry " " #__VA_ARGS__, &More::entry, CRF_OK, n, [](More &c) { __VA_ARGS__; })

int main() {
  const auto ARG = CRF_ERR_INVALID_ARG, SHAPE = CRF_ERR_SHAPE, RANGE = CRF_ERR_RANGE, UNS = CRF_ERR_UNSUPPORTED;
  const float inf = std::numeric_limits<float>::infinity();
  for (Entry2 e : {&More::norm, &More::sink, &More::shared, &More::logp}) {
    expect2("right", e, CRF_OK, 1, [](More &) {});
    expect2("another device", e, ARG, 0, [](More &c) { c.ctx.device = 1; });
  }
  for (Entry2 e : {&More::norm, &More::sink, &More::shared}) {
    expect2("k_pool", e, ARG, 0, [](More &c) { c.pool.k_pool = nullptr; });
    expect2("page_stride", e, SHAPE, 0, [](More &c) { c.pool.page_stride = 2040; });
    expect2("layer", e, RANGE, 0, [](More &c) { c.layer = 3; });
    expect2("layer", e, RANGE, 0, [](More &c) { c.layer = -1; });
    expect2("n_seqs", e, SHAPE, 0, [](More &c) { c.batch.n_seqs = -1; });
    expect2("2^30 tokens", e, UNS, 0, [](More &c) { c.batch.table_stride = c.batch.max_pages = (1 << 26) + 1; });
    expect2("2^30 rows", e, UNS, 0, [](More &c) { c.batch.n_rows = (1 << 28) + 1; });
    expect2("row_start", e, ARG, 0, [](More &c) { c.batch.row_start = nullptr; });
    expect2("q", e, ARG, 0, [](More &c) { c.q = c.at + 2; });
    expect2("q rows overlap", e, SHAPE, 0, [](More &c) { c.q_ld = 248; });
    expect2("output rows overlap", e, SHAPE, 0, [](More &c) { c.o_ld = 0; });
    expect2("in place with two strides", e, SHAPE, 0, [](More &c) { c.o_ld = 512; });
    expect2("no row", e, CRF_OK, 0, [](More &c) { c.batch.n_rows = 0; });
  }
  NOT(norm, ARG, c.k_norm = nullptr);
  NOT(norm, ARG, c.q_norm = nullptr);
  NOT(norm, ARG, c.k_norm = c.at + 8);
  NOT(norm, ARG, c.q_norm = c.at + 2);
  NOT(norm, ARG, c.q = nullptr);
  DONE(norm, 1, c.q = nullptr; c.q_out = nullptr; c.q_norm = nullptr);
  NOT(norm, UNS, c.rope.rotary_dim = 72);
  NOT(norm, ARG, c.rope.layout = 2);
  for (Entry2 e : {&More::sink, &More::shared}) {
    expect2("scale", e, SHAPE, 0, [](More &c) { c.scale = -1.f; });
    expect2("scale", e, SHAPE, 0, [=](More &c) { c.scale = inf; });
    expect2("out", e, ARG, 0, [](More &c) { c.out = nullptr; });
    expect2("lse", e, ARG, 0, [](More &c) { c.lse = (float *)(c.at + 2); });
    expect2("no lse", e, CRF_OK, 1, [](More &c) { c.lse = nullptr; });
  }
  NOT(sink, SHAPE, c.window = -1);
  NOT(sink, SHAPE, c.sinks = -1);
  NOT(sink, SHAPE, c.sinks = INT32_MIN);
  NOT(sink, SHAPE, c.sinks = -1; c.batch.n_rows = 0);
  DONE(sink, 1, c.sinks = INT32_MAX; c.window = INT32_MAX);
  DONE(sink, 1, c.sinks = 0);
  NOT(no_groups, ARG, (void)c);
  NOT(shared, SHAPE, c.groups.n_groups = -1);
  NOT(shared, SHAPE, c.groups.n_groups = 6);
  NOT(shared, ARG, c.groups.seq_start = nullptr);
  NOT(shared, ARG, c.groups.shared_len = nullptr);
  NOT(shared, ARG, c.groups.shared_len = (int32_t *)(c.at + 1));
  DONE(shared, 1, c.groups = (crf_seq_groups{0, nullptr, nullptr}));
  DONE(shared, 1, c.groups.n_groups = 5);
  NOT(logp, ARG, c.dtype = 2);
  NOT(logp, SHAPE, c.n_rows = -1);
  NOT(logp, SHAPE, c.vocab = 0);
  NOT(logp, SHAPE, c.n_tokens = -1);
  NOT(logp, SHAPE, c.top = -1);
  NOT(logp, SHAPE, c.top = 30; c.vocab = 20);
  NOT(logp, UNS, c.top = 33);
  NOT(logp, UNS, c.vocab = (1 << 30) + 1; c.ld = c.vocab);
  NOT(logp, SHAPE, c.ld = 99);
  DONE(logp, 1, c.ld = 0; c.n_rows = 1);
  NOT(logp, ARG, c.logits = nullptr);
  NOT(logp, ARG, c.logits = c.at + 1);
  NOT(logp, ARG, c.logits = c.at + 2; c.dtype = CRF_F32);
  DONE(logp, 1, c.logits = c.at + 2);
  NOT(logp, ARG, c.tokens = nullptr);
  NOT(logp, ARG, c.logprob = nullptr);
  NOT(logp, ARG, c.tokens = (int32_t *)(c.at + 2));
  DONE(logp, 1, c.tokens = nullptr; c.logprob = nullptr; c.n_tokens = 0);
  NOT(logp, ARG, c.top_token = nullptr);
  NOT(logp, ARG, c.top_logprob = (float *)(c.at + 2));
  DONE(logp, 1, c.top = 0; c.top_token = nullptr; c.top_logprob = nullptr);
  NOT(logp, ARG, c.entropy = (float *)(c.at + 1));
  NOT(logp, ARG, c.lsum = (float *)(c.at + 3));
  DONE(logp, 1, c.entropy = c.lsum = nullptr);
  DONE(logp, 0, c.n_rows = 0; c.logits = nullptr);
  // what a right call hands to the kernels
  More c;
  c.window = 7;
  if (c.sink() != CRF_OK || g_attn.sinks != 4 || g_attn.window != 7) ++g_wrong, printf("sinks\n");
  if (c.attend() != CRF_OK || g_attn.sinks != 0) ++g_wrong, printf("sinks of paged attention\n");
  if (c.norm() != CRF_OK || g_rope.k_norm != c.at || g_rope.eps != 1e-5f) ++g_wrong, printf("norms\n");
  if (c.append() != CRF_OK || g_rope.k_norm) ++g_wrong, printf("norms of the rotary append\n");
  if (c.shared() != CRF_OK || g_shared.n_groups != 2 || g_shared.a.window != 0) ++g_wrong, printf("groups\n");
  c.ctx.paged_part = nullptr;
  if (c.logp() != CRF_OK || g_logp.part_floats != 0) ++g_wrong, printf("log probabilities without room for parts\n");
  if (crf_token_logprobs(nullptr, 0, nullptr, 0, 0, 1, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr, nullptr,
                         nullptr) != ARG)
    ++g_wrong, printf("no context\n");
  if (g_wrong) return 1;
  printf("ok %d\n", g_checked);
  return 0;
}
