// The pages of a cache that many sequences share: copying, forking, extending,
// freeing and compacting them, with the map (how many sequences hold each page,
// block tables, lengths) on the device.
//
// Every choice is deterministic: free pages are taken lowest first, in the order
// of the sequences that need them.  A plan is made by one workgroup, which holds
// one bit per page in LDS (bit set: the page is in use), counts the bits of a
// run of words per thread and scans the counts; the pages' bytes are moved by a
// launch of its own over all compute units.
//
// Moving the bytes is HBM bound: a compaction that moves 710 of 2700 pages of 28 layers,
// bf16, takes 138 us for 651 MB, 4.7 TB/s (a large copy: 5.0).  The plans are latency: one
// workgroup, a chain of loads, a scan and stores (fork 5.1 us, extend 5.1, compact 7.8,
// free 3.3); more workgroups would have to agree on the order of the free pages.
#include "paged.hpp"

namespace crf {
namespace {

constexpr int PNT = 1024;               // threads of a plan
constexpr int PAGE_WORDS = PAGED_MAX_PAGES / 64;  // 64 KB of LDS

CRF_DEV int pages_of(int tokens, int page_size) {  // (tokens in [0, 2^31))
  return (int)((unsigned)tokens / (unsigned)page_size + ((unsigned)tokens % (unsigned)page_size != 0));
}

// Exclusive prefix sums of a and b over the workgroup's PNT threads, and their totals.
struct Pair {
  unsigned a, b;
};
CRF_DEV Pair block_scan(unsigned a, unsigned b, Pair *wsum, Pair &total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Pair x{a, b};
  wave_prefix([&](auto c, auto rows) {
    x.a += (unsigned)from_lane<c(), rows()>((int)x.a);
    x.b += (unsigned)from_lane<c(), rows()>((int)x.b);
  });
  __syncthreads();  // (wsum of an earlier scan has been read)
  if (lane == 63) wsum[wave] = x;
  __syncthreads();
  Pair base{0, 0};
  total = Pair{0, 0};
#pragma unroll
  for (int w = 0; w < PNT / 64; ++w) {
    const Pair t = wsum[w];
    if (w < wave) base.a += t.a, base.b += t.b;
    total.a += t.a, total.b += t.b;
  }
  return Pair{base.a + x.a - a, base.b + x.b - b};
}

// The last i in [0, n) with key[i] <= x (key[0] is 0, keys ascend).
CRF_DEV int last_at_most(const unsigned *key, int n, unsigned x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (key[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The page of rank k among the set bits of word(0), word(1), ..: thread t counts the
// words from t * per on, and before[t] is the number of bits in those of the threads
// before it.  One thread a rank: the free pages of a pool often lie side by side, and
// the thread that counts them would else hand them out one after the other (32
// sequences taking two pages each at most: 10.2 us against 5.1).
template <typename W>
CRF_DEV int page_of_rank(unsigned k, const unsigned *before, int per, W word) {
  const int t = last_at_most(before, PNT, k);
  k -= before[t];
  int w = t * per;
  uint64_t x = word(w);
  for (unsigned c; k >= (c = __popcll(x)); x = word(++w)) k -= c;
  int page = 64 * w;
#pragma unroll
  for (int half = 32; half; half >>= 1) {
    const unsigned c = __popcll(x & (((uint64_t)1 << half) - 1));
    if (k >= c) k -= c, x >>= half, page += half;
  }
  return page;
}

// bits[w]: pages 64 w .. 64 w + 63 in use; pages past n_pages count as `pad`.
CRF_DEV void load_bits(const int32_t *refs, int n_pages, uint64_t *bits, bool pad) {
  const int lane = threadIdx.x % 64, words = (n_pages + 63) / 64;
  for (int w0 = threadIdx.x / 64; w0 < words; w0 += 8 * (PNT / 64)) {
    int r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = (w0 + k * (PNT / 64)) * 64 + lane;
      r[k] = i < n_pages ? refs[i] : (int)pad;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int w = w0 + k * (PNT / 64);
      const uint64_t m = __builtin_amdgcn_ballot_w64(r[k] > 0);
      if (lane == 0 && w < words) bits[w] = m;
    }
  }
  __syncthreads();
}

// ---------------------------------------------------------------- copying

// Chunks of 16 bytes: pair i holds 2 pools x layers x cpp of them.  A thread takes
// CUN of a pair's chunks, CNT apart, all loads in flight before the first store.
constexpr int CNT = 256, CUN = 8;

struct CopyArgs {
  PagePools from, to;
  int per_pair, blocks_per_pair, cpp;  // chunks of a pair; workgroups of a pair; chunks of a page
  FastDiv cpp_div;
  int half;                            // layers * cpp: chunks of the K pool
  int n;
  const int32_t *n_dev;                // compaction: the number of pairs
  int *err;
};

CRF_DEV void copy_pair(const CopyArgs &a, int sp, int dp, int first) {
  const char *s[CUN];
  char *d[CUN];
  u32x4 x[CUN];
#pragma unroll
  for (int u = 0; u < CUN; ++u) {
    int c = first + u * CNT + threadIdx.x;
    s[u] = nullptr;
    if (c >= a.per_pair) continue;
    const bool v = c >= a.half;
    if (v) c -= a.half;
    const int l = div_by(c, a.cpp_div), o = c - l * a.cpp;
    s[u] = (v ? a.from.v : a.from.k) + l * a.from.layer_bytes + sp * a.from.page_bytes + (int64_t)o * 16;
    d[u] = (v ? a.to.v : a.to.k) + l * a.to.layer_bytes + dp * a.to.page_bytes + (int64_t)o * 16;
    x[u] = ld16(s[u]);
  }
#pragma unroll
  for (int u = 0; u < CUN; ++u)
    if (s[u]) st16(d[u], x[u]);
}

__global__ __launch_bounds__(CNT) void pages_copy_kernel(const CopyArgs a, const int32_t *src, const int32_t *dst) {
  const int64_t blocks = (int64_t)a.n * a.blocks_per_pair;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int i = (int)(b / a.blocks_per_pair), part = (int)(b % a.blocks_per_pair);
    const int sp = src[i], dp = dst[i];
    if (sp < 0 || sp >= a.from.n_pages || dp < 0 || dp >= a.to.n_pages) {
      if (threadIdx.x == 0) atomicOr(a.err, (int)CRF_DEVERR_BLOCK_TABLE);
      continue;
    }
    copy_pair(a, sp, dp, part * CNT * CUN);
  }
}

CopyArgs copy_args(const PagePools &from, const PagePools &to, int layers, int bytes, int n, int *err) {
  CopyArgs a{};
  a.from = from;
  a.to = to;
  a.cpp = bytes / 16;
  a.half = layers * a.cpp;
  a.per_pair = 2 * a.half;
  a.blocks_per_pair = (a.per_pair + CNT * CUN - 1) / (CNT * CUN);
  a.cpp_div = fast_div(a.cpp);
  a.n = n;
  a.err = err;
  return a;
}

// ---------------------------------------------------------------- forking

// state[i]: the page that takes the copy of fork i's begun page, -1 where it needs
// none, -2 where the fork is refused.  A child that is named twice is forked by the
// first that names it.  A thread plans up to LPT forks next to each other.
constexpr int LPT = PAGED_MAX_LIST / PNT;

__global__ __launch_bounds__(PNT) void fork_plan_kernel(const PageMap m, int n, const int32_t *parents,
                                                        const int32_t *children, int32_t *state) {
  __shared__ uint64_t bits[PAGE_WORDS];
  __shared__ int claim[PAGED_MAX_LIST];
  __shared__ unsigned before[PNT];
  __shared__ Pair wsum[PNT / 64];
  const int tid = threadIdx.x, each = (n + PNT - 1) / PNT, i0 = tid * each, i1 = min(n, i0 + each);
  for (int s = tid; s < m.n_seqs; s += PNT) claim[s] = n;
  int child[LPT], len[LPT];  // len: the parent's, -1 where the fork is refused
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    const int i = i0 + k;
    len[k] = -1;
    child[k] = 0;
    if (k >= each || i >= i1) continue;
    const int p = parents[i], c = children[i];
    if (p < 0 || p >= m.n_seqs || c < 0 || c >= m.n_seqs || p == c || m.lengths[c] != 0) continue;
    const int l = m.lengths[p];
    if (l < 0 || (int64_t)l > (int64_t)m.max_pages * m.page_size) continue;
    len[k] = l;
    child[k] = c;
  }
  load_bits(m.refs, m.n_pages, bits, true);
#pragma unroll
  for (int k = 0; k < LPT; ++k)
    if (len[k] >= 0) atomicMin(&claim[child[k]], i0 + k);
  __syncthreads();
  unsigned want = 0;  // forks that need a page
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    if (len[k] >= 0 && claim[child[k]] != i0 + k) len[k] = -1;
    want += len[k] > 0 && len[k] % m.page_size != 0;
  }
  const int words = (m.n_pages + 63) / 64, per = (words + PNT - 1) / PNT;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  unsigned free = 0;
  for (int w = w0; w < w1; ++w) free += __popcll(~bits[w]);
  Pair total, at = block_scan(want, free, wsum, total);
  before[tid] = at.b;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    const int i = i0 + k;
    if (k >= each || i >= i1) continue;
    int page = len[k] < 0 ? -2 : -1, err = len[k] < 0 ? (int)CRF_DEVERR_BATCH : 0;
    if (len[k] > 0 && len[k] % m.page_size != 0) {
      if (at.a < total.b) {  // free pages in ascending order, one to each
        page = page_of_rank(at.a, before, per, [&](int w) { return ~bits[w]; });
        m.refs[page] = 1;
      } else {
        page = -2;
        err = (int)CRF_DEVERR_PAGES;
      }
      ++at.a;
    }
    state[i] = page;
    if (err) atomicOr(m.err, err);
    else m.lengths[child[k]] = len[k];
  }
}

// Block row 0 of a fork: its table row and the counts of the full pages that it
// shares; the others copy the begun page.
__global__ __launch_bounds__(CNT) void fork_apply_kernel(const PageMap m, const CopyArgs a, const int32_t *parents,
                                                         const int32_t *children, const int32_t *state) {
  const int i = blockIdx.y, page = state[i];
  if (page == -2) return;
  const int32_t *from = m.tables + (int64_t)parents[i] * m.table_stride;
  int32_t *to = m.tables + (int64_t)children[i] * m.table_stride;
  const int len = m.lengths[children[i]], full = len / m.page_size;
  if (blockIdx.x == 0) {
    for (int j = threadIdx.x; j < full; j += CNT) {
      const int e = from[j];
      to[j] = e;
      if (e < 0 || e >= m.n_pages)
        atomicOr(m.err, (int)CRF_DEVERR_BLOCK_TABLE);
      else
        atomicAdd(&m.refs[e], 1);
    }
    if (threadIdx.x == 0 && page >= 0) to[full] = page;
    return;
  }
  if (page < 0) return;
  const int sp = from[full];
  if (sp < 0 || sp >= m.n_pages) {
    if (threadIdx.x == 0) atomicOr(m.err, (int)CRF_DEVERR_BLOCK_TABLE);
    return;
  }
  copy_pair(a, sp, page, (blockIdx.x - 1) * CNT * CUN);
}

// ---------------------------------------------------------------- extending

// Every sequence s grows by n_new[s] tokens; the pages that this takes are the
// lowest free ones, in the order of the sequences.  The first sequence for which
// too few are left and every later one that needs any keep their length.
__global__ __launch_bounds__(PNT) void extend_kernel(const PageMap m, const int32_t *n_new) {
  __shared__ uint64_t bits[PAGE_WORDS];
  __shared__ unsigned first[PAGED_MAX_LIST + 1];  // pages wanted before a sequence's ...
  __shared__ int slot[PAGED_MAX_LIST];            // ... which is the rank of its table's entry -slot
  __shared__ unsigned before[PNT];
  __shared__ Pair wsum[PNT / 64];
  const int tid = threadIdx.x, each = (m.n_seqs + PNT - 1) / PNT, s0 = tid * each, s1 = min(m.n_seqs, s0 + each);
  int grow[LPT], len[LPT];
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    const bool have = k < each && s0 + k < s1;
    grow[k] = have ? n_new[s0 + k] : 0;
    len[k] = have ? m.lengths[s0 + k] : 0;
  }
  load_bits(m.refs, m.n_pages, bits, true);
  unsigned need[LPT], want = 0;
  int held[LPT];
  bool bad = false;
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    if (grow[k] != 0 && (grow[k] < 0 || len[k] < 0 || (int64_t)len[k] + grow[k] > (int64_t)m.max_pages * m.page_size)) {
      grow[k] = 0;
      bad = true;
    }
    held[k] = grow[k] ? pages_of(len[k], m.page_size) : 0;
    need[k] = grow[k] ? (unsigned)(pages_of(len[k] + grow[k], m.page_size) - held[k]) : 0;
    want += need[k];  // (at most 2^12 sequences of 2^19 pages)
  }
  if (bad) atomicOr(m.err, (int)CRF_DEVERR_BATCH);
  const int words = (m.n_pages + 63) / 64, per = (words + PNT - 1) / PNT;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  unsigned free = 0;
  for (int w = w0; w < w1; ++w) free += __popcll(~bits[w]);
  Pair total, at = block_scan(want, free, wsum, total);
  before[tid] = at.b;
  bool none = false;
#pragma unroll
  for (int k = 0; k < LPT; ++k) {
    if (k >= each || s0 + k >= s1) continue;
    first[s0 + k] = at.a;
    slot[s0 + k] = held[k] - (int)at.a;
    at.a += need[k];
    const bool lack = need[k] && at.a > total.b;
    if (grow[k] && !lack) m.lengths[s0 + k] = len[k] + grow[k];
    none |= lack;
  }
  if (none) atomicOr(m.err, (int)CRF_DEVERR_PAGES);
  if (tid == 0) first[m.n_seqs] = total.a;
  __syncthreads();
  for (unsigned r = tid; r < min(total.a, total.b); r += PNT) {
    const int s = last_at_most(first, m.n_seqs, r);
    if (first[s + 1] > total.b) continue;
    const int page = page_of_rank(r, before, per, [&](int w) { return ~bits[w]; });
    m.tables[(int64_t)s * m.table_stride + slot[s] + (int)r] = page;
    m.refs[page] = 1;
  }
}

// ---------------------------------------------------------------- freeing

__global__ __launch_bounds__(CNT) void free_kernel(const PageMap m, int n, const int32_t *seqs) {
  __shared__ int len_s;
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = seqs[i];
    if (s < 0 || s >= m.n_seqs) {
      if (threadIdx.x == 0) atomicOr(m.err, (int)CRF_DEVERR_BATCH);
      continue;
    }
    __syncthreads();  // (the length before has been read)
    // (a sequence that is named twice is freed by whoever takes its length)
    if (threadIdx.x == 0) len_s = atomicExch(&m.lengths[s], 0);
    __syncthreads();
    const int len = len_s;
    if (len < 0 || (int64_t)len > (int64_t)m.max_pages * m.page_size) {
      if (threadIdx.x == 0) atomicOr(m.err, (int)CRF_DEVERR_BATCH);
      continue;
    }
    const int held = pages_of(len, m.page_size);
    for (int j = threadIdx.x; j < held; j += CNT) {
      const int e = m.tables[(int64_t)s * m.table_stride + j];
      if (e < 0 || e >= m.n_pages) {
        atomicOr(m.err, (int)CRF_DEVERR_BLOCK_TABLE);
      } else if (atomicSub(&m.refs[e], 1) <= 0) {  // held by nobody
        atomicAdd(&m.refs[e], 1);
        atomicOr(m.err, (int)CRF_DEVERR_BATCH);
      }
    }
  }
}

// ---------------------------------------------------------------- compacting

// With L pages in use, the k-th page in use at or past L moves to the k-th free
// page below L: no page is both a source and a destination, so the copies need no
// order and the old map stays readable until its pages are reused.
__global__ __launch_bounds__(PNT) void compact_plan_kernel(const PageMap m, int32_t *refs_out, int32_t *remap,
                                                           int32_t *moves, int32_t *counts) {
  __shared__ uint64_t bits[PAGE_WORDS];
  __shared__ unsigned holes_before[PNT], movers_before[PNT];
  __shared__ Pair wsum[PNT / 64];
  const int tid = threadIdx.x;
  load_bits(m.refs, m.n_pages, bits, false);
  const int words = (m.n_pages + 63) / 64, per = (words + PNT - 1) / PNT;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  unsigned count = 0;
  Pair total;
  for (int w = w0; w < w1; ++w) count += __popcll(bits[w]);
  (void)block_scan(count, 0, wsum, total);
  const int live = (int)total.a;
  // word w's pages below L
  auto below = [&](int w) {
    return 64 * w + 64 <= live ? ~(uint64_t)0 : 64 * w >= live ? 0 : ((uint64_t)1 << (live - 64 * w)) - 1;
  };
  auto hole = [&](int w) { return ~bits[w] & below(w); };
  auto mover = [&](int w) { return bits[w] & ~below(w); };
  unsigned holes = 0, movers = 0;
  for (int w = w0; w < w1; ++w) {
    holes += __popcll(hole(w));
    movers += __popcll(mover(w));
  }
  const Pair at = block_scan(holes, movers, wsum, total);
  holes_before[tid] = at.a;
  movers_before[tid] = at.b;
  if (tid == 0) {
    counts[0] = live;
    counts[1] = (int)total.b;
  }
  __syncthreads();
  for (unsigned k = tid; k < total.b; k += PNT) {
    const int src = page_of_rank(k, movers_before, per, mover), dst = page_of_rank(k, holes_before, per, hole);
    moves[2 * k] = src;
    moves[2 * k + 1] = dst;
    remap[src] = dst;
    refs_out[dst] = m.refs[src];
  }
  __syncthreads();  // (refs_out may be m.refs)
  for (int p0 = tid; p0 < m.n_pages; p0 += 8 * PNT) {
    int r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = p0 + k * PNT < live ? m.refs[p0 + k * PNT] : 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int p = p0 + k * PNT;
      if (p >= m.n_pages) break;
      const bool used = (bits[p / 64] >> (p % 64)) & 1;
      if (p >= live) refs_out[p] = 0;
      else if (used) refs_out[p] = r[k];
      if (p < live || !used) remap[p] = used ? p : -1;
    }
  }
}

// The first n_seqs workgroups rewrite a sequence's table each, the others copy.
__global__ __launch_bounds__(CNT) void compact_apply_kernel(const PageMap m, const PageMap out, const CopyArgs a,
                                                            const int32_t *remap, const int32_t *moves) {
  if ((int)blockIdx.x < m.n_seqs) {
    const int s = blockIdx.x, len = m.lengths[s];
    if (len < 0 || (int64_t)len > (int64_t)m.max_pages * m.page_size) {
      if (threadIdx.x == 0) atomicOr(m.err, (int)CRF_DEVERR_BATCH);
      return;
    }
    const int held = pages_of(len, m.page_size);
    for (int j = threadIdx.x; j < held; j += CNT) {
      const int e = m.tables[(int64_t)s * m.table_stride + j];
      const int to = e >= 0 && e < m.n_pages ? remap[e] : -1;
      if (to < 0) atomicOr(m.err, (int)CRF_DEVERR_BLOCK_TABLE);
      out.tables[(int64_t)s * out.table_stride + j] = to;
    }
    if (threadIdx.x == 0 && out.lengths != m.lengths) out.lengths[s] = len;
    return;
  }
  const int64_t blocks = (int64_t)*a.n_dev * a.blocks_per_pair;
  for (int64_t b = blockIdx.x - m.n_seqs; b < blocks; b += gridDim.x - m.n_seqs) {
    const int i = (int)(b / a.blocks_per_pair), part = (int)(b % a.blocks_per_pair);
    copy_pair(a, moves[2 * i], moves[2 * i + 1], part * CNT * CUN);
  }
}

// workgroups of a copy whose count only the device knows: eight to a CU
constexpr int COPY_GRID = 2048;

}  // namespace

hipError_t launch_pages_copy(hipStream_t s, const PagePools &from, const PagePools &to, int layers, int bytes, int n,
                             const int32_t *src, const int32_t *dst, int *err) {
  if (n <= 0 || layers <= 0) return hipSuccess;
  CopyArgs a = copy_args(from, to, layers, bytes, n, err);
  const int64_t blocks = (int64_t)n * a.blocks_per_pair;
  hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)(blocks < MOST_GROUPS ? blocks : MOST_GROUPS)), dim3(CNT), 0, s, a,
                     src, dst);
  return hipGetLastError();
}

hipError_t launch_pages_fork(hipStream_t s, const PageMap &m, const PagePools &pool, int layers, int bytes, int n,
                             const int32_t *parents, const int32_t *children, int32_t *state) {
  if (n <= 0) return hipSuccess;
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(PNT), 0, s, m, n, parents, children, state);
  const CopyArgs a = copy_args(pool, pool, layers, bytes, n, m.err);
  hipLaunchKernelGGL(fork_apply_kernel, dim3(1 + a.blocks_per_pair, n), dim3(CNT), 0, s, m, a, parents, children,
                     state);
  return hipGetLastError();
}

hipError_t launch_pages_extend(hipStream_t s, const PageMap &m, const int32_t *n_new) {
  if (m.n_seqs <= 0) return hipSuccess;
  hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(PNT), 0, s, m, n_new);
  return hipGetLastError();
}

hipError_t launch_pages_free(hipStream_t s, const PageMap &m, int n, const int32_t *seqs) {
  if (n <= 0) return hipSuccess;
  hipLaunchKernelGGL(free_kernel, dim3(n < MOST_GROUPS ? n : MOST_GROUPS), dim3(CNT), 0, s, m, n, seqs);
  return hipGetLastError();
}

hipError_t launch_pages_compact(hipStream_t s, const PageMap &in, const PageMap &out, const PagePools &pool, int layers,
                                int bytes, int32_t *remap, int32_t *moves, int32_t *counts) {
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(PNT), 0, s, in, out.refs, remap, moves, counts);
  CopyArgs a = copy_args(pool, pool, layers, bytes, in.n_pages / 2, in.err);
  a.n_dev = counts + 1;
  hipLaunchKernelGGL(compact_apply_kernel, dim3(in.n_seqs + COPY_GRID), dim3(CNT), 0, s, in, out, a, remap, moves);
  return hipGetLastError();
}

}  // namespace crf
