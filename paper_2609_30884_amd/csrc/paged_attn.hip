// Attention of the new tokens of many sequences over their pages of one cache.
//
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = 2^(c q_r . k_j - ref_r),  c = scale log2 e,
// over the keys j at or before the row's position (and within `window` of it).
//
// Rows: the G query heads of a KV head that read the same keys lie next to each
// other on the rows of a tile (row = token * G + head), so that a step of one token
// fills G rows and every K/V tile is loaded once for the group.  Lengths are read on
// the device; nothing about a sequence but bounds is known to the host.
//
// Two kernels share the arithmetic.
//   rows:  tiles of 128 rows, 4 waves of 32, all reading K/V tiles that the
//          workgroup stages together (compute bound: chunks of a prompt);
//   keys:  tiles of 32 rows, whose keys the waves share out, each staging its own
//          (HBM bound: single tokens and drafts).  Nothing but the page table is
//          shared while keys stream, so a wave never waits for another.
// Each wave computes S^T = K Q^T (keys on MFMA rows, query rows on columns), so a
// lane owns one query row and 16 of a block's 32 keys, and O^T = V^T P^T straight
// from those registers.  K and V go from the pages into LDS by loads with an LDS
// destination (64-bit addresses: a layer of a pool may pass 4 GiB), in 16-byte chunks
// XOR-swizzled by row.
//
// The reference ref is no running maximum: a block's probabilities are formed with
// the one there is, and only where a lane's sum passes 2^8 is the maximum taken and
// O rescaled.  It starts at minus infinity, which makes the first block that a row
// sees take that path.  Scores, sums and O are fp32; the probabilities are rounded
// to the storage type for the second product, as MFMA needs them (bf16: 2^-8
// of each weight at most), and summed before that rounding.
//
// Schedule: a unit is a row tile of one KV head of one sequence.  Few units: the
// work (keys times rows) is dealt out evenly, a contiguous stretch to each resident
// workgroup; a unit cut by a border leaves partials, which the workgroup that
// finishes last joins in the order of the keys (results do not depend on who that
// is).  Many: one unit a workgroup, longest of a sequence first.
#include <math.h>

#include <type_traits>

#include "paged.hpp"

namespace crf {
namespace {

constexpr float PSUM_MAX = 256.0f;  // a lane's sum of a block's probabilities that needs no new reference
constexpr int PGCAP = 2048;         // page numbers staged in LDS at a time
constexpr int ML_CAP = 2048;        // (reference, sum) pairs that a join holds in LDS
constexpr int MANY = 4;             // units per resident workgroup from which none is split
constexpr int MIN_KEYS = 256;       // keys that a workgroup is worth

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

CRF_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
CRF_DEV s16x4 ld_tr(const bf16 *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(const __attribute__((address_space(3))) void *)p);
}
CRF_DEV f32x16 mfma32f(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
// 16 bytes a lane from global memory to lds + 16 * lane
CRF_DEV void gload16(const char *g, void *lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

template <typename T, int HD>
struct Layout {
  static constexpr int ROWB = HD * (int)sizeof(T);  // bytes of a key's row
  static constexpr int CH = ROWB / 16;              // 16-byte chunks of it
  static constexpr int RPI = 64 / CH;               // rows that one load of a wave covers
  static constexpr int EPC = 16 / (int)sizeof(T);   // elements of a chunk
  static constexpr int KS = HD / (2 * EPC);         // steps of two chunks along a row
  static constexpr int HB = HD / 32;                // 32-row blocks of O^T
  // chunk slot of chunk c in K row r: conflict-free 16-byte reads of 8 rows
  static CRF_DEV int kslot(int r, int c) { return c ^ (r & (CH < 16 ? CH - 1 : 15)); }
  // and in V row r: bf16 transpose reads of 4 rows land on distinct banks; fp32
  // rows are read along the row
  static CRF_DEV int vslot(int r, int c) {
    if (sizeof(T) == 4) return c;
    if (HD == 128) return c ^ ((0xCA60 >> (4 * (r & 3))) & 15);
    return c ^ (2 * (r & 3));
  }
};

// A lane's query row: KS x 16 bytes.
template <typename T, int HD>
struct QFrag {
  u32x4 f[Layout<T, HD>::KS];
  CRF_DEV void load(const T *row, int g) {
#pragma unroll
    for (int s = 0; s < Layout<T, HD>::KS; ++s) f[s] = ld16(row + (2 * s + g) * Layout<T, HD>::EPC);
  }
};

// Raw scores of 32 keys (LDS rows r0 ..) against the wave's 32 rows.
template <typename T, int HD>
CRF_DEV f32x16 scores(const T *kt, int r0, const QFrag<T, HD> &q, int g, int l32) {
  using L = Layout<T, HD>;
  f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
  const int r = r0 + l32;
#pragma unroll
  for (int s = 0; s < L::KS; ++s) {
    const u32x4 k = ld16(kt + r * HD + L::kslot(r, 2 * s + g) * L::EPC);
    if constexpr (sizeof(T) == 2) {
      acc = mfma32(as_bf16x8(k), as_bf16x8(q.f[s]), acc);
    } else {
      const f32x4 a = __builtin_bit_cast(f32x4, k), b = __builtin_bit_cast(f32x4, q.f[s]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = mfma32f(a[e], b[e], acc);
    }
  }
  return acc;
}

// The keys that a lane's row sees: [lo, hi]; bad: some pages of the unit are out of
// range, whose keys nobody sees.
struct Seen {
  int lo, hi;
  bool bad;
  const int *pages;  // staged page numbers, the first of logical page `first`
  int first;
  FastDiv ps_div;
};

template <int HD>
struct RowState {
  f32x16 o[HD / 32];
  float ref, l;
  CRF_DEV void clear() {
#pragma unroll
    for (int b = 0; b < HD / 32; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[b][v] = 0.f;
    ref = -INFINITY;
    l = 0.f;
  }
};

CRF_DEV bool not_finite16(int h) { return (h & 0x7f80) == 0x7f80; }

// One block of 32 keys, key0 .. key0 + 31 in LDS rows r0 ..: scores, probabilities,
// O += P V.  MASK: some row does not see some key of it.  A value that is not finite
// takes no part in a row that does not see its key, though the product multiplies it
// by zero: where a masked block holds such values, they are taken out of the product
// and brought back where a weight is not zero.
template <typename T, int HD, bool MASK>
CRF_DEV void block32(const T *kt, const T *vt, int r0, int key0, const QFrag<T, HD> &q, RowState<HD> &st, float c,
                     int lane, const Seen &seen) {
  using L = Layout<T, HD>;
  const int g = lane / 32, l32 = lane % 32;
  f32x16 s = scores<T, HD>(kt, r0, q, g, l32);
  if constexpr (MASK) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = key0 + 8 * (v / 4) + 4 * g + v % 4;
      bool hide = key < seen.lo || key > seen.hi;
      if (seen.bad && !hide) hide = seen.pages[div_by(key, seen.ps_div) - seen.first] < 0;
      if (hide) s[v] = -INFINITY;
    }
  }
  float p[16], sum = 0.f;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    p[v] = fast_exp2(fmaf(s[v], c, -st.ref));
    sum += p[v];
  }
  if (__builtin_amdgcn_ballot_w64(!(sum <= PSUM_MAX))) {  // (also where the sum is no number)
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
    // only rows that need one: a row's result does not depend on the tile's others
    const float other = __shfl_xor(sum, 32, 64);
    const bool raise = !(sum <= PSUM_MAX) || !(other <= PSUM_MAX);
    const float ref = raise ? fmaxf(st.ref, mx) : st.ref;
    const float alpha = ref == -INFINITY ? 1.f : fast_exp2(st.ref - ref);
    const float base = ref == -INFINITY ? 0.f : ref;
    st.ref = ref;
    st.l *= alpha;
#pragma unroll
    for (int b = 0; b < L::HB; ++b) st.o[b] *= alpha;
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = fast_exp2(fmaf(s[v], c, -base));
      sum += p[v];
    }
  }
  st.l += sum;

  if constexpr (sizeof(T) == 2) {
    bf16x8 pf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[h][e] = f2bf(p[8 * h + e]);
    // transpose reads: 16-lane group t covers hd 16 (t & 1) .. + 15 of a 32-row block
    // and key rows 4 (t / 2) + 0..3; slots 4-7 hold the rows 8 further on
    const int tg = lane / 16;
    const int tk = 4 * (tg >> 1) + (lane % 16) / 4, th = 16 * (tg & 1) + 4 * (lane % 4);
#pragma unroll
    for (int b = 0; b < L::HB; ++b) {
      const int hd = 32 * b + th;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int ra = r0 + 16 * h + tk, rb = ra + 8;
        const s16x4 lo = ld_tr(vt + ra * HD + L::vslot(ra, hd / 8) * 8 + hd % 8);
        const s16x4 hi = ld_tr(vt + rb * HD + L::vslot(rb, hd / 8) * 8 + hd % 8);
        s16x4 x[2] = {lo, hi};
        if constexpr (MASK) {
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= not_finite16(lo[e]) || not_finite16(hi[e]);
          if (__builtin_amdgcn_ballot_w64(odd)) {
            s16x4 plus[2], minus[2], nan[2];
            bf16x8 on;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int w = (uint16_t)x[e / 4][e % 4];
              plus[e / 4][e % 4] = w == 0x7f80 ? 0x3f80 : 0;
              minus[e / 4][e % 4] = w == 0xff80 ? 0x3f80 : 0;
              nan[e / 4][e % 4] = not_finite16(w) && (w & 0x7f) ? 0x3f80 : 0;
              if (not_finite16(w)) x[e / 4][e % 4] = 0;
              on[e] = (float)pf[h][e] != 0.f ? f2bf(1.f) : f2bf(0.f);
            }
            auto add = [&](const s16x4 (&ind)[2], float value) {
              f32x16 n;
#pragma unroll
              for (int v = 0; v < 16; ++v) n[v] = 0.f;
              n = mfma32(__builtin_bit_cast(bf16x8, ind), on, n);
#pragma unroll
              for (int v = 0; v < 16; ++v)
                if (n[v] > 0.f) st.o[b][v] += value;
            };
            add(plus, INFINITY);
            add(minus, -INFINITY);
            add(nan, NAN);
          }
        }
        st.o[b] = mfma32(__builtin_bit_cast(bf16x8, x), pf[h], st.o[b]);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = r0 + 8 * (v / 4) + 4 * g + v % 4;
#pragma unroll
      for (int b = 0; b < L::HB; ++b) {
        float x = vt[r * HD + 32 * b + l32];
        if constexpr (MASK) {
          const bool odd = (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) == 0x7f800000u;
          if (__builtin_amdgcn_ballot_w64(odd)) {
            const float on = p[v] != 0.f ? 1.f : 0.f;
            auto add = [&](bool is, float value) {
              f32x16 n;
#pragma unroll
              for (int w = 0; w < 16; ++w) n[w] = 0.f;
              n = mfma32f(is ? 1.f : 0.f, on, n);
#pragma unroll
              for (int w = 0; w < 16; ++w)
                if (n[w] > 0.f) st.o[b][w] += value;
            };
            add(x == INFINITY, INFINITY);
            add(x == -INFINITY, -INFINITY);
            add(x != x, NAN);
            if (odd) x = 0.f;
          }
        }
        st.o[b] = mfma32f(x, p[v], st.o[b]);
      }
    }
  }
}

// ---------------------------------------------------------------- schedule

// Row tiles of a sequence and their work in key x row units, a straight line in the
// tile (its keys end where its tokens do) up to a ceiling given by the window:
// work(t) = min(base + (t + 1) BM, cap) + over.
struct SeqWork {
  int64_t base, cap, over;
  int tiles, bm;
  __host__ __device__ int64_t before(int t) const {  // work of the tiles before t
    const int64_t room = cap - base;
    const int64_t k = room <= 0 ? 0 : room / bm < t ? room / bm : t;
    return k * base + bm * (k * (k + 1) / 2) + (t - k) * cap + t * over;
  }
};

// A unit, or the part of one, that a workgroup computes.
struct Task {
  int seq, kvh, tile;
  int start, n, len;  // first row, new tokens and whole length of the sequence
  int t0, t1;         // key tiles of the part
  int parts, part;    // parts of the unit and which this is
  int owner;          // workgroup of the unit's first part
};

struct Shape {
  int G, nkv, window, bm, bkv;  // query heads of a KV head; rows and keys of a tile

  __host__ __device__ SeqWork work(int n, int len) const {
    SeqWork w;
    w.tiles = (int)(((int64_t)n * G + bm - 1) / bm);
    w.bm = bm;
    w.base = (int64_t)(len - n) * G;
    w.cap = window > 0 ? (int64_t)window * G + bm : INT64_MAX / 4;
    w.over = (int64_t)bkv * G;
    return w;
  }
  __host__ __device__ int64_t seq_work(int n, int len) const {
    const SeqWork w = work(n, len);
    return w.before(w.tiles) * nkv;
  }
  __host__ __device__ int first_key(const Task &t) const {  // of the tile's first row
    const int pos = t.len - t.n + (int)((int64_t)t.tile * bm / G);
    return window > 0 && pos >= window ? pos - window + 1 : 0;
  }
  __host__ __device__ int last_key(const Task &t) const {  // of the tile's last row
    const int64_t r = ((int64_t)t.tile + 1) * bm, rows = (int64_t)t.n * G;
    return t.len - t.n + (int)(((r < rows ? r : rows) - 1) / G);
  }
  // Unit i of the sequence's, whole: longest first, its KV heads next to each other.
  __host__ __device__ void whole(int64_t i, Task &t) const {
    t.kvh = (int)(i % nkv);
    t.tile = work(t.n, t.len).tiles - 1 - (int)(i / nkv);
    t.t0 = first_key(t) / bkv;
    t.t1 = last_key(t) / bkv + 1;
    t.parts = 1;
  }
  // What workgroup wg, whose stretch ends at `end`, computes from position `at` of
  // all work on, `at` being in the sequence, whose work begins at seq_base; returns
  // where it stops (the end of the unit or of the stretch).
  __host__ __device__ int64_t part_at(int64_t at, int64_t end, int64_t share, int wg, int64_t seq_base, Task &t) const {
    const SeqWork w = work(t.n, t.len);
    const int64_t one = w.before(w.tiles), off = at - seq_base;
    t.kvh = (int)(off / one);
    const int64_t rem = off - t.kvh * one;
    int lo = 0, hi = w.tiles;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (w.before(mid) <= rem) lo = mid;
      else hi = mid;
    }
    t.tile = lo;
    const int64_t u0 = seq_base + t.kvh * one + w.before(lo), cost = w.before(lo + 1) - w.before(lo), u1 = u0 + cost;
    const int64_t stop = u1 < end ? u1 : end;
    const int k0 = first_key(t) / bkv, k = last_key(t) / bkv + 1 - k0;
    t.t0 = k0 + (int)((at - u0) * k / cost);
    t.t1 = stop == u1 ? k0 + k : k0 + (int)((stop - u0) * k / cost);
    t.owner = (int)(u0 / share);
    t.parts = (int)((u1 - 1) / share) - t.owner + 1;
    t.part = wg - t.owner;
    return stop;
  }
};

// Work of a workgroup when `total` is dealt out to at most `slots`, and how many get any.
__host__ __device__ inline void deal(int64_t total, int64_t least, int slots, int64_t &share, int &n_wg) {
  const int64_t want = total / least < 1 ? 1 : total / least < slots ? total / least : slots;
  share = (total + want - 1) / want;
  n_wg = (int)((total + share - 1) / share);
}

// Stretch of workgroup `bid`: neighbouring stretches, which share keys, lie on one
// XCD (bid % 8); -1: none.
__host__ __device__ inline int stretch_of(int bid, int n_wg) {
  const int per = (n_wg + 7) / 8, wg = (bid % 8) * per + bid / 8;
  return bid / 8 < per && wg < n_wg ? wg : -1;
}

// Partials lie in two slots a workgroup: the unit that its stretch begins inside,
// and the one that begins in its stretch and goes on past it.
__host__ __device__ inline int part_slot(int owner, int part) { return part == 0 ? 2 * owner + 1 : 2 * (owner + part); }

template <int NT>
struct Scan {
  int64_t wsum[NT / 64];
  // exclusive prefix of v over the workgroup, *total the sum
  CRF_DEV int64_t run(int64_t v, int64_t *total) {
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) wsum[w] = x;
    __syncthreads();
    int64_t at = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      if (i < w) at += wsum[i];
      sum += wsum[i];
    }
    *total = sum;
    return at + x - v;
  }
};

template <int NT>
struct Schedule {
  const PagedAttn &p;
  Scan<NT> &scan;
  int &found;
  int64_t &found_base;
  Shape sh;
  bool many;
  int wg;
  int64_t share, at, end;  // many: next unit and their number; else the stretch [at, end) of all work
  int seq;                 // sequence that holds `at`, -1 before the first search
  int64_t seq_base;        // where its work begins

  // Sums the batch and takes this workgroup's stretch; false: nothing to do.
  CRF_DEV bool begin(int slots) {
    int64_t w = 0, u = 0, total_w, total_u;
    for (int s = threadIdx.x; s < p.b.n_seqs; s += NT) {
      int start, len;
      const int n = seq_new(p.b, s, start, len);
      if (n == 0) continue;
      w += sh.seq_work(n, len);
      u += (int64_t)sh.work(n, len).tiles * sh.nkv;
    }
    (void)scan.run(w, &total_w);
    (void)scan.run(u, &total_u);
    many = slots == 0 || total_u >= (int64_t)MANY * slots;
    seq = -1;
    if (many) {
      at = blockIdx.x;
      end = total_u;
      return at < end;
    }
    if (total_w == 0) return false;
    int n_wg;
    deal(total_w, (int64_t)MIN_KEYS * sh.G, slots, share, n_wg);
    wg = stretch_of(blockIdx.x, n_wg);
    if (wg < 0) return false;
    at = wg * share;
    end = at + share < total_w ? at + share : total_w;
    return true;
  }

  // Sequence that holds position x of the prefix sums of f(new tokens, length).
  template <typename F>
  CRF_DEV void find(int64_t x, F f) {
    int64_t done = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += NT) {
      const int s = s0 + threadIdx.x;
      int start, len;
      const int n = s < p.b.n_seqs ? seq_new(p.b, s, start, len) : 0;
      const int64_t v = n > 0 ? f(n, len) : 0;
      int64_t total;
      const int64_t b = done + scan.run(v, &total);
      if (v > 0 && x >= b && x < b + v) {
        found = s;
        found_base = b;
      }
      done += total;
      if (x < done) break;
    }
    __syncthreads();
    seq = __builtin_amdgcn_readfirstlane(found);
    const int64_t b = found_base;
    seq_base = ((int64_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32) |
               (uint32_t)__builtin_amdgcn_readfirstlane((int)b);
  }

  // The next task; false: done.
  CRF_DEV bool next(Task &t) {
    if (at >= end) return false;
    if (many) {
      find(at, [&](int n, int len) { return (int64_t)sh.work(n, len).tiles * sh.nkv; });
      t.seq = seq;
      t.n = seq_new(p.b, seq, t.start, t.len);
      sh.whole(at - seq_base, t);
      at += gridDim.x;
      return true;
    }
    if (seq < 0) {
      find(at, [&](int n, int len) { return sh.seq_work(n, len); });
      t.n = seq_new(p.b, seq, t.start, t.len);
    } else {
      for (;; ++seq) {  // (`at` is before the end of all work, so some sequence holds it)
        t.n = seq_new(p.b, seq, t.start, t.len);
        const int64_t w = t.n > 0 ? sh.seq_work(t.n, t.len) : 0;
        if (at < seq_base + w) break;
        seq_base += w;
      }
    }
    t.seq = seq;
    at = sh.part_at(at, end, share, wg, seq_base, t);
    return true;
  }
};

template <typename T, int HD>
struct Writer {
  const PagedAttn &p;
  const Task &t;
  int G, row0, rows;  // first row of the tile and its rows

  CRF_DEV void locate(int r, int64_t &token, int &head) const {
    const int a = row0 + r;
    token = t.start + a / G;
    head = t.kvh * G + a % G;
  }
  // four elements from e on of the tile's row r: o / l, and the row's log-sum
  CRF_DEV void out4(int r, int e, f32x4 o, float ref, float l) const {
    int64_t token;
    int head;
    locate(r, token, head);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *dst = (T *)p.out + token * p.out_ld + head * HD + e;
    o *= inv;
    if constexpr (sizeof(T) == 2)
      st8(dst, pack_bf16x4(o[0], o[1], o[2], o[3]));
    else
      *reinterpret_cast<f32x4 *>(dst) = o;
    if (e == 0 && p.lse)
      p.lse[token * p.nq + head] = l == 0.f ? -INFINITY : 0.69314718055994531f * (ref + log2f(l));
  }
  template <int BM>
  CRF_DEV float *part_row(int slot, int r) const {
    return p.part + ((int64_t)slot * BM + r) * (HD + 4);
  }
};

// Counts this workgroup's part of the unit as done; the one that finishes last
// joins all parts.  ml: ML_CAP pairs of LDS that nobody uses.
template <typename T, int HD, int BM, int NT>
CRF_DEV void join(const Writer<T, HD> &wr, const Task &t, float2 *ml, int &last) {
  const PagedAttn &p = wr.p;
  const int tid = threadIdx.x;
  agent_flush();
  __syncthreads();
  if (tid == 0) {
    last = agent_ticket(&p.tickets[t.owner]) == (unsigned)t.parts - 1;
    if (last)
      __hip_atomic_store(&p.tickets[t.owner], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  const int step = ML_CAP / t.parts;  // rows joined at a time
  for (int r0 = 0; r0 < wr.rows; r0 += step) {
    const int rows = min(step, wr.rows - r0);
    for (int i = tid; i < rows * t.parts; i += NT) {
      const int part = i % t.parts, r = r0 + i / t.parts;
      const uint64_t u = __hip_atomic_load((const uint64_t *)(wr.template part_row<BM>(part_slot(t.owner, part), r) + HD),
                                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      ml[i] = make_float2(__builtin_bit_cast(float, (uint32_t)u), __builtin_bit_cast(float, (uint32_t)(u >> 32)));
    }
    __syncthreads();
    for (int i = tid; i < rows * (HD / 4); i += NT) {
      const int r = i / (HD / 4), e = 4 * (i % (HD / 4));
      const float2 *m = ml + r * t.parts;
      float ref = -INFINITY, l = 0.f;
      for (int k = 0; k < t.parts; ++k) ref = fmaxf(ref, m[k].x);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int k = 0; k < t.parts; ++k) {
        if (m[k].y == 0.f) continue;  // (a part of which the row sees nothing)
        const float w = fast_exp2(m[k].x - ref);
        l += w * m[k].y;
        o += w * ld_agent16(wr.template part_row<BM>(part_slot(t.owner, k), r0 + r) + e);
      }
      wr.out4(r0 + r, e, o, ref, l);
    }
    __syncthreads();
  }
}

CRF_DEV void st_ml(float *p, float ref, float l) {
  __hip_atomic_store((uint64_t *)p,
                     (uint64_t)__builtin_bit_cast(uint32_t, ref) | (uint64_t)__builtin_bit_cast(uint32_t, l) << 32,
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---------------------------------------------------------------- keys and values from the pages

// Stages page numbers and loads rows of keys and values.
template <typename T, int HD, bool UNI>
struct Pages {
  using L = Layout<T, HD>;
  const PagedBatch &b;
  const char *zeros;
  int *pg;     // LDS, PGCAP numbers: logical page first + i
  int *bad;    // LDS: some page of the unit is out of range
  int first, len, kvh;
  const int32_t *table;

  CRF_DEV void fill(int page, int end_key, int nt) {  // pages page .. that hold keys before end_key
    first = page;
    const int last = div_by(min(end_key, len) - 1, b.ps_div);
    for (int i = threadIdx.x; i < PGCAP && page + i <= last; i += nt) {
      int q = table[page + i];
      if (q < 0 || q >= b.n_pages) {
        atomicOr(b.err, (int)CRF_DEVERR_BLOCK_TABLE);
        q = -1;
        *bad = 1;
      }
      pg[i] = q;
    }
  }

  // ROWS keys from key0 on (a multiple of ROWS) to LDS rows lds_row0 ..; keys past the
  // sequence and on pages out of range arrive as zeros.  Always 2 * ROWS / RPI loads.
  template <int ROWS>
  CRF_DEV void load(int key0, T *kdst, T *vdst, int lds_row0, int lane) const {
    const int lrow = lane / L::CH, lslot = lane % L::CH;
    constexpr int GRP = ROWS < 16 ? ROWS : 16;  // rows that share a page when page_size % 16 == 0
#pragma unroll
    for (int g0 = 0; g0 < ROWS; g0 += GRP) {
      const int kg = key0 + g0;
      bool whole = false;
      int64_t off = 0;
      if (UNI) {
        const int lp = div_by(kg, b.ps_div);
        const int q = kg < len ? __builtin_amdgcn_readfirstlane(pg[lp - first]) : -1;
        whole = q >= 0 && kg + GRP <= len;
        off = (int64_t)q * b.page_bytes + ((int64_t)kvh * b.page_size + (kg - lp * b.page_size)) * L::ROWB;
      }
      if (whole) {
        const char *kb = b.k + off, *vb = b.v + off;
#pragma unroll
        for (int i = 0; i < GRP; i += L::RPI) {
          const int row = i + lrow, tr = lds_row0 + g0 + row;
          gload16(kb + (uint32_t)(row * L::ROWB + L::kslot(tr, lslot) * 16), kdst + (lds_row0 + g0 + i) * HD);
          gload16(vb + (uint32_t)(row * L::ROWB + L::vslot(tr, lslot) * 16), vdst + (lds_row0 + g0 + i) * HD);
        }
      } else {
#pragma unroll
        for (int i = 0; i < GRP; i += L::RPI) {
          const int row = i + lrow, tr = lds_row0 + g0 + row, key = kg + row;
          int q = -1, slot = 0;
          if (key < len) {
            const int lp = div_by(key, b.ps_div);
            q = pg[lp - first];
            slot = key - lp * b.page_size;
          }
          const int64_t o = (int64_t)q * b.page_bytes + ((int64_t)kvh * b.page_size + slot) * L::ROWB;
          const char *kp = q >= 0 ? b.k + o + L::kslot(tr, lslot) * 16 : zeros;
          const char *vp = q >= 0 ? b.v + o + L::vslot(tr, lslot) * 16 : zeros;
          gload16(kp, kdst + (lds_row0 + g0 + i) * HD);
          gload16(vp, vdst + (lds_row0 + g0 + i) * HD);
        }
      }
    }
  }
};

// ---------------------------------------------------------------- tiles of 128 rows

template <typename T, int HD, bool UNI>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(const PagedAttn p, int slots) {
  using L = Layout<T, HD>;
  constexpr int NW = 4, NT = 64 * NW, BM = 32 * NW, BKV = sizeof(T) == 2 ? 64 : 32, TILE = BKV * HD;
  __shared__ __align__(16) T ks0[TILE], ks1[TILE], vs0[TILE], vs1[TILE];
  __shared__ int pg[PGCAP];
  __shared__ int bad, last, found;
  __shared__ int64_t found_base;
  __shared__ Scan<NT> scan;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  Schedule<NT> sch{p, scan, found, found_base, Shape{p.nq / p.nkv, p.nkv, p.window, BM, BKV}};
  if (!sch.begin(slots)) return;
  const int G = sch.sh.G;
  Task t;
  while (sch.next(t)) {
    const int rows = min((int64_t)BM, (int64_t)t.n * G - (int64_t)t.tile * BM);
    const Writer<T, HD> wr{p, t, G, t.tile * BM, rows};
    const int base = t.len - t.n;
    // this lane's row (padding rows repeat the last one)
    const int r = wave * 32 + l32, row = t.tile * BM + min(r, rows - 1);
    const int tok = row / G, head = t.kvh * G + row % G, pos = base + tok;
    const int pos_lo = base + (t.tile * BM + min(wave * 32, rows - 1)) / G;
    const int pos_hi = base + (t.tile * BM + min(wave * 32 + 31, rows - 1)) / G;
    QFrag<T, HD> q;
    q.load((const T *)p.q + (int64_t)(t.start + tok) * p.q_ld + head * HD, g);
    RowState<HD> st;
    st.clear();
    Pages<T, HD, UNI> pages{p.b, p.zeros, pg, &bad, 0, t.len, t.kvh, p.b.tables + (int64_t)t.seq * p.b.table_stride};
    const int far = p.window > 0 ? p.window - 1 : INT32_MAX;  // keys before its own that a row sees
    const int first_seen = pos_lo > far ? pos_lo - far : 0, last_first = pos_hi > far ? pos_hi - far : 0;
    __syncthreads();  // the task before has left LDS
    if (tid == 0) bad = 0;
    __syncthreads();
    const int end_key = t.t1 * BKV;

    auto tile = [&](int it, const T *kt, const T *vt, T *kn, T *vn) {
      const int kt0 = it * BKV;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (it + 1 < t.t1) {
        if (div_by(min(kt0 + 2 * BKV, t.len) - 1, p.b.ps_div) >= pages.first + PGCAP) {
          pages.fill(div_by(kt0, p.b.ps_div), end_key, NT);
          __syncthreads();
        }
        pages.template load<BKV / NW>(kt0 + BKV + wave * (BKV / NW), kn, vn, wave * (BKV / NW), lane);
      }
      if (wave * 32 >= rows || kt0 > pos_hi || kt0 + BKV <= first_seen) return;
      const Seen seen{pos > far ? pos - far : 0, pos, bad != 0, pg, pages.first, p.b.ps_div};
      if (kt0 + BKV - 1 > pos_lo || kt0 < last_first || bad) {
#pragma unroll
        for (int kb = 0; kb < BKV; kb += 32)
          block32<T, HD, true>(kt, vt, kb, kt0 + kb, q, st, p.scale_log2, lane, seen);
      } else {
#pragma unroll
        for (int kb = 0; kb < BKV; kb += 32)
          block32<T, HD, false>(kt, vt, kb, kt0 + kb, q, st, p.scale_log2, lane, seen);
      }
    };

    if (t.t0 < t.t1) {
      pages.fill(div_by(t.t0 * BKV, p.b.ps_div), end_key, NT);
      __syncthreads();
      pages.template load<BKV / NW>(t.t0 * BKV + wave * (BKV / NW), ks0, vs0, wave * (BKV / NW), lane);
    }
    for (int it = t.t0; it < t.t1; it += 2) {
      tile(it, ks0, vs0, ks1, vs1);
      if (it + 1 < t.t1) tile(it + 1, ks1, vs1, ks0, vs0);
    }

    const float l = st.l + __shfl_xor(st.l, 32, 64);
    if (t.parts == 1) {
      if (r < rows)
#pragma unroll
        for (int b = 0; b < L::HB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            wr.out4(r, 32 * b + 8 * i + 4 * g,
                    f32x4{st.o[b][4 * i], st.o[b][4 * i + 1], st.o[b][4 * i + 2], st.o[b][4 * i + 3]}, st.ref, l);
      continue;
    }
    if (r < rows) {
      float *dst = wr.template part_row<BM>(part_slot(t.owner, t.part), r);
#pragma unroll
      for (int b = 0; b < L::HB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          st_agent16(dst + 32 * b + 8 * i + 4 * g,
                     f32x4{st.o[b][4 * i], st.o[b][4 * i + 1], st.o[b][4 * i + 2], st.o[b][4 * i + 3]});
      if (g == 0) st_ml(dst + HD, st.ref, l);
    }
    join<T, HD, BM, NT>(wr, t, (float2 *)vs0, last);
  }
}

// ---------------------------------------------------------------- tiles of 32 rows, keys shared out

template <typename T, int HD>
struct KeysCfg {
  // (fp32 heads of 128: two waves' two stages of 32 keys fill the LDS that four take else)
  static constexpr int NW = sizeof(T) * HD > 256 ? 2 : 4;
  static constexpr int WG_PER_CU = sizeof(T) * HD * NW * 128 > 65536 ? 1 : 2;
};

template <typename T, int HD, bool UNI>
__global__ __launch_bounds__((64 * KeysCfg<T, HD>::NW)) void attn_keys_kernel(const PagedAttn p, int slots) {
  using L = Layout<T, HD>;
  constexpr int NW = KeysCfg<T, HD>::NW, NT = 64 * NW, BM = 32, BKV = 32 * NW, TILE = BKV * HD;
  constexpr int LOADS = 2 * 32 / L::RPI;  // of a wave's stage
  __shared__ __align__(16) T ks0[TILE], ks1[TILE], vs0[TILE], vs1[TILE];
  __shared__ int pg[PGCAP];
  __shared__ float2 wml[NW][32];
  __shared__ int bad, last, found;
  __shared__ int64_t found_base;
  __shared__ Scan<NT> scan;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  Schedule<NT> sch{p, scan, found, found_base, Shape{p.nq / p.nkv, p.nkv, p.window, BM, BKV}};
  if (!sch.begin(slots)) return;
  const int G = sch.sh.G;
  Task t;
  while (sch.next(t)) {
    const int rows = min((int64_t)BM, (int64_t)t.n * G - (int64_t)t.tile * BM);
    const Writer<T, HD> wr{p, t, G, t.tile * BM, rows};
    const int base = t.len - t.n;
    const int row = t.tile * BM + min(l32, rows - 1);
    const int tok = row / G, head = t.kvh * G + row % G, pos = base + tok;
    const int pos_lo = base + t.tile * BM / G, pos_hi = base + (t.tile * BM + rows - 1) / G;
    QFrag<T, HD> q;
    q.load((const T *)p.q + (int64_t)(t.start + tok) * p.q_ld + head * HD, g);
    RowState<HD> st;
    st.clear();
    Pages<T, HD, UNI> pages{p.b, p.zeros, pg, &bad, 0, t.len, t.kvh, p.b.tables + (int64_t)t.seq * p.b.table_stride};
    const int far = p.window > 0 ? p.window - 1 : INT32_MAX;
    const int first_seen = pos_lo > far ? pos_lo - far : 0, last_first = pos_hi > far ? pos_hi - far : 0;
    __syncthreads();
    if (tid == 0) bad = 0;
    __syncthreads();

    // stretches of tiles whose pages fit the staged table
    for (int a = t.t0; a < t.t1;) {
      const int fp = div_by(a * BKV, p.b.ps_div);
      const int64_t keys = ((int64_t)fp + PGCAP) * p.b.page_size;  // end of the staged pages
      const int z = keys / BKV < t.t1 ? (int)(keys / BKV) : t.t1;
      pages.fill(fp, z * BKV, NT);
      __syncthreads();
      const bool odd = bad != 0;
      const Seen seen{pos > far ? pos - far : 0, pos, odd, pg, fp, p.b.ps_div};
      auto load = [&](int it, T *k, T *v) { pages.template load<32>(it * BKV + wave * 32, k, v, wave * 32, lane); };
      auto step = [&](int it, T *k, T *v) {
        if (it + 1 < z)
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const int key0 = it * BKV + wave * 32;
        if (key0 <= pos_hi && key0 + 32 > first_seen) {
          if (key0 + 31 > pos_lo || key0 < last_first || odd)
            block32<T, HD, true>(k, v, wave * 32, key0, q, st, p.scale_log2, lane, seen);
          else
            block32<T, HD, false>(k, v, wave * 32, key0, q, st, p.scale_log2, lane, seen);
        }
        // the stage is read before it is loaded again
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (it + 2 < z) load(it + 2, k, v);
      };
      load(a, ks0, vs0);
      if (a + 1 < z) load(a + 1, ks1, vs1);
      for (int it = a; it < z; it += 2) {
        step(it, ks0, vs0);
        if (it + 1 < z) step(it + 1, ks1, vs1);
      }
      a = z;
      __syncthreads();
    }

    // join the waves: O of wave w at 32 x HD floats w of ks0 and ks1
    const float lw = st.l + __shfl_xor(st.l, 32, 64);
    auto osum = [&](int w) {
      constexpr int PER = (int)(sizeof(T) * TILE / (32 * HD * 4));  // waves' O in one array
      return (f32x4 *)(w < PER ? ks0 : ks1) + (w % PER) * 32 * (HD / 4);
    };
    {
      f32x4 *o = osum(wave);
#pragma unroll
      for (int b = 0; b < L::HB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[l32 * (HD / 4) + ((8 * b + 2 * i + g) ^ (l32 & 15))] =
              f32x4{st.o[b][4 * i], st.o[b][4 * i + 1], st.o[b][4 * i + 2], st.o[b][4 * i + 3]};
      if (g == 0) wml[wave][l32] = make_float2(st.ref, lw);
    }
    __syncthreads();
    for (int i = tid; i < rows * (HD / 4); i += NT) {
      const int r = i / (HD / 4), c4 = i % (HD / 4);
      float ref = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) ref = fmaxf(ref, wml[w][r].x);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 m = wml[w][r];
        if (m.y == 0.f) continue;
        const float k = fast_exp2(m.x - ref);
        l += k * m.y;
        o += k * osum(w)[r * (HD / 4) + (c4 ^ (r & 15))];
      }
      if (t.parts == 1) {
        wr.out4(r, 4 * c4, o, ref, l);
      } else {
        float *dst = wr.template part_row<BM>(part_slot(t.owner, t.part), r);
        st_agent16(dst + 4 * c4, o);
        if (c4 == 0) st_ml(dst + HD, ref, l);
      }
    }
    if (t.parts > 1) join<T, HD, BM, NT>(wr, t, (float2 *)vs0, last);
  }
}

template <typename T, int HD, bool UNI>
hipError_t launch(hipStream_t s, const PagedAttn &p) {
  const int G = p.nq / p.nkv;
  // up to 32 rows to a sequence and KV head: the keys are shared out
  const bool keys = (int64_t)p.b.max_new * G <= 32;
  const int bm = keys ? 32 : 128;
  const int resident = p.n_cu * (keys ? KeysCfg<T, HD>::WG_PER_CU : 2);
  const int64_t room = p.part ? p.part_floats / (2 * bm * (HD + 4)) : 0;  // two slots a workgroup
  int slots = (int)(room < resident ? room : resident);
  if (slots > PAGED_TICKETS) slots = PAGED_TICKETS;
  slots = slots / 8 * 8;
  // (a sequence's last tile may be short)
  const int64_t most = ((int64_t)p.b.n_rows * G / bm + p.b.n_seqs) * p.nkv;
  const int64_t grid = most < (int64_t)MANY * slots ? slots : most;
  if (grid < 1) return hipSuccess;
  const dim3 g((unsigned)(grid < (1 << 24) ? grid : 1 << 24));
  if (keys)
    hipLaunchKernelGGL((attn_keys_kernel<T, HD, UNI>), g, dim3(64 * KeysCfg<T, HD>::NW), 0, s, p, slots);
  else
    hipLaunchKernelGGL((attn_rows_kernel<T, HD, UNI>), g, dim3(256), 0, s, p, slots);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_uni(hipStream_t s, const PagedAttn &p) {
  return p.b.page_size % 16 == 0 ? launch<T, HD, true>(s, p) : launch<T, HD, false>(s, p);
}

}  // namespace

hipError_t launch_paged_attn(hipStream_t s, bool f32, const PagedAttn &p) {
  if (p.b.n_seqs <= 0 || p.b.n_rows <= 0) return hipSuccess;
  if (f32) return p.hd == 128 ? launch_uni<float, 128>(s, p) : launch_uni<float, 64>(s, p);
  return p.hd == 128 ? launch_uni<bf16, 128>(s, p) : launch_uni<bf16, 64>(s, p);
}

}  // namespace crf
