// Attention of a batch whose sequences share long prefixes: the keys and values of a
// group's first tokens are read once for all of its sequences' new tokens.
//
//   o_r = sum_j p_rj v_j / sum_j p_rj  as in attention over the pages, the keys of a row
// being its group's shared ones and its sequence's own.  The sum over the keys is cut into
// parts, each with its reference, sum and O, which are joined at the end.
//
// Two launches.  The first computes the parts: an item is a group's shared keys with the
// new tokens of all its sequences (neighbours among the rows) on the rows, or a sequence's
// own keys with its own new tokens; a unit is a tile of 128 rows of one KV head of an item
// and a chunk of its keys.  The chunk's length follows from all the items, which every
// workgroup works out from the lengths on the device, an item a thread.  A row sees the keys up
// to its own position, also among the shared ones, so that a group whose sequences are shorter
// than it says is right all the same.  The second launch joins each row's parts, in the order
// of the keys.
//
// Measured (bf16, heads of 128), against each sequence reading the shared keys itself:
//   64 next tokens, four documents of 4096 to 16384 with 16 sequences each, 20 to 500 keys of
//     their own, 28/4 heads    48 us against 171, three batches in turn (one or two, which the
//     memory-side cache holds, 40): 4.4 us until a workgroup knows its unit, 4.5 until its
//     first keys are there, 24 for 118 MB (4.9 TB/s), 3 to store the parts, 7 for the second
//     launch;
//   32 about one of 16384    33 us against 83;
//   four about one of 16384    28 against 36: the same chain;
//   two times eight drafts of 8 over 8192    46 against 73: products of full tiles on half of the
//     workgroups that stay resident (choose() below), 13 at the rate of a large matrix product;
//   fp32, four times eight next tokens over 3000, 3/1 heads    38 against 50.
// Tried when the first of these took 48 to 49 us: four stages of 32 keys instead of two of 64, 51;
// parts stored whole rows at a time by way of LDS, 54; a body for up to 32 rows whose keys the
// waves share out, 55 (it spills); a chunk chosen so that one round of workgroups just holds all
// units, 50.
#include <math.h>

#include <algorithm>

#include "paged_tiles.hpp"
#include "serving.hpp"

namespace crf {
namespace {

constexpr int NW = 4, NT = 64 * NW, BM = 32 * NW;
// Key tiles of a chunk, at least.  2: two sequences over 8192 24 us instead of 23, eight over
// 3000 20.8 instead of 19.8 (more parts to join).
constexpr int SHORTEST = 4;
// Bytes of K and V that the sequences read by themselves at most, as far as the host can tell,
// up to which they do.  Shared against by themselves, us: 25 MB (eight sequences over 3000,
// 12/2 heads) 19.8 / 18.4, 34 MB (two over 8192, 28/4 heads) 23.2 / 21.7, 82 MB (200 over 300,
// 12/2) 23.5 / 25.9, 135 MB (four over 16384, 28/4) 28.0 / 35.7.
constexpr int64_t SMALL_READS = 40 << 20;
constexpr int LONGEST = 1 << 26;  // more than any sequence has

// What the second launch needs of a sequence: its new tokens, and the parts of its own keys and
// of its group's shared ones.
struct Parts {
  int base, chunks, row0, n;  // first row of the parts, chunks of the keys, first token and tokens of the item
};
struct Info {
  Parts own, shared;
};

// Items 0 .. n_groups - 1 are the groups' shared keys, the others the sequences' own.
struct Item {
  int row0, n;  // new tokens
  int lo, hi;   // keys
  int seq;      // whose block table names them
  int group;    // of a sequence that shares (else -1)
};

// The groups in LDS: first sequences (n + 1), shared lengths, rows, and where their parts lie.
struct Groups {
  int *start, *shared, *row0, *rows, *base, *chunks;
  int n;
  static constexpr int WORDS = 6 * (SHARED_MAX_GROUPS + 1);
  CRF_DEV Groups(int *lds, int groups) : n(groups) {
    int **const all[6] = {&start, &shared, &row0, &rows, &base, &chunks};
#pragma unroll
    for (int i = 0; i < 6; ++i) *all[i] = lds + i * (SHARED_MAX_GROUPS + 1);
  }
  // Group g; one that contradicts the batch is flagged and shares nothing.
  CRF_DEV void stage(const SharedAttn &p, int g) const {
    const PagedBatch &b = p.a.b;
    const int s0 = p.seq_start[g], s1 = p.seq_start[g + 1], len = p.shared_len[g];
    bool right = s0 >= 0 && s0 <= s1 && s1 <= b.n_seqs && len >= 0;
    int r0 = 0, r1 = 0;
    if (right && s0 < s1) {
      const int whole = b.length[s0];
      r0 = b.row_start[s0];
      r1 = b.row_start[s1];
      right = len <= whole && (int64_t)whole <= (int64_t)b.max_pages * b.page_size && r0 >= 0 && r0 <= r1 &&
              r1 <= b.n_rows;
    }
    if (!right) atomicOr(b.err, (int)CRF_DEVERR_BATCH);
    const bool any = right && s0 < s1 && r0 < r1;
    start[g] = s0;
    if (g == n - 1) start[n] = s1;
    shared[g] = any ? len : 0;
    row0[g] = r0;
    rows[g] = any ? r1 - r0 : 0;
  }
  // The group that holds sequence s (-1: none).
  CRF_DEV int of(int s) const {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (start[mid] <= s) lo = mid;
      else hi = mid;
    }
    return n > 0 && start[lo] <= s && s < start[lo + 1] ? lo : -1;
  }
};

// Item i; a sequence's tokens are those of seq_new().
CRF_DEV Item item_of(const SharedAttn &p, const Groups &gr, int i, int row0, int n, int len) {
  Item t{0, 0, 0, 0, 0, -1};
  if (i < gr.n) {
    t.hi = gr.shared[i];
    t.seq = t.hi > 0 ? gr.start[i] : 0;
    t.row0 = gr.row0[i];
    t.n = t.hi > 0 ? gr.rows[i] : 0;
  } else if (i < gr.n + p.a.b.n_seqs) {
    t = Item{row0, n, 0, len, i - gr.n, -1};
    const int g = n > 0 ? gr.of(t.seq) : -1;
    // (rows that do not lie among the group's have no part there)
    if (g >= 0 && gr.shared[g] > 0 && row0 >= gr.row0[g] && row0 + n <= gr.row0[g] + gr.rows[g]) {
      t.group = g;
      t.lo = min(gr.shared[g], len);
    }
  }
  return t;
}
CRF_DEV Item item_of(const SharedAttn &p, const Groups &gr, int i) {
  int row0 = 0, n = 0, len = 0;
  if (i >= gr.n && i < gr.n + p.a.b.n_seqs) n = seq_new(p.a.b, i - gr.n, row0, len);
  return item_of(p, gr, i, row0, n, len);
}

// Sums over the workgroup, the same in every thread.
CRF_DEV float4 total(float4 v, float4 *lds) {
  wave_prefix([&](auto c, auto rows) {
    v.x += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, v.x)));
    v.y += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, v.y)));
    v.z += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, v.z)));
    v.w += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, v.w)));
  });
  if (threadIdx.x % 64 == 63) lds[threadIdx.x / 64] = v;
  __syncthreads();
  float4 t = lds[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) t = make_float4(t.x + lds[w].x, t.y + lds[w].y, t.z + lds[w].z, t.w + lds[w].w);
  return t;
}

// The units of all items and the rows of their parts, which every workgroup works out, an item a
// thread.
//
// The units of an item: its chunks and KV heads, row tile after row tile; where there are several
// tiles, each tile's begin at a multiple of 8, so that those that share keys lie on one XCD
// (blockIdx.x % 8).
template <int BKV>
struct Plan {
  const SharedAttn &p;
  int G;
  int chunk = 0;  // key tiles of a unit (0: no item is computed)

  CRF_DEV int row_tiles(const Item &t) const { return (t.n * G + BM - 1) / BM; }
  CRF_DEV int first_tile(const Item &t) const { return t.lo / BKV; }
  CRF_DEV int key_tiles(const Item &t) const {
    return t.n > 0 && t.hi > t.lo ? (t.hi + BKV - 1) / BKV - first_tile(t) : 0;
  }
  CRF_DEV int chunks(const Item &t) const { return chunk > 0 ? (key_tiles(t) + chunk - 1) / chunk : 0; }
  CRF_DEV int tile_units(const Item &t) const {
    const int n = chunks(t) * p.a.nkv;
    return row_tiles(t) > 1 ? (n + 7) / 8 * 8 : n;
  }
  // What an item brings to the choice of the chunk: work in tiles, units at the least, rows of
  // parts at the least, and rows times key tiles.
  CRF_DEV void add(const Item &t, float4 &sum) const {
    const float k = key_tiles(t), tiles = (float)row_tiles(t) * p.a.nkv, rows = (float)t.n * p.a.nq;
    if (k > 0) sum = make_float4(sum.x + tiles * k, sum.y + tiles, sum.z + rows, sum.w + rows * k);
  }
  // The chunk's length: as many units as half of the workgroups that stay resident (the
  // sequences' own come on top; with 0.35 / 0.5 / 0.62 / 0.75 of them the 64 above take 52.0 /
  // 48.5 / 47.6 / 55.5 us, the 32 35.1 / 32.9 / 33.3 / 38.0, two times eight drafts of 8 over 8192
  // 48.4 / 45.2 / 47.5 / 44.8, 64 over 2000 with up to 1000 of their own 36.3 / 32.7 / 30.8 / 32.8),
  // and parts for which there is room: an item of k tiles has
  // k / c + 1 parts at most.  (Rounded sums: 2^-10 to spare.)
  CRF_DEV void choose(float4 sum) {
    const float spare = p.part_rows - sum.z * (1.f + 0x1p-10f);
    float c = fmaxf((float)SHORTEST, ceilf(sum.x / (0.5f * p.slots)));
    c = fminf(fmaxf(c, ceilf(sum.w / spare * (1.f + 0x1p-10f))), (float)LONGEST);
    chunk = spare > 0 ? (int)c : 0;
    // (sequences or groups that claim the same rows over and over)
    if (chunk == 0 && threadIdx.x == 0) atomicOr(p.a.b.err, (int)CRF_DEVERR_BATCH);
  }
};

struct Unit {
  int row0, n, lo, hi, seq;  // of the item
  int until;                 // its sequences: seq .. until - 1
  int base, number;          // first row of its parts, and which of its units this is
};

template <typename T, int HD, bool UNI>
__global__ __launch_bounds__(NT, 2) void shared_parts_kernel(const SharedAttn p) {
  using L = Layout<T, HD>;
  constexpr int BKV = sizeof(T) == 2 ? 64 : 32, TILE = BKV * L::ROWB;
  __shared__ __align__(16) char stages[2][2 * TILE];  // the groups while a unit is found; then K, then V
  __shared__ int pg[PGCAP];
  __shared__ int token_pos[BM];
  __shared__ float4 sums[NW];
  __shared__ int2 ends[NW];
  __shared__ Unit unit;
  __shared__ int bad;
  static_assert(Groups::WORDS * 4 <= sizeof stages, "groups in LDS");
  const PagedAttn &a = p.a;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  const int G = a.nq / a.nkv;
  const Groups gr((int *)&stages[0][0], p.n_groups);
  const int items = p.n_groups + a.b.n_seqs;
  const bool one = items <= NT;  // an item to a thread
  auto stage_groups = [&] {
    for (int i = tid; i < p.n_groups; i += NT) gr.stage(p, i);
    __syncthreads();
  };
  int my_row0 = 0, my_n = 0, my_len = 0;  // (the sequence's, while the groups are on their way)
  if (tid >= p.n_groups && tid < items) my_n = seq_new(a.b, tid - p.n_groups, my_row0, my_len);
  if (tid == 0) bad = 0;
  if (tid < BM) token_pos[tid] = -1;
  stage_groups();
  Plan<BKV> plan{p, G};
  Item it = item_of(p, gr, tid, my_row0, my_n, my_len);
  {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    plan.add(it, sum);
#pragma unroll 1
    for (int i = tid + NT; i < items; i += NT) plan.add(item_of(p, gr, i), sum);
    plan.choose(total(sum, sums));
  }
  // Goes over all items: puts the one that holds unit u into LDS; returns how many units there are.
  auto scan = [&](int u, bool write) {
    int units = 0, part_rows = 0;  // of the items before
#pragma unroll 1
    for (int i0 = 0; i0 < items; i0 += NT) {
      if (!one) it = item_of(p, gr, i0 + tid);
      const int num = plan.row_tiles(it) * plan.tile_units(it), own = it.n * a.nq * plan.chunks(it);
      int from = num, base = own;  // the item's first unit, the first row of its parts
      wave_prefix([&](auto c, auto rows) {
        from += from_lane<c(), rows()>(from);
        base += from_lane<c(), rows()>(base);
      });
      __syncthreads();  // (the ends before have been read)
      if (lane == 63) ends[wave] = make_int2(from, base);
      __syncthreads();
      from += units - num;
      base += part_rows - own;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w < wave) from += ends[w].x, base += ends[w].y;
        units += ends[w].x;
        part_rows += ends[w].y;
      }
      if (u >= from && u < from + num) {
        const int i = i0 + tid, until = i < p.n_groups ? gr.start[i + 1] : it.seq + 1;
        unit = Unit{it.row0, it.n, it.lo, it.hi, it.seq, until, base, u - from};
      }
      if (write) {  // (the groups lie before the sequences)
        const int i = i0 + tid, chunks = plan.chunks(it);
        if (i < p.n_groups) {
          gr.base[i] = base;
          gr.chunks[i] = chunks;
        }
        __syncthreads();
        if (i >= p.n_groups && i < items) {
          Info f{{base, chunks, it.row0, plan.chunk > 0 ? it.n : 0}, {0, 0, 0, 0}};
          if (it.group >= 0)
            f.shared = Parts{gr.base[it.group], gr.chunks[it.group], gr.row0[it.group], gr.rows[it.group]};
          ((Info *)p.info)[i - p.n_groups] = f;
        }
      }
    }
    return units;
  };
  // The units, of which the first (the groups') are the longest, are dealt out back and forth.  The
  // first half of the workgroups, one to a CU, begins with its last unit, so that those which
  // share a CU with one of the second half are the ones with short units (otherwise 64 sequences
  // over 2000 tokens with up to 1000 of their own, 28/4 heads, 37.4 us instead of 32.8, 48 over
  // eight documents, 12/2, 27.7 instead of 25.8; two times eight drafts 45.2 instead of 45.6).
  const int wg = (int)blockIdx.x, half = (int)gridDim.x / 2;
  const int begin = wg < half ? half - 1 - wg : wg;
  const int units = scan(begin, wg == 0);
#pragma unroll 1
  for (int round = 0;; ++round) {
    const int nth = round * (int)gridDim.x + (round % 2 ? (int)gridDim.x - 1 - begin : begin);
    if (nth >= units) break;
    if (round > 0) {  // (the items are worked out again: kept, their registers would be spilled)
      __syncthreads();  // (the unit before has left LDS)
      stage_groups();
      it = item_of(p, gr, tid);
      scan(nth, false);
      if (tid == 0) bad = 0;
      if (tid < BM) token_pos[tid] = -1;
    }
    __syncthreads();
    const Unit u{__builtin_amdgcn_readfirstlane(unit.row0), __builtin_amdgcn_readfirstlane(unit.n),
                 __builtin_amdgcn_readfirstlane(unit.lo),   __builtin_amdgcn_readfirstlane(unit.hi),
                 __builtin_amdgcn_readfirstlane(unit.seq),  __builtin_amdgcn_readfirstlane(unit.until),
                 __builtin_amdgcn_readfirstlane(unit.base), __builtin_amdgcn_readfirstlane(unit.number)};
    const int n = u.n, lo = u.lo, hi = u.hi;
    const Item item{u.row0, n, lo, hi, u.seq, -1};
    const int each = plan.tile_units(item), tile = u.number / each, x = u.number - tile * each;
    const int chunks = plan.chunks(item), kvh = x / chunks, part = x - kvh * chunks;
    if (kvh >= a.nkv) continue;  // (up to a multiple of 8)
    const int rows = min(BM, n * G - tile * BM), row0 = tile * BM;
    const int t0 = plan.first_tile(item) + part * plan.chunk, t1 = min(t0 + plan.chunk, (hi + BKV - 1) / BKV);
    const int first = u.row0 + row0 / G, tokens = (row0 + rows - 1) / G - row0 / G + 1;  // of the tile

    // this lane's row (padding rows repeat the last one)
    const int r = wave * 32 + l32, row = row0 + min(r, rows - 1);
    const int tok = row / G, head = kvh * G + row - tok * G;
    QFrag<T, HD> q;
    q.load((const T *)a.q + (int64_t)(u.row0 + tok) * a.q_ld + head * HD, g);
    // positions of the tile's tokens in the item's sequences (-1: in none; the largest where row
    // starts descend and several claim a token: no matter which comes first)
    auto place = [&](int start, int m, int len) {
      for (int t = max(start, first); t < min(start + m, first + tokens); ++t)
        atomicMax(&token_pos[t - first], len - m + t - start);
    };
    if (one) {
      if (tid >= p.n_groups && it.n > 0 && it.seq >= u.seq && it.seq < u.until) place(it.row0, it.n, it.hi);
    } else {
      for (int s = u.seq + tid; s < u.until; s += NT) {
        int start, len;
        const int m = seq_new(a.b, s, start, len);
        place(start, m, len);
      }
    }
    Pages<T, HD, UNI, BKV / NW> pages{a.b, a.zeros, pg, &bad, 0, hi, kvh, wave * (BKV / NW), lane,
                                      a.b.tables + (int64_t)u.seq * a.b.table_stride};
    const int end_key = t1 * BKV;
    pages.fill(div_by(t0 * BKV, a.b.ps_div), end_key, NT);
    RowState<HD> st;
    __syncthreads();
    const int last_key = min(token_pos[u.row0 + tok - first], hi - 1);  // of those that the row sees
    int least = last_key, most = last_key;
#pragma unroll
    for (int o = 16; o >= 1; o /= 2) {
      least = min(least, __shfl_xor(least, o, 64));
      most = max(most, __shfl_xor(most, o, 64));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    const int whole_to = wave * 32 < rows ? least + 1 : 0;  // keys before it are seen by every row of the wave
    bool careful = false, strictly = false;
    uint64_t strict = 0;
#pragma unroll 1
    for (;;) {
      st.clear();
      const lds_mem *mem = (const lds_mem *)&stages[0][0];
      auto load = [&](int i) {
        const lds_mem *k = mem + ((i - t0) & 1) * 2 * TILE;
        pages.load(i * BKV + wave * (BKV / NW), k, k + TILE);
      };
      load(t0);
      // A tile's data is there, the next one's is on its way (each wave passes here once a
      // tile, wherever it then goes).
      auto arrive = [&](int i) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (i + 1 < t1) {
          if (div_by(min((i + 2) * BKV, hi) - 1, a.b.ps_div) >= pages.first + PGCAP) {
            pages.fill(div_by(i * BKV, a.b.ps_div), end_key, NT);
            __syncthreads();
          }
          load(i + 1);
        }
      };
      q.arrived();
#pragma unroll 1
      for (int i = t0; i < t1;) {
        int taken = 0;  // blocks of the tile
        for (;;) {
          arrive(i);
          const int kt0 = i * BKV;
          if (i == t0 || kt0 + BKV > whole_to || kt0 < lo || bad || careful) break;
          const lds_mem *kt = mem + ((i - t0) & 1) * 2 * TILE;
          taken = whole_blocks<T, HD, BKV / 32>(kt, kt + TILE, q, st, a.scale_log2, lane);
          if (taken < BKV / 32) break;
          taken = 0;
          if (++i == t1) break;
        }
        if (i == t1) break;
        const int kt0 = i * BKV;
        if (wave * 32 < rows && kt0 <= most && kt0 + BKV > lo) {
          const Seen<false> seen{lo, last_key, lo, whole_to, hi, bad != 0, pg, pages.first, a.b.ps_div, strict, 0};
          const lds_mem *kt = mem + ((i - t0) & 1) * 2 * TILE;
#pragma unroll 1
          for (int kb = 32 * taken; kb < BKV; kb += 32)
            if (careful)
              block<T, HD, CAREFUL>(kt + kb * L::ROWB, kt + TILE + kb * L::ROWB, kt0 + kb, q, st, a.scale_log2, lane,
                                    seen);
            else
              block<T, HD, SOME>(kt + kb * L::ROWB, kt + TILE + kb * L::ROWB, kt0 + kb, q, st, a.scale_log2, lane,
                                 seen);
        }
        ++i;
      }
      const uint64_t odd = not_finite(st);
      const bool again = __syncthreads_or(odd != 0);
      if (strictly || !again) break;
      if (careful) strict = odd;
      strictly = careful;
      careful = true;
      pages.fill(div_by(t0 * BKV, a.b.ps_div), end_key, NT);
      __syncthreads();
    }

    const float l = st.l + __shfl_xor(st.l, 32, 64);
    if (r < rows) {
      const int64_t slot = u.base + ((int64_t)part * a.nkv + kvh) * n * G + row0 + r;
      float *o = p.o + slot * HD + 4 * g;
#pragma unroll
      for (int i = 0; i < 4 * L::HB; ++i)
        *(f32x4 *)(o + 8 * i) = f32x4{st.o[i / 4][4 * (i % 4)], st.o[i / 4][4 * (i % 4) + 1],
                                      st.o[i / 4][4 * (i % 4) + 2], st.o[i / 4][4 * (i % 4) + 3]};
      if (g == 0) p.ml[slot] = make_float2(st.ref, l);
    }
  }
}

// One token's heads of one KV head a workgroup, HD / 4 lanes a row.
template <typename T, int HD>
__global__ __launch_bounds__(NT) void shared_join_kernel(const SharedAttn p) {
  constexpr int LANES = HD / 4, ROWS = NT / LANES;
  const PagedAttn &a = p.a;
  const int tid = threadIdx.x, G = a.nq / a.nkv, e = 4 * (tid % LANES);
  const Info *info = (const Info *)p.info;
  __shared__ int owner;
#pragma unroll 1
  for (int64_t unit = blockIdx.x; unit < (int64_t)a.b.n_rows * a.nkv; unit += gridDim.x) {
    const int token = (int)(unit / a.nkv), kvh = (int)(unit - (int64_t)token * a.nkv);
    __syncthreads();
    if (tid == 0) owner = -1;
    __syncthreads();
    // Where row starts descend, several sequences may claim the token: it is the last one's.  (Their
    // Infos stored to one place could come out as a mixture, which names parts that nobody has
    // laid out.)
    int claims = -1;
    for (int s = tid; s < a.b.n_seqs; s += NT) {
      const int row0 = info[s].own.row0, n = info[s].own.n;
      if (token >= row0 && token < row0 + n) claims = s;
    }
    if (claims >= 0) atomicMax(&owner, claims);
    __syncthreads();
    const int whose = __builtin_amdgcn_readfirstlane(owner);
    if (whose < 0) continue;  // a row of nobody
    const Info f = info[whose];
    const int parts = f.shared.chunks + f.own.chunks;
    for (int r = tid / LANES; r < G; r += ROWS) {
      auto slot = [&](int j) {
        const bool s = j < f.shared.chunks;
        const Parts &q = s ? f.shared : f.own;
        const int c = s ? j : j - f.shared.chunks;
        return (int64_t)q.base + ((int64_t)c * a.nkv + kvh) * q.n * G + (token - q.row0) * G + r;
      };
      float top = -INFINITY, l = 0.f;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      // (a part of which the row sees nothing weighs nothing)
      constexpr int U = 8;
#pragma unroll 1
      for (int j0 = 0; j0 < parts; j0 += U) {
        float2 m[U];
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t at = slot(min(j0 + u, parts - 1));
          m[u] = p.ml[at];
          x[u] = *(const f32x4 *)(p.o + at * HD + e);
        }
        float most = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (j0 + u >= parts) m[u].y = 0.f;
          if (m[u].y != 0.f) most = fmaxf(most, m[u].x);
        }
        if (l != 0.f) {
          const float w = rescale(top, most);
          l *= w;
          sum *= w;
        }
        top = most;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (m[u].y == 0.f) continue;
          const float w = rescale(m[u].x, top);
          l = fmaf(w, m[u].y, l);
#pragma unroll
          for (int v = 0; v < 4; ++v) sum[v] = fmaf(w, x[u][v], sum[v]);
        }
      }
      const int head = kvh * G + r;
      sum *= l == 0.f ? 0.f : 1.f / l;
      T *dst = (T *)a.out + (int64_t)token * a.out_ld + head * HD + e;
      if constexpr (sizeof(T) == 2)
        st8(dst, pack_bf16x4(sum[0], sum[1], sum[2], sum[3]));
      else
        *(f32x4 *)dst = sum;
      if (e == 0 && a.lse)
        a.lse[(int64_t)token * a.nq + head] =
            l == 0.f ? -INFINITY : 0.69314718055994531f * (top + __builtin_amdgcn_logf(l));
    }
  }
}

template <typename T, int HD>
hipError_t launch(hipStream_t s, const SharedAttn &p) {
  const PagedBatch &b = p.a.b;
  const dim3 grid((unsigned)p.slots);
  if (b.page_size % 16 == 0)
    hipLaunchKernelGGL((shared_parts_kernel<T, HD, true>), grid, dim3(NT), 0, s, p);
  else
    hipLaunchKernelGGL((shared_parts_kernel<T, HD, false>), grid, dim3(NT), 0, s, p);
  const int64_t units = (int64_t)b.n_rows * p.a.nkv;
  hipLaunchKernelGGL((shared_join_kernel<T, HD>), dim3((unsigned)(units < MOST_GROUPS ? units : MOST_GROUPS)), dim3(NT),
                     0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_attn(hipStream_t s, bool f32, SharedAttn p) {
  const PagedBatch &b = p.a.b;
  if (b.n_seqs <= 0 || b.n_rows <= 0) return hipSuccess;
  const int G = p.a.nq / p.a.nkv;
  // the sequences' table, then the parts' rows
  const int64_t table = (int64_t)b.n_seqs * (int64_t)(sizeof(Info) / 4);
  const int64_t rows = (p.a.part_floats - table) / (p.a.hd + 2);
  p.part_rows = rows < INT32_MAX ? (int)rows : INT32_MAX;
  // Without a group, where a sequence fills a tile by itself, where all that the sequences read
  // by themselves is little, or without room for four parts of every row, each sequence reads
  // its shared keys itself.
  // Where the caller does not bound the new tokens, up to two a sequence on average count as short
  // ones: 64 next tokens about four documents without a bound took 226 us instead of 51 (a chunk
  // among them is then computed here as well: one of 200 over 6000 beside 200 next tokens about 512,
  // 12/2 heads, 71 us instead of 68, heads of 64 53 instead of 44; up to eight a sequence would have
  // a chunk of 448 over 12000 beside 64, 28/4 heads, take 225 instead of 126).
  const int64_t most = p.max_new > 0 || b.n_rows > 2 * (int64_t)b.n_seqs ? b.max_new : 2;
  const int64_t reads = (int64_t)b.n_seqs * std::min<int64_t>((int64_t)b.max_pages * b.page_size, (int64_t)1 << 24) *
                        p.a.nkv * p.a.hd * (f32 ? 8 : 4);
  if (p.n_groups == 0 || p.n_groups > SHARED_MAX_GROUPS || most * G > BM || reads <= SMALL_READS ||
      rows < 4 * (int64_t)b.n_rows * p.a.nq)
    return launch_paged_attn(s, f32, p.a);
  p.info = p.a.part;
  p.o = p.a.part + table;
  p.ml = (float2 *)(p.o + (int64_t)p.part_rows * p.a.hd);
  p.slots = 2 * p.a.n_cu / 8 * 8;
  if (p.slots < 8) p.slots = 8;
  if (f32) return p.a.hd == 128 ? launch<float, 128>(s, p) : launch<float, 64>(s, p);
  return p.a.hd == 128 ? launch<bf16, 128>(s, p) : launch<bf16, 64>(s, p);
}

}  // namespace crf
