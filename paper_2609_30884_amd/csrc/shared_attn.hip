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
// workgroup works out from the lengths on the device: as many units as workgroups stay
// resident.  The second joins each row's parts, in the order of the keys.
#include <math.h>

#include <algorithm>

#include "paged_tiles.hpp"
#include "serving.hpp"

namespace crf {
namespace {

constexpr int NW = 4, NT = 64 * NW, BM = 32 * NW;
constexpr int SHORTEST = 2;        // key tiles of a chunk, at least
constexpr int LONGEST = 1 << 26;   // more than any sequence has

// What the second launch needs of an item.
struct Info {
  int base;    // first row of its parts
  int chunks;  // of its keys
  int row0, n; // its new tokens
  int group;   // of a sequence that shares (else -1)
  int pad[3];
};

// Items 0 .. n_groups - 1 are the groups', the others the sequences'.
struct Item {
  int row0, n;  // new tokens
  int lo, hi;   // keys
  int seq;      // whose block table names them
  int group;
};

struct Groups {
  const int *start, *shared;  // LDS: first sequences (n + 1), shared lengths
  int n;
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

// A group's shared length; one that contradicts the batch is flagged and shares nothing.
CRF_DEV int shared_of(const SharedAttn &p, int g) {
  const PagedBatch &b = p.a.b;
  const int s0 = p.seq_start[g], s1 = p.seq_start[g + 1], n = p.shared_len[g];
  bool right = s0 >= 0 && s0 <= s1 && s1 <= b.n_seqs && n >= 0;
  if (right && s0 < s1) {
    const int len = b.length[s0], r0 = b.row_start[s0], r1 = b.row_start[s1];
    right = n <= len && (int64_t)len <= (int64_t)b.max_pages * b.page_size && r0 >= 0 && r0 <= r1 && r1 <= b.n_rows;
  }
  if (!right) atomicOr(b.err, (int)CRF_DEVERR_BATCH);
  return right && s0 < s1 ? n : 0;
}

CRF_DEV Item item_of(const SharedAttn &p, const Groups &gr, int i) {
  const PagedBatch &b = p.a.b;
  Item t{0, 0, 0, 0, 0, -1};
  if (i < gr.n) {
    t.hi = gr.shared[i];
    if (t.hi > 0) {
      t.seq = gr.start[i];
      t.row0 = b.row_start[t.seq];
      t.n = b.row_start[gr.start[i + 1]] - t.row0;
    }
  } else if (i < gr.n + b.n_seqs) {
    t.seq = i - gr.n;
    t.n = seq_new(b, t.seq, t.row0, t.hi);
    const int g = t.n > 0 ? gr.of(t.seq) : -1;
    // (rows that do not lie among the group's have no part there)
    if (g >= 0 && gr.shared[g] > 0 && t.row0 >= b.row_start[gr.start[g]] &&
        t.row0 + t.n <= b.row_start[gr.start[g + 1]]) {
      t.group = g;
      t.lo = gr.shared[g] < t.hi ? gr.shared[g] : t.hi;
    }
  }
  return t;
}

// The units of all items and the rows of their parts.  Every wave works them out, 64 items
// at a time, in doubles (whole numbers below 2^53).
struct Plan {
  const SharedAttn &p;
  const Groups &gr;
  int bkv, G;
  int chunk = 0;  // key tiles of a unit (0: no item is computed)
  Item it;        // the lane's item of the last block of 64

  Item found;       // in the lane that find() returns: the item that holds the unit ...
  double from, base; // ... where its units and the rows of its parts begin

  CRF_DEV int items() const { return gr.n + p.a.b.n_seqs; }
  CRF_DEV int row_tiles(const Item &t) const { return (t.n * G + BM - 1) / BM; }
  CRF_DEV int first_tile(const Item &t) const { return t.lo / bkv; }
  CRF_DEV int key_tiles(const Item &t) const {
    return t.n > 0 && t.hi > t.lo ? (t.hi + bkv - 1) / bkv - first_tile(t) : 0;
  }
  CRF_DEV int chunks(const Item &t) const { return chunk > 0 ? (key_tiles(t) + chunk - 1) / chunk : 0; }

  static CRF_DEV double total(double v) {
    wave_prefix([&](auto c, auto rows) { v += from_lane<c(), rows()>(v); });
    return last(v);
  }
  static CRF_DEV double last(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)u, 63));
  }

  // The chunk's length: units for `slots` workgroups, and parts for which there is room.
  CRF_DEV void choose(int slots) {
    double work = 0, lists = 0, rows = 0, row_keys = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < items(); i0 += 64) {
      it = item_of(p, gr, i0 + threadIdx.x % 64);
      const double k = key_tiles(it), t = (double)row_tiles(it) * p.a.nkv, r = (double)it.n * p.a.nq;
      work += total(t * k);
      lists += total(k > 0 ? t : 0);
      rows += total(k > 0 ? r : 0);
      row_keys += total(r * k);
    }
    const double room = fmax(slots - lists, 0.5 * slots), spare = p.part_rows - rows;
    double c = fmax((double)SHORTEST, ceil(work / room));
    // an item of k tiles has k / c + 1 parts at most
    c = fmin(fmax(c, ceil(row_keys / spare)), (double)LONGEST);
    chunk = __builtin_amdgcn_readfirstlane(spare > 0 ? (int)c : 0);
    // (sequences or groups that claim the same rows over and over)
    if (chunk == 0 && threadIdx.x == 0) atomicOr(p.a.b.err, (int)CRF_DEVERR_BATCH);
  }

  // Goes over all items, whose units it counts; leaves the one that holds unit u in the lane
  // that it returns (-1: none).  write: where the items go for the second launch; known: the
  // lanes' items are those of the one block there is.
  CRF_DEV int find(double u, double &units, Info *write, bool known) {
    double rows = 0;
    int where = -1;
    units = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < items(); i0 += 64) {
      const int i = i0 + threadIdx.x % 64;
      if (!known) it = item_of(p, gr, i);
      const double c = chunks(it), num = (double)row_tiles(it) * p.a.nkv * c, own = (double)it.n * p.a.nq * c;
      double sum = num, r = own;
      wave_prefix([&](auto cc, auto rr) { sum += from_lane<cc(), rr()>(sum); });
      wave_prefix([&](auto cc, auto rr) { r += from_lane<cc(), rr()>(r); });
      const double f = units + sum - num, b = rows + r - own;
      if (write && i < items()) write[i] = Info{(int)b, (int)c, it.row0, chunk > 0 ? it.n : 0, it.group, {0, 0, 0}};
      const uint64_t m = __builtin_amdgcn_ballot_w64(num > 0 && u >= f && u < f + num);
      if (m) {
        where = __builtin_ctzll(m);
        found = it;
        from = f;
        base = b;
      }
      units += last(sum);
      rows += last(r);
    }
    return where;
  }
};

CRF_DEV int uniform(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

template <typename T, int HD, bool UNI>
__global__ __launch_bounds__(NT, 2) void shared_parts_kernel(const SharedAttn p) {
  using L = Layout<T, HD>;
  constexpr int BKV = sizeof(T) == 2 ? 64 : 32, TILE = BKV * L::ROWB;
  __shared__ __align__(16) char stages[2][2 * TILE];  // K, then V
  __shared__ int pg[PGCAP];                           // the groups while a unit is found, then its pages
  __shared__ int token_pos[BM];
  __shared__ int bad;
  static_assert(PGCAP >= 2 * SHARED_MAX_GROUPS + 1, "groups in LDS");
  const PagedAttn &a = p.a;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  const int G = a.nq / a.nkv;
  const Groups gr{pg, pg + SHARED_MAX_GROUPS + 1, p.n_groups};
  Plan plan{p, gr, BKV, G};
  // units of neighbouring numbers, which share keys, lie on one XCD (blockIdx.x % 8)
  const int xcd = blockIdx.x % 8, per_xcd = gridDim.x / 8;
  double units = 0, per = 0;
#pragma unroll 1
  for (int round = 0;; ++round) {
    const int nth = (int)(blockIdx.x / 8) + round * per_xcd;
    if (round > 0 && nth >= per) break;
    __syncthreads();  // (the unit before has left LDS)
    for (int i = tid; i <= p.n_groups; i += NT) {
      pg[i] = p.n_groups > 0 ? p.seq_start[i] : 0;
      if (i < p.n_groups) pg[SHARED_MAX_GROUPS + 1 + i] = shared_of(p, i);
    }
    __syncthreads();
    if (round == 0) {
      plan.choose(p.slots);
      plan.find(-1, units, blockIdx.x == 0 && wave == 0 ? (Info *)p.info : nullptr, plan.items() <= 64);
      per = ceil(units / 8);
      if (nth >= per) break;
    }
    const double u = xcd * per + nth;
    if (u >= units) break;
    double all;
    const int at = plan.find(u, all, nullptr, round == 0 && plan.items() <= 64);
    if (at < 0) break;  // (cannot be: all waves count alike)
    const int row_first = uniform(plan.found.row0, at), n = uniform(plan.found.n, at), lo = uniform(plan.found.lo, at),
              hi = uniform(plan.found.hi, at), seq = uniform(plan.found.seq, at);
    const Item item{row_first, n, lo, hi, seq, -1};
    const int v = uniform((int)(u - plan.from), at), base = uniform((int)plan.base, at);
    const int tiles = plan.row_tiles(item), chunks = plan.chunks(item);
    const int tile = v % tiles, part = v / tiles % chunks, kvh = v / tiles / chunks;
    const int rows = min(BM, n * G - tile * BM), row0 = tile * BM;
    const int t0 = plan.first_tile(item) + part * plan.chunk, t1 = min(t0 + plan.chunk, (hi + BKV - 1) / BKV);
    const int token0 = row0 / G, tokens = (row0 + rows - 1) / G - token0 + 1;

    // positions of the tile's tokens (-1: of no sequence)
    __syncthreads();  // (the groups have been read)
    if (tid < BM) token_pos[tid] = -1;
    __syncthreads();
    for (int s = seq + tid; s < a.b.n_seqs; s += NT) {
      int start, len;
      const int m = seq_new(a.b, s, start, len), first = row_first + token0;
      if (start >= first + tokens) break;
      for (int t = max(start, first); t < min(start + m, first + tokens); ++t) token_pos[t - first] = len - m + t - start;
    }
    __syncthreads();

    // this lane's row (padding rows repeat the last one)
    const int r = wave * 32 + l32, row = row0 + min(r, rows - 1);
    const int tok = row / G, head = kvh * G + row - tok * G;
    const int last_key = min(token_pos[tok - token0], hi - 1);  // of those that the row sees
    int least = last_key, most = last_key;
#pragma unroll
    for (int o = 16; o >= 1; o /= 2) {
      least = min(least, __shfl_xor(least, o, 64));
      most = max(most, __shfl_xor(most, o, 64));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    QFrag<T, HD> q;
    q.load((const T *)a.q + (int64_t)(row_first + tok) * a.q_ld + head * HD, g);
    RowState<HD> st;
    Pages<T, HD, UNI, BKV / NW> pages{a.b, a.zeros, pg, &bad, 0, hi, kvh, wave * (BKV / NW), lane,
                                      a.b.tables + (int64_t)seq * a.b.table_stride};
    const int whole_to = wave * 32 < rows ? least + 1 : 0;  // keys before it are seen by every row of the wave
    const int end_key = t1 * BKV;
    if (tid == 0) bad = 0;
    bool careful = false, strictly = false;
    uint64_t strict = 0;
#pragma unroll 1
    for (;;) {
      st.clear();
      __syncthreads();  // the positions, or the pass before, have left LDS
      const lds_mem *mem = (const lds_mem *)&stages[0][0];
      auto load = [&](int i, int stage) {
        const lds_mem *k = mem + stage * 2 * TILE;
        pages.load(i * BKV + wave * (BKV / NW), k, k + TILE);
      };
      pages.fill(div_by(t0 * BKV, a.b.ps_div), end_key, NT);
      __syncthreads();
      load(t0, 0);
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
          load(i + 1, (i + 1 - t0) & 1);
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
          const Seen<false> seen{lo,  last_key,    lo,         whole_to, hi, bad != 0,
                                 pg,  pages.first, a.b.ps_div, strict,   0};
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
      const bool once_more = __syncthreads_or(odd != 0);
      if (strictly || !once_more) break;
      if (careful) strict = odd;
      strictly = careful;
      careful = true;
    }

    const float l = st.l + __shfl_xor(st.l, 32, 64);
    if (r < rows) {
      const int64_t slot = base + ((int64_t)part * a.nkv + kvh) * n * G + row0 + r;
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
    for (int s = tid; s < a.b.n_seqs; s += NT) {
      const Info &f = info[p.n_groups + s];
      if (token >= f.row0 && token < f.row0 + f.n) owner = s;
    }
    __syncthreads();
    if (owner < 0) continue;  // a row of nobody
    const Info own = info[p.n_groups + owner];
    Info shared{};
    if (own.group >= 0) shared = info[own.group];
    const int parts = shared.chunks + own.chunks;
    for (int r = tid / LANES; r < G; r += ROWS) {
      auto slot = [&](int j) {
        const Info &f = j < shared.chunks ? shared : own;
        const int c = j < shared.chunks ? j : j - shared.chunks;
        return (int64_t)f.base + ((int64_t)c * a.nkv + kvh) * f.n * G + (token - f.row0) * G + r;
      };
      float top = -INFINITY;
      for (int j = tid % LANES; j < parts; j += LANES) {
        const float2 m = p.ml[slot(j)];
        if (m.y != 0.f) top = fmaxf(top, m.x);
      }
#pragma unroll
      for (int o = LANES / 2; o >= 1; o /= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
      float l = 0.f;
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
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (j0 + u >= parts || m[u].y == 0.f) continue;
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
  const dim3 grid((unsigned)p.slots);
  if (p.a.b.page_size % 16 == 0)
    hipLaunchKernelGGL((shared_parts_kernel<T, HD, true>), grid, dim3(NT), 0, s, p);
  else
    hipLaunchKernelGGL((shared_parts_kernel<T, HD, false>), grid, dim3(NT), 0, s, p);
  const int64_t units = (int64_t)p.a.b.n_rows * p.a.nkv;
  hipLaunchKernelGGL((shared_join_kernel<T, HD>), dim3((unsigned)(units < MOST_GROUPS ? units : MOST_GROUPS)), dim3(NT),
                     0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_attn(hipStream_t s, bool f32, SharedAttn p) {
  const PagedBatch &b = p.a.b;
  if (b.n_seqs <= 0 || b.n_rows <= 0) return hipSuccess;
  const int G = p.a.nq / p.a.nkv;
  // the items' table, then the parts' rows
  const int64_t table = ((int64_t)p.n_groups + b.n_seqs) * (int64_t)(sizeof(Info) / 4);
  const int64_t rows = (p.a.part_floats - table) / (p.a.hd + 2);
  p.part_rows = rows < INT32_MAX ? (int)rows : INT32_MAX;
  // Without a group, where a sequence fills a tile by itself, or without room for four parts
  // of every row, each sequence reads its shared keys itself.
  if (p.n_groups == 0 || p.n_groups > SHARED_MAX_GROUPS || (int64_t)b.max_new * G > BM ||
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
