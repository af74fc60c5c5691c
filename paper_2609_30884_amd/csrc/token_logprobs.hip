// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits.
//
//   m = max z,  S = sum e^(z - m),  lse = m + ln S,  ln p_t = (z_t - m) - ln S,
//   H = ln S - (sum e^(z - m) (z - m)) / S   (every term of the sum has one sign),
// and the k largest z by (value, lowest index).
//
// One pass over the logits, which is what bounds it: HBM (2048 rows of 152064 in bf16 117 us, 5.3
// TB/s; streams that are only read reach 5.2 to 5.9 here), or for few rows a chain of latencies (one row in fp32 5.0 us, with 5 alternatives 8.6:
// launch, loads, sums, the parts' stores, ticket and loads, and the alternatives' order; a row
// that one workgroup takes 3.2 and 5.2).  A thread keeps the maximum so far and its two sums,
// rescaled where a batch of its loads brings a larger value, to which each batch's terms are
// added as one sum; a row goes to several workgroups
// where rows are few, and the last of them to finish joins the parts, in their order.  Sums are
// fp32.
//
// The most likely tokens are found on the way.  A wave keeps a list in LDS of the keys (value
// in its order as an integer, then the lowest index) that reach a threshold below which none of
// the workgroup's k largest lies.  At first it is the same for all four waves: of what a quarter
// of k of each wave's lanes reach with their first maxima, in the leading 16 bits, the least, so
// that k lanes of the workgroup reach it, however few of one wave's do.  Whenever a wave's list
// runs full it is cut to its k largest, and its k-th is that wave's threshold from then on.  Later
// elements of a wave have larger indices, so that only larger values can still enter, and a load
// costs one comparison: the few that hold a larger value are put side by side in LDS, and the lanes
// offer their elements to the list.  The waves' lists, then the parts', are joined by counting for
// each key how many are larger.  (64 rows with 20 alternatives: 39 us when every wave had a
// threshold of its own and inserted from registers, 20 when the parts were read through the
// caches after an acquire, 15.5 so; 1024 rows 184 and 73.)
#include <float.h>
#include <math.h>

#include <algorithm>

#include "serving.hpp"

namespace crf {
namespace {

constexpr int NT = 256, NW = NT / 64;
// 16-byte loads of a thread in flight.  8: 2048 rows of 152064 in bf16 114 us instead of 117, but
// 2048 rows of 2000 with 5 alternatives 24 instead of 14 (registers).
constexpr int BATCH = 4;
constexpr int LIST = 128;  // keys of a wave: k, and one to a lane
static_assert(LOGP_MAX_TOP + 64 <= LIST, "keys");
constexpr float LOG2E = 1.4426950408889634f;
// Workgroups that a row is shared out to: until there are FILL of them, none with fewer than
// SMALLEST loads of 16 bytes, and no row that one workgroup has in flight at once.  us with
// FILL 256 / 512 / 1024 / 2048: 64 rows of 152064 in bf16 with 20 alternatives 17.4 / 15.7 / 17.2
// / 23.5, without 9.9 / 9.8 / 12.3 / 15.7, 256 rows 33 / 31 / 29 / 36, 300 rows of 32000 14.0 /
// 15.6 / 18.5 / 26.  SMALLEST 256 / 512 / 1024: a row of 152064 in fp32 with 5 alternatives 8.8 /
// 8.8 / 9.4, of 32000 9.1 / 8.1 / 8.3; a row of 2000 shared by two 7.6, by none 5.2; four of
// 8000 in bf16 by two 9.1, by none 6.0.
constexpr int FILL = 512, SMALLEST = 512;

typedef unsigned long long Key;  // order of the value, ~index; 0: none
typedef __attribute__((address_space(3))) Key lds_key;

// Values in their order as integers: NaN above all, -0 as +0; none is 0.
CRF_DEV uint32_t order(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
  return z != z ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
CRF_DEV float value(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o); }
CRF_DEV Key key(float z, int index) { return (Key)order(z) << 32 | (uint32_t)~index; }
CRF_DEV int bits_below(uint64_t m) {  // bits of m below this lane
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}
CRF_DEV float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The LDS of a wave's own list is read and written in order within the wave.
CRF_DEV void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The largest number of the leading 16 bits that at least k of the lanes' values reach: all the
// bits that bf16 has, and for fp32 a bound that lets few more in (with all 32: 8 rows of 152064
// in bf16 with 20 alternatives 14.6 us instead of 13.0, a row in fp32 with 5 9.5 and 8.8; written
// out 12.7 and 8.6, as a loop 13.5 and 9.1; two bits a step, three counts each, 13.0 and 8.7).
CRF_DEV uint32_t reached_by(uint32_t v, int k) {
  uint32_t least = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t more = least | 1u << b;
    if (__popcll(__builtin_amdgcn_ballot_w64(v >= more)) >= k) least = more;
  }
  return least;
}

// How many of the n <= 64 keys that the wave's lanes hold are larger than the lane's own;
// `keys` is room for 64.
CRF_DEV int place(Key own, lds_key *keys, int n) {
  const int lane = threadIdx.x % 64;
  keys[lane] = lane < n ? own : 0;
  wave_order();
  int rank = 0;
#pragma unroll 1
  for (int l = 0; l < n; l += 16) {
    Key other[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) other[i] = keys[l + i];
#pragma unroll
    for (int i = 0; i < 16; ++i) rank += other[i] > own;
  }
  wave_order();
  return rank;
}

// Puts the k largest of the wave's n <= LIST keys in front, largest first; returns how many.
CRF_DEV int keep_largest(lds_key *list, int n, int k) {
  const int lane = threadIdx.x % 64;
  wave_order();
  Key a = lane < n ? list[lane] : 0, b = lane + 64 < n ? list[lane + 64] : 0;
  wave_order();
  if (n > 64) {
    // a value that k of the lanes' larger ones reach: no key below it is one of the k
    const Key least = (Key)reached_by((uint32_t)((a > b ? a : b) >> 32), k) << 32;
    const uint64_t ma = __builtin_amdgcn_ballot_w64(a >= least && a), mb = __builtin_amdgcn_ballot_w64(b >= least && b);
    const int na = __popcll(ma), both = na + __popcll(mb);
    if (both <= 64) {
      if (ma >> lane & 1) list[bits_below(ma)] = a;
      if (mb >> lane & 1) list[na + bits_below(mb)] = b;
      wave_order();
      n = both;
      a = lane < n ? list[lane] : 0;
      wave_order();
    } else {  // (equal values: each key's place among all of them)
      int ra = 0, rb = 0;
      for (int l = 0; l < n; ++l) {
        const Key other = list[l];
        ra += other > a;
        rb += other > b;
      }
      wave_order();
      if (a && ra < k) list[ra] = a;
      if (b && rb < k) list[rb] = b;
      wave_order();
      return k;
    }
  }
  const int rank = place(a, list, n);
  if (a && rank < k) list[rank] = a;
  wave_order();
  return n < k ? n : k;
}

// A running maximum and the sums over e^(z - m) and e^(z - m) (z - m).
struct Sums {
  float m, s, w;
  CRF_DEV void to(float most) {
    const float d = fmaxf(m - most, -1e4f), a = exp2_fast(d * LOG2E);
    w = a * fmaf(s, d, w);
    s *= a;
    m = most;
  }
  CRF_DEV void add(float z) {
    const float d = z - m, e = exp2_fast(d * LOG2E);
    s += e;
    w = fmaf(e, fmaxf(d, -1e4f), w);  // (-inf weighs nothing; NaN stays in e)
  }
  CRF_DEV void add(const Sums &v) {  // (to the same m)
    s += v.s;
    w += v.w;
  }
  // Over the wave's lanes, in one order.
  CRF_DEV void wave() {
    float most = m;
    wave_prefix([&](auto c, auto rows) {
      const int v = __builtin_bit_cast(int, most);
      most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, c(), rows(), 0xf, false)));
    });
    to(last(most));
    wave_prefix([&](auto c, auto rows) {
      s += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, s)));
      w += __builtin_bit_cast(float, from_lane<c(), rows()>(__builtin_bit_cast(int, w)));
    });
    s = last(s);
    w = last(w);
  }
  static CRF_DEV float last(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
  }
};

template <typename T>
struct Elements;  // 16 bytes as floats; NONE: -inf in all of them
template <>
struct Elements<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;
  static CRF_DEV void get(u32x4 v, float *f) {
    const f32x4 x = __builtin_bit_cast(f32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = x[i];
  }
};
template <>
struct Elements<bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xff80ff80u;
  static CRF_DEV void get(u32x4 v, float *f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
    }
  }
};

CRF_DEV float at(const float *z, int64_t i) { return z[i]; }
CRF_DEV float at(const bf16 *z, int64_t i) { return bf2f(z[i]); }

// A part's results: maximum, sums, k keys.
struct Part {
  const TokenLogprobs &p;
  int64_t slot;
  CRF_DEV uint64_t *at() const { return (uint64_t *)p.part + slot * (2 + LOGP_MAX_TOP); }
  CRF_DEV void store(int i, uint64_t v) const {
    __hip_atomic_store(at() + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  CRF_DEV uint64_t load(int i) const { return __hip_atomic_load(at() + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
  CRF_DEV void store(const Sums &v) const {
    store(0, (uint64_t)__builtin_bit_cast(uint32_t, v.s) << 32 | __builtin_bit_cast(uint32_t, v.m));
    store(1, __builtin_bit_cast(uint32_t, v.w));
  }
  CRF_DEV Sums sums() const {
    const uint64_t a = load(0);
    Sums v;
    v.m = __builtin_bit_cast(float, (uint32_t)a);
    v.s = __builtin_bit_cast(float, (uint32_t)(a >> 32));
    v.w = __builtin_bit_cast(float, (uint32_t)load(1));
    return v;
  }
};

// (Four workgroups a CU: 1024 rows with 20 alternatives 73 us, with the 136 registers of three
// 77; five spill: 87.)
template <typename T, bool TOP>
__global__ __launch_bounds__(NT, 4) void token_logprobs_kernel(const TokenLogprobs p, int parts, int each) {
  constexpr int E = Elements<T>::N;
  __shared__ Sums wave_sums[NW];
  __shared__ Key lists[TOP ? NW : 1][TOP ? LIST : 1];
  __shared__ Key best[TOP ? LOGP_MAX_TOP : 1], flat[TOP ? 64 : 1];
  // a batch's loads that hold something to enter, with their numbers; then the parts' keys
  __shared__ __align__(16) u32x4 held[TOP ? NW : 1][TOP ? BATCH * 64 : 1];
  __shared__ uint16_t held_at[TOP ? NW : 1][TOP ? BATCH * 64 : 1];
  __shared__ uint32_t reach[NW];
  __shared__ int count[NW];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int k = p.top, V = p.vocab;
  lds_key *const list = (lds_key *)lists[TOP ? wave : 0];
  const float per_k = 1.f / (TOP ? k : 1);

  // The k largest of the waves' lists of n keys each into `best`, largest first.
  auto join_waves = [&](int n) {
    if (lane == 0) count[wave] = n;
    if (tid < LOGP_MAX_TOP) best[tid] = 0;
    __syncthreads();
    int start[NW], all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      start[w] = all;
      all += count[w];
    }
    if (__builtin_amdgcn_readfirstlane(all) <= 64) {  // a lane to each
      if (wave == 0) {
        int w = 0;
#pragma unroll
        for (int i = 1; i < NW; ++i) w = lane >= start[i] ? i : w;
        int first = start[0];
#pragma unroll
        for (int i = 1; i < NW; ++i) first = w == i ? start[i] : first;
        const Key own = lane < all ? lists[w][lane - first] : 0;
        const int rank = place(own, (lds_key *)flat, all);
        if (own && rank < k) best[rank] = own;
      }
    } else {
      n = keep_largest(list, n, k);
      if (lane < LOGP_MAX_TOP && lane >= n) list[lane] = 0;
      __syncthreads();
      if (tid < NW * LOGP_MAX_TOP) {
        // a key's place is its own in its list and how many are larger in the others
        const int w = tid / LOGP_MAX_TOP, i = tid % LOGP_MAX_TOP;
        const Key own = lists[w][i];
        int rank = i;
#pragma unroll
        for (int o = 1; o < NW; ++o) {
          const Key *other = lists[(w + o) % NW];
          int larger = 0;
#pragma unroll
          for (int size = LOGP_MAX_TOP / 2; size >= 1; size /= 2)
            if (other[larger + size - 1] > own) larger += size;
          rank += larger + (other[larger] > own);
        }
        if (own && rank < k) best[rank] = own;
      }
    }
    __syncthreads();
  };
  // The least of the waves' numbers.
  auto least_of_waves = [&](uint32_t v) {
    if (lane == 0) reach[wave] = v;
    __syncthreads();
    return min(min(reach[0], reach[1]), min(reach[2], reach[3]));
  };
  static_assert(NW == 4, "waves");
  const int quarter = (k + NW - 1) / NW;  // what a quarter of k lanes of each wave reach, k of the workgroup do

#pragma unroll 1
  for (int64_t unit = blockIdx.x; unit < (int64_t)p.n_rows * parts; unit += gridDim.x) {
    const int64_t row = parts == 1 ? unit : (int)unit / parts;  // (shared out rows are few)
    const int part = (int)(unit - row * parts);
    const T *z = (const T *)p.logits + row * p.ld;
    // loads of 16 bytes: `loads` of them from element `head` on, single elements before and behind
    const int head = min(V, (int)(-(uintptr_t)z / sizeof(T) % E)), loads = (V - head) / E;
    const T *body = z + head;
    const int l0 = min(loads, part * each), l1 = min(loads, l0 + each);
    Sums sum{-FLT_MAX, 0.f, 0.f};
    int n = 0;             // keys of the list
    float above = NAN;     // values that are not at most this one enter it
    __syncthreads();       // (the unit before has left LDS)
    // A key a lane, which enters the list if it is to.
    auto offer = [&](Key v, bool enters) {
      uint64_t m = __builtin_amdgcn_ballot_w64(enters);
      if (!m) return;
      if (n + __popcll(m) > LIST) {
        n = keep_largest(list, n, k);
        above = value((uint32_t)(list[k - 1] >> 32));
        m = __builtin_amdgcn_ballot_w64(enters && v > list[k - 1]);
      }
      if (m >> lane & 1) list[n + bits_below(m)] = v;
      n += __popcll(m);
    };
    u32x4 next[BATCH];
    auto load = [&](int a) {
#pragma unroll
      for (int j = 0; j < BATCH; ++j) next[j] = ld16(body + (int64_t)min(a + j * NT + tid, l1 - 1) * E);
    };
    if (l0 < l1) load(l0);
#pragma unroll 1
    for (int a = l0; a < l1; a += BATCH * NT) {
      u32x4 x[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const bool mine = a + j * NT + tid < l1;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j][i] = mine ? next[j][i] : Elements<T>::NONE;
      }
      if (a + BATCH * NT < l1) load(a + BATCH * NT);
      float largest[BATCH], most = -INFINITY;
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        float f[E];
        Elements<T>::get(x[j], f);
        largest[j] = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) largest[j] = fmaxf(largest[j], f[e]);
        most = fmaxf(most, largest[j]);
      }
      if (most > sum.m) sum.to(most);
      const int steps = (l1 - a - wave * 64 + NT - 1) / NT;  // of the wave that hold anything
      // A load's terms, then the loads', are added up by themselves: a sum of hundreds rounds every
      // single term that is added to it, like ones to the same side.  Rows of 152064 with each term
      // added by itself, and so: ln S off by -7e-7 and -2e-8 on average for normal logits (5.3e-6 and
      // 1.3e-6 at most), by 1.1e-5 and 2.5e-7 where all but the largest are alike; times are equal.
      Sums batch{sum.m, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        if (j >= steps) break;
        float f[E];
        Elements<T>::get(x[j], f);
        Sums one{sum.m, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) one.add(f[e]);
        batch.add(one);
      }
      sum.add(batch);
      if constexpr (TOP) {
        if (a == l0) {  // a value that k of the workgroup's lanes' maxima reach
          uint32_t o = least_of_waves(reached_by(order(most), quarter)) - 1;
          if (o == 0x7fffffffu) --o;  // (zero's own place below is -0, which equals it)
          above = value(o);
        }
        // loads that hold something to enter (NaN, which is no maximum, is in the sum) are put
        // side by side, and their elements offered, one a lane
        int loads_held = 0;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const uint64_t m =
              __builtin_amdgcn_ballot_w64(a + j * NT + tid < l1 && (!(largest[j] <= above) || sum.s != sum.s));
          if (!m) continue;
          if (m >> lane & 1) {
            held[TOP ? wave : 0][TOP ? loads_held + bits_below(m) : 0] = x[j];
            held_at[TOP ? wave : 0][TOP ? loads_held + bits_below(m) : 0] = (uint16_t)(j * NT + tid);
          }
          loads_held += __popcll(m);
        }
        if (loads_held) {
          wave_order();
#pragma unroll 1
          for (int c = 0; c < loads_held * E; c += 64) {
            const bool mine = c + lane < loads_held * E;
            const int h = mine ? (c + lane) / E : 0, e = lane % E;
            const float v = at((const T *)&held[TOP ? wave : 0][TOP ? h : 0], e);
            const int i = head + (a + held_at[TOP ? wave : 0][TOP ? h : 0]) * E + e;
            offer(key(v, i), mine && !(v <= above));
          }
          wave_order();
        }
      }
    }
    // the elements before and behind the loads: at most one a lane
    const int tail = head + loads * E;
    if (wave == 0 && ((part == 0 && head > 0) || (part == parts - 1 && tail < V))) {
      const int i = lane < E ? lane : tail + lane - E;
      const bool mine = lane < E ? part == 0 && i < head : part == parts - 1 && i < V;
      const float v = mine ? at(z, i) : -INFINITY;
      if (v > sum.m) sum.to(v);
      sum.add(v);
      if constexpr (TOP) offer(key(v, i), mine && !(v < above));  // (equal ones may lie before those of the list)
    }
    sum.wave();
    if (lane == 0) wave_sums[wave] = sum;
    if constexpr (TOP) {
      join_waves(n);
    } else {
      __syncthreads();
    }
    Sums all = wave_sums[lane < NW ? lane : 0];
    if (lane >= NW) all.s = all.w = 0.f;
    all.wave();
    if (parts > 1) {
      const Part mine{p, unit};
      if (tid == 0) mine.store(all);
      if (TOP && tid < k) mine.store(2 + tid, best[tid]);
      agent_flush();
      __syncthreads();
      if (tid == 0) {
        last = agent_ticket(&p.tickets[row]) == (unsigned)parts - 1;
        if (last) __hip_atomic_store(&p.tickets[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      // (the parts are read past the caches, as they were written: no line of them is in one)
      if (!last) continue;
      all = Part{p, row * parts + min(lane, parts - 1)}.sums();
      if (lane >= parts) all.s = all.w = 0.f;
      if (TOP) {  // (at most a quarter of LOGP_PARTS parts to a wave)
        const int q = (parts + NW - 1) / NW, first = wave * q, keys_held = max(0, min(q, parts - first)) * k;
        constexpr int PER = (LOGP_PARTS / NW * LOGP_MAX_TOP + 63) / 64;
        static_assert(PER * 64 * sizeof(Key) <= BATCH * 64 * sizeof(u32x4), "keys of a quarter of the parts");
        const Part from{p, row * parts + min(first, parts - 1)};
        Key keys[PER];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {  // (the quotient of numbers below 2^10 is exact)
          const int x = max(0, min(i * 64 + lane, keys_held - 1)), part_of = (int)((x + 0.5f) * per_k);
          keys[i] = from.load(part_of * (2 + LOGP_MAX_TOP) + 2 + x - part_of * k);
        }
        lds_key *const mine = (lds_key *)&held[TOP ? wave : 0][0];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (i * 64 + lane >= keys_held) keys[i] = 0;
          most = max(most, (uint32_t)(keys[i] >> 32));
          mine[i * 64 + lane] = keys[i];
        }
        const Key least = (Key)max(1u, least_of_waves(reached_by(most, quarter))) << 32;
        n = 0;
#pragma unroll 1
        for (int c = 0; c < keys_held; c += 64) offer(mine[c + lane], mine[c + lane] >= least);
        join_waves(n);
      }
      all.wave();
    }

    // (a row of -inf alone: every probability is zero)
    const float ln_s = logf(all.s);
    auto log_p = [&](float v) { return all.s == 0.f ? -INFINITY : (v - all.m) - ln_s; };
    if (tid == 0) {
      if (p.lse) p.lse[row] = all.s == 0.f ? -INFINITY : all.m + ln_s;
      if (p.entropy) p.entropy[row] = all.s == 0.f ? 0.f : ln_s - all.w / all.s;
    }
    for (int64_t j = tid; j < p.n_tokens; j += NT) {
      const int t = p.tokens[row * p.n_tokens + j];
      float v = 0.f;
      if (t >= V) {
        atomicOr(p.err, (int)CRF_DEVERR_TOKEN);
        v = -INFINITY;
      } else if (t >= 0) {
        v = log_p(at(z, t));
      }
      p.logprob[row * p.n_tokens + j] = v;
    }
    if (TOP && tid < k) {
      p.top_token[row * k + tid] = (int)~(uint32_t)best[tid];
      p.top_logprob[row * k + tid] = log_p(value((uint32_t)(best[tid] >> 32)));
    }
  }
}

template <typename T>
hipError_t launch(hipStream_t s, const TokenLogprobs &p) {
  constexpr int E = Elements<T>::N;
  const int64_t loads = (int64_t)p.vocab / E;
  const int64_t room = p.n_rows <= p.n_tickets ? p.part_floats / 2 / (2 + LOGP_MAX_TOP) / p.n_rows : 1;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>({(FILL + p.n_rows - 1) / p.n_rows, LOGP_PARTS, room}));
  // (whole steps of a workgroup to a part)
  const int64_t least = loads <= BATCH * NT ? BATCH * NT : SMALLEST;
  const int64_t each = std::max<int64_t>(((loads + most - 1) / most + NT - 1) / NT * NT, least);
  const int64_t parts = std::max<int64_t>(1, (loads + each - 1) / each), units = parts * p.n_rows;
  const dim3 grid((unsigned)std::min<int64_t>(units, LOGP_MOST_GROUPS));
  if (p.top > 0)
    hipLaunchKernelGGL((token_logprobs_kernel<T, true>), grid, dim3(NT), 0, s, p, (int)parts, (int)each);
  else
    hipLaunchKernelGGL((token_logprobs_kernel<T, false>), grid, dim3(NT), 0, s, p, (int)parts, (int)each);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(hipStream_t s, bool f32, const TokenLogprobs &p) {
  if (p.n_rows <= 0) return hipSuccess;
  return f32 ? launch<float>(s, p) : launch<bf16>(s, p);
}

}  // namespace crf
