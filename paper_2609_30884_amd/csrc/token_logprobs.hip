// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits.
//
//   m = max z,  S = sum e^(z - m),  lse = m + ln S,  ln p_t = (z_t - m) - ln S,
//   H = ln S - (sum e^(z - m) (z - m)) / S   (every term of the sum has one sign),
// and the k largest z by (value, lowest index).
//
// One pass over the logits, which is what bounds it: HBM, or for few rows a chain of
// latencies.  A thread keeps the maximum so far and its two sums, rescaled where a batch of
// its loads brings a larger value; a row goes to several workgroups where rows are few, and
// the last of them to finish joins the parts, in their order.  Sums are fp32.
//
// The most likely tokens are found on the way.  A wave keeps a list in LDS of the keys (value
// in its order as an integer, then the lowest index) that exceed a threshold, of which at
// least k are known to reach it: at first the k-th largest of its lanes' first maxima, later
// the k-th largest of the list, taken whenever the list runs full.  Later elements of a wave
// have larger indices, so that only larger values can still enter, and a step costs one
// comparison an element.  The waves' lists, then the parts', are joined by counting for each
// key how many are larger.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "serving.hpp"

namespace crf {
namespace {

constexpr int NT = 256, NW = NT / 64;
constexpr int BATCH = 4;                    // 16-byte loads of a thread in flight
constexpr int LIST = 64 * 8 + LOGP_MAX_TOP; // keys of a wave: a step's, and k
constexpr float LOG2E = 1.4426950408889634f;
// Workgroups that a row is shared out to: until there are FILL of them, none smaller than
// SMALLEST loads of 16 bytes.
constexpr int FILL = 1024, SMALLEST = 256;

typedef unsigned long long Key;  // order of the value, ~index; 0: none

// Values in their order as integers: NaN above all, -0 as +0; none is 0.
CRF_DEV uint32_t order(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
  return z != z ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
CRF_DEV float value(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o); }
CRF_DEV Key key(float z, int index) { return (Key)order(z) << 32 | (uint32_t)~index; }
CRF_DEV Key lane_key(Key v, int lane) {
  return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
CRF_DEV int bits_below(uint64_t m) {  // bits of m below this lane
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}
CRF_DEV float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The LDS of a wave's own list is read and written in order within the wave.
CRF_DEV void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Puts the k largest of the wave's n <= LIST keys in front, largest first; returns how many.
CRF_DEV int keep_largest(Key *list, int n, int k, int lane) {
  constexpr int PER = (LIST + 63) / 64;
  wave_order();
  Key own[PER], most = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    own[i] = i * 64 + lane < n ? list[i * 64 + lane] : 0;
    most = own[i] > most ? own[i] : most;
  }
  if (n > 64) {
    // no key below the k-th largest of the lanes' largest is one of the k
    int above = 0;
#pragma unroll 4
    for (int l = 0; l < 64; ++l) above += lane_key(most, l) > most;
    const Key least = lane_key(most, __builtin_ctzll(__builtin_amdgcn_ballot_w64(above == k - 1)));
    n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool stays = own[i] >= least;
      const uint64_t m = __builtin_amdgcn_ballot_w64(stays);
      if (stays) list[n + bits_below(m)] = own[i];
      n += __popcll(m);
    }
    wave_order();
#pragma unroll
    for (int i = 0; i < PER; ++i) own[i] = i * 64 + lane < n ? list[i * 64 + lane] : 0;
  }
  int rank[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) rank[i] = 0;
  if (n <= 64) {
    for (int l = 0; l < n; ++l) rank[0] += lane_key(own[0], l) > own[0];
  } else {
    for (int l = 0; l < n; ++l) {
      const Key other = list[l];
#pragma unroll
      for (int i = 0; i < PER; ++i) rank[i] += other > own[i];
    }
  }
  wave_order();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (own[i] && rank[i] < k) list[rank[i]] = own[i];
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
  // Over the wave's lanes, in one order.
  CRF_DEV void wave() {
    to(wave_max(m));
    s = wave_sum(s);
    w = wave_sum(w);
  }
};

template <typename T>
struct Elements;  // 16 bytes as floats
template <>
struct Elements<float> {
  static constexpr int N = 4;
  static CRF_DEV void get(u32x4 v, float *f) {
    const f32x4 x = __builtin_bit_cast(f32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = x[i];
  }
};
template <>
struct Elements<bf16> {
  static constexpr int N = 8;
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

template <typename T, bool TOP>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(const TokenLogprobs p, int parts) {
  constexpr int E = Elements<T>::N;
  __shared__ Sums wave_sums[NW];
  __shared__ Key lists[TOP ? NW : 1][TOP ? LIST : 1];
  __shared__ Key best[TOP ? LOGP_MAX_TOP : 1];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int k = p.top, V = p.vocab;
  Key *const list = lists[TOP ? wave : 0];

  // The k largest of the waves' lists, each sorted, of n[w] <= k keys.
  auto join_waves = [&](int n) {
    if (lane < LOGP_MAX_TOP && lane >= n) list[lane] = 0;
    if (tid < LOGP_MAX_TOP) best[tid] = 0;
    __syncthreads();
    if (tid < NW * LOGP_MAX_TOP) {
      const Key own = lists[TOP ? tid / LOGP_MAX_TOP : 0][TOP ? tid % LOGP_MAX_TOP : 0];
      int rank = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll 8
        for (int i = 0; i < LOGP_MAX_TOP; ++i) rank += lists[TOP ? w : 0][TOP ? i : 0] > own;
      if (own && rank < k) best[rank] = own;
    }
    __syncthreads();
  };

#pragma unroll 1
  for (int64_t unit = blockIdx.x; unit < (int64_t)p.n_rows * parts; unit += gridDim.x) {
    const int64_t row = unit / parts;
    const int part = (int)(unit - row * parts);
    const T *z = (const T *)p.logits + row * p.ld;
    // 16-byte loads, the first of which may begin before the row and the last end behind it
    const int ahead = (int)((uintptr_t)z / sizeof(T) % E);
    const int loads = (int)(((int64_t)V + ahead + E - 1) / E);
    const int each = (loads + parts - 1) / parts;
    const int64_t l0 = (int64_t)part * each;
    const int64_t l1 = l0 + each < loads ? l0 + each : loads;
    Sums sum{-FLT_MAX, 0.f, 0.f};
    int n = 0;             // keys of the list
    float above = 0.f;     // values that are not at most this one enter it
    bool begun = false;    // a threshold is there
    __syncthreads();       // (the unit before has left LDS)
#pragma unroll 1
    for (int64_t a = l0; a < l1; a += BATCH * NT) {
      float f[BATCH][E];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int64_t l = a + j * NT + tid, i = l * E - ahead;
        if (l < l1 && i >= 0 && i + E <= V) {
          Elements<T>::get(ld16(z + i), f[j]);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) f[j][e] = l < l1 && i + e >= 0 && i + e < V ? at(z, i + e) : -INFINITY;
        }
      }
      float most = sum.m;
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) most = fmaxf(most, f[j][e]);
      if (most > sum.m) sum.to(most);
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) sum.add(f[j][e]);
      if constexpr (TOP) {
        if (!begun) {  // the k-th largest of the lanes' maxima
          begun = true;
          uint32_t own = 0;
#pragma unroll
          for (int j = 0; j < BATCH; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) own = max(own, order(f[j][e]));
          int greater = 0, equal = 0;
#pragma unroll 4
          for (int l = 0; l < 64; ++l) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)own, l);
            greater += o > own;
            equal += o == own;
          }
          const uint64_t m = __builtin_amdgcn_ballot_w64(greater < k && greater + equal >= k);
          uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)own, __builtin_ctzll(m)) - 1;
          if (o == 0x7fffffffu) --o;  // (zero's own place below is -0, which equals it)
          above = value(o);
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          uint64_t any = 0;
#pragma unroll
          for (int e = 0; e < E; ++e) any |= __builtin_amdgcn_ballot_w64(!(f[j][e] <= above));
          if (!any) continue;
          const int64_t i = (a + j * NT + tid) * E - ahead;
          const bool mine = a + j * NT + tid < l1;
          auto enters = [&](int e) {
            return __builtin_amdgcn_ballot_w64(mine && !(f[j][e] <= above) && i + e >= 0 && i + e < V);
          };
          int more = 0;
#pragma unroll
          for (int e = 0; e < E; ++e) more += __popcll(enters(e));
          if (n + more > LIST) {
            n = keep_largest(list, n, k, lane);
            above = value((uint32_t)(list[k - 1] >> 32));
          }
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint64_t m = enters(e);
            if (m >> lane & 1) list[n + bits_below(m)] = key(f[j][e], (int)(i + e));
            n += __popcll(m);
          }
        }
      }
    }
    sum.wave();
    if (lane == 0) wave_sums[wave] = sum;
    if constexpr (TOP) {
      n = keep_largest(list, n, k, lane);
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
      if (!last) continue;
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      if (TOP) {  // (at most a quarter of LOGP_PARTS parts to a wave)
        static_assert(LOGP_PARTS / NW * LOGP_MAX_TOP <= LIST, "keys of a quarter of the parts");
        const int q = (parts + NW - 1) / NW, first = wave * q, count = max(0, min(q, parts - first)) * k;
        for (int i = lane; i < count; i += 64)
          list[i] = Part{p, row * parts + first + i / k}.load(2 + i % k);
        join_waves(keep_largest(list, count, k, lane));
      }
      all = Part{p, row * parts + min(lane, parts - 1)}.sums();
      if (lane >= parts) all.s = all.w = 0.f;
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
  int64_t parts = (FILL + (int64_t)p.n_rows - 1) / p.n_rows;
  parts = std::min<int64_t>({parts, LOGP_PARTS, (int64_t)p.vocab / (E * SMALLEST), p.part_floats / 2 / (2 + LOGP_MAX_TOP) / p.n_rows});
  if (parts < 1 || p.n_rows > p.n_tickets) parts = 1;
  const int64_t units = parts * p.n_rows;
  const dim3 grid((unsigned)std::min<int64_t>(units, LOGP_MOST_GROUPS));
  if (p.top > 0)
    hipLaunchKernelGGL((token_logprobs_kernel<T, true>), grid, dim3(NT), 0, s, p, (int)parts);
  else
    hipLaunchKernelGGL((token_logprobs_kernel<T, false>), grid, dim3(NT), 0, s, p, (int)parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(hipStream_t s, bool f32, const TokenLogprobs &p) {
  if (p.n_rows <= 0) return hipSuccess;
  return f32 ? launch<float>(s, p) : launch<bf16>(s, p);
}

}  // namespace crf
