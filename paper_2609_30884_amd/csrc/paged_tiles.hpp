// Attention over tiles of 32 query rows and blocks of 32 keys from the pages of a cache:
// the arithmetic and the loads that the kernels over a page pool share.
#pragma once
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.hpp"

namespace crf {
namespace {

// A lane's sum of a block's 16 probabilities that needs no new reference.  Every raise
// costs its workgroup two blocks of the slow kind (about 2 us): with 2^8, scores of
// normal queries and keys raised up to 7 of 18 tiles of the chunks in a window above
// (48.6 us instead of 34.6).
constexpr float PSUM_MAX = 65536.0f;
constexpr int PGCAP = 2048;  // page numbers staged in LDS at a time

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

CRF_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
CRF_DEV f32x16 mfma32f(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
typedef __attribute__((address_space(3))) char lds_mem;
CRF_DEV u32x4 lds16(const lds_mem *p) { return *(const __attribute__((address_space(3))) u32x4 *)p; }
CRF_DEV s16x4 lds_tr(const lds_mem *p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p); }

// Loads of 16 bytes a lane straight to LDS, lane L's to lds + 16 L, for K and V
// together.  Written out, so that the compiler neither waits for them by itself (it would
// before every read of an LDS address that it cannot tell apart) nor needs a copy of the
// loop for each stage: they have no register to return to, and the kernels wait by count
// before they read.  M0, which nothing else here uses, takes the LDS address; the first
// wait states are those between a lane read into a scalar register and a vector memory
// instruction that uses it, the others those between M0 and its use.
//
// One page: raw buffer resources of the K and V rows (loads past their end return zero).
CRF_DEV uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
CRF_DEV u32x4 resource(const void *base, uint32_t bytes) {
  const uint64_t a = (uint64_t)base;
  return u32x4{scalar((uint32_t)a), scalar((uint32_t)(a >> 32) & 0xffffu), scalar(bytes), 0x00020000u};
}
// N x 1 KiB of K and of V, load i's at i KiB: the instruction's offset counts in both addresses.
template <int N>
CRF_DEV void dma_page(u32x4 kr, u32x4 vr, const lds_mem *kl, const lds_mem *vl, const uint32_t (&ko)[4], uint32_t vo) {
  const uint32_t k = scalar((uint32_t)(uintptr_t)kl), v = scalar((uint32_t)(uintptr_t)vl);
  if constexpr (N == 4)
    asm volatile(
        "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %7, 0 offen lds\n\t"
        "buffer_load_dwordx4 %3, %7, 0 offen offset:0x400 lds\n\tbuffer_load_dwordx4 %4, %7, 0 offen offset:0x800 lds\n\t"
        "buffer_load_dwordx4 %5, %7, 0 offen offset:0xc00 lds\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %6, %8, 0 offen lds\n\t"
        "buffer_load_dwordx4 %6, %8, 0 offen offset:0x400 lds\n\tbuffer_load_dwordx4 %6, %8, 0 offen offset:0x800 lds\n\t"
        "buffer_load_dwordx4 %6, %8, 0 offen offset:0xc00 lds"
        :
        : "s"(k), "s"(v), "v"(ko[0]), "v"(ko[1]), "v"(ko[2]), "v"(ko[3]), "v"(vo), "s"(kr), "s"(vr)
        : "memory");
  else
    asm volatile(
        "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
        "buffer_load_dwordx4 %3, %5, 0 offen offset:0x400 lds\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %6, 0 offen lds\n\t"
        "buffer_load_dwordx4 %4, %6, 0 offen offset:0x400 lds"
        :
        : "s"(k), "s"(v), "v"(ko[0]), "v"(ko[1]), "v"(vo), "s"(kr), "s"(vr)
        : "memory");
}
// Rows of their own: an address a lane.
CRF_DEV void dma_row(const char *k, const char *v, const lds_mem *kl, const lds_mem *vl) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, off"
      :
      : "s"(scalar((uint32_t)(uintptr_t)kl)), "s"(scalar((uint32_t)(uintptr_t)vl)), "v"(k), "v"(v)
      : "memory");
}

template <typename T, int HD>
struct Layout {
  static constexpr int ROWB = HD * (int)sizeof(T);  // bytes of a key's row
  static constexpr int CH = ROWB / 16;              // 16-byte chunks of it
  static constexpr int RPI = 64 / CH;               // rows that one load of a wave covers
  static constexpr int EPC = 16 / (int)sizeof(T);   // elements of a chunk
  static constexpr int KS = HD / (2 * EPC);         // steps of two chunks along a row
  static constexpr int HB = HD / 32;                // 32-row blocks of O^T
  // Chunk c of K row r lies at slot c ^ (r & 15) (8 chunks: r & 7): 16-byte reads of 8
  // rows land on distinct banks.
  static CRF_DEV int kslot(int r, int c) { return c ^ (r & (CH < 16 ? CH - 1 : 15)); }
  // And of V row r: bf16 transpose reads of 4 rows land on distinct banks; fp32 rows
  // are read along the row.
  static CRF_DEV int vslot(int r, int c) {
    if (sizeof(T) == 4) return c;
    if (HD == 128) return c ^ ((0xCA60 >> (4 * (r & 3))) & 15);
    return c ^ (2 * (r & 3));
  }
  // Byte addresses of a lane's reads in a tile, of which the others follow by an XOR
  // of the chunk bits and by constants: K row l32, chunk g (chunk 2 i + g: ^ 32 i) ...
  static CRF_DEV uint32_t kaddr(int lane) { return (lane % 32) * ROWB + kslot(lane % 32, lane / 32) * 16; }
  // ... V by transpose reads: 16-lane group t covers hd 16 (t & 1) .. + 15 of a 32-row
  // block b of O^T (^ 64 b) and key rows 4 (t / 2) + 0..3; fp32: row 4 g, column l32.
  static CRF_DEV uint32_t vaddr(int lane) {
    if (sizeof(T) == 4) return 4 * (lane / 32) * ROWB + lane % 32 * 4;
    const int t = lane / 16, r = 4 * (t >> 1) + lane % 16 / 4, hd = 16 * (t & 1) + 4 * (lane % 4);
    return r * ROWB + vslot(r, hd / 8) * 16 + hd % 8 * 2;
  }
};

// Keeps a value from being formed once and held through a loop: the few operations
// that derive addresses from it cost less than the registers.
CRF_DEV void fresh(uint32_t &x) { asm volatile("" : "+v"(x)); }

// A lane's query row: KS x 16 bytes.
template <typename T, int HD>
struct QFrag {
  u32x4 f[Layout<T, HD>::KS];
  CRF_DEV void load(const T *row, int g) {
#pragma unroll
    for (int s = 0; s < Layout<T, HD>::KS; ++s) f[s] = ld16(row + (2 * s + g) * Layout<T, HD>::EPC);
  }
  // The row has arrived.  (Else the compiler, which does not count the loads to LDS, waits
  // inside the loop over the keys for what it takes for these loads: for the next tile.)
  CRF_DEV void arrived() {
#pragma unroll
    for (int s = 0; s < Layout<T, HD>::KS; ++s) asm volatile("" : "+v"(f[s]));
  }
};

// The keys that a lane's row sees: [lo, hi]; bad: some pages of the unit are out of
// range, whose keys nobody sees.  SINKS: besides them the first `sinks` keys.
template <bool SINKS>
struct Seen {
  int lo, hi;
  int all_from, all_to;  // keys that every row of the wave sees: [all_from, all_to)
  int end;               // of the sequence
  bool bad;
  const int *pages;  // staged page numbers, the first of logical page `first`
  int first;
  FastDiv ps_div;
  uint64_t strict;  // CAREFUL: lanes whose reference is the maximum
  int sinks;
  CRF_DEV bool all(int key0) const {
    return (key0 >= all_from || (SINKS && key0 + 32 <= sinks)) && key0 + 32 <= all_to;
  }
};

template <int HD>
struct RowState {
  f32x16 o[HD / 32];
  float ref, l;
  CRF_DEV bool finite() const {  // (what the lane holds of its row)
    float z = 0.f;
#pragma unroll
    for (int b = 0; b < HD / 32; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) z = fmaf(o[b][v], 0.f, z);
    return z == 0.f;
  }
  CRF_DEV void clear() {
#pragma unroll
    for (int b = 0; b < HD / 32; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[b][v] = 0.f;
    ref = -INFINITY;
    l = 0.f;
  }
};

// Raw scores of NB blocks of 32 keys (K rows from kt on) against the wave's 32 rows.
// bf16: the K fragments are read two steps ahead of the products that use them (the
// scheduling barriers keep the compiler from regrouping them).
template <typename T, int HD, int NB>
CRF_DEV void scores(const lds_mem *kt, const QFrag<T, HD> &q, int lane, f32x16 (&s)[NB]) {
  using L = Layout<T, HD>;
  f32x16 zero;
#pragma unroll
  for (int v = 0; v < 16; ++v) zero[v] = 0.f;
  u32x4 kf[3][NB];
  uint32_t ka = L::kaddr(lane);
  fresh(ka);
  auto kread = [&](int step, u32x4 (&f)[NB]) {
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) f[kb] = lds16(kt + 32 * kb * L::ROWB + (ka ^ (32 * step)));
  };
  kread(0, kf[0]);
  kread(1, kf[1]);
#pragma unroll
  for (int i = 0; i < L::KS; ++i) {
    if (i + 2 < L::KS) kread(i + 2, kf[(i + 2) % 3]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      if constexpr (sizeof(T) == 2) {
        s[kb] = mfma32(as_bf16x8(kf[i % 3][kb]), as_bf16x8(q.f[i]), i == 0 ? zero : s[kb]);
      } else {
        const f32x4 a = __builtin_bit_cast(f32x4, kf[i % 3][kb]), b = __builtin_bit_cast(f32x4, q.f[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[kb] = mfma32f(a[e], b[e], i == 0 && e == 0 ? zero : s[kb]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// How a block of keys is taken.  ALL: every row sees all of it and keeps its reference.
// SOME: some row does not see some key, or needs another reference.  CAREFUL: a value
// that is not finite may belong to a key that some row does not see: the product would
// multiply it by that row's weight zero, so such values are taken out of the product and
// added where the row sees the key (however small its weight: a softmax has no zero).
//
// A unit runs without it first, and again with it if some row's result is not finite; the
// references are raised as before, so that a row that saw none of those values keeps every
// bit.  A third run is for rows that still are not: their reference is the maximum (STRICT),
// as large values times weights of up to PSUM_MAX may have passed the range.  Which rows
// those are depends on what they see alone.
enum Take { ALL, SOME, CAREFUL };
constexpr float STRICT = 16.f;  // a lane's 16 weights of up to 1

// The lanes of the rows that are not finite; a row's two lanes agree.
template <int HD>
CRF_DEV uint64_t not_finite(const RowState<HD> &st) {
  const uint64_t m = __builtin_amdgcn_ballot_w64(!st.finite());
  return m | m >> 32 | m << 32;
}

// O += P V for the probabilities p of 32 keys (V rows from vt on).  CAREFUL: bit v of `on`
// is set where the row sees the key of p[v].
//
// In bf16 the probabilities are rounded, to nearest, to the type that the matrix instructions
// take; their sum is formed before that.  The reference is not the row's maximum, so that the
// largest weight is rounded too.  Off from 64 bits, of the outputs' RMS, heads of 128 over 16000
// keys: 0.0023; with a maximum as the reference 0.0020; with probabilities in 32 bits, which need
// products at an eighth of the rate, 0.0017, the outputs' own rounding.  No part of it is one-sided.
template <typename T, int HD, Take TAKE>
CRF_DEV void weigh(const lds_mem *vt, const float (&p)[16], RowState<HD> &st, int lane, uint32_t on_bits = 0) {
  using L = Layout<T, HD>;
  uint32_t va = L::vaddr(lane);
  fresh(va);
  // infinities of each sign counted where the row sees them; no number counts as both
  f32x16 plus, minus;
  auto settle = [&](f32x16 &o) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if (plus[v] > 0.f) o[v] += INFINITY;
      if (minus[v] > 0.f) o[v] -= INFINITY;
    }
  };
  if constexpr (TAKE == CAREFUL)
#pragma unroll
    for (int v = 0; v < 16; ++v) plus[v] = minus[v] = 0.f;
  if constexpr (sizeof(T) == 2) {
    bf16x8 pf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[h][e] = f2bf(p[8 * h + e]);
    // slots 4-7 of a fragment hold the rows 8 further on
#pragma unroll
    for (int b = 0; b < L::HB; ++b) {
      s16x4 x[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          x[h][k] = lds_tr(vt + (16 * h + 8 * k) * L::ROWB + (va ^ (64 * b)));
      if constexpr (TAKE == CAREFUL) {
        f32x16 zero;
#pragma unroll
        for (int v = 0; v < 16; ++v) zero[v] = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          s16x4 up[2], down[2];
          bf16x8 on;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int w = (uint16_t)x[h][e / 4][e % 4];
            const bool out = (w & 0x7f80) == 0x7f80, nan = out && (w & 0x7f);
            up[e / 4][e % 4] = nan || w == 0x7f80 ? 0x3f80 : 0;
            down[e / 4][e % 4] = nan || w == 0xff80 ? 0x3f80 : 0;
            if (out) x[h][e / 4][e % 4] = 0;
            on[e] = on_bits >> (8 * h + e) & 1 ? f2bf(1.f) : f2bf(0.f);
          }
          plus = mfma32(__builtin_bit_cast(bf16x8, up), on, h == 0 ? zero : plus);
          minus = mfma32(__builtin_bit_cast(bf16x8, down), on, h == 0 ? zero : minus);
        }
        settle(st.o[b]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) st.o[b] = mfma32(__builtin_bit_cast(bf16x8, x[h]), pf[h], st.o[b]);
    }
  } else {
#pragma unroll
    for (int b = 0; b < L::HB; ++b) {
      float x[16];
#pragma unroll
      for (int v = 0; v < 16; ++v)
        x[v] = *(const __attribute__((address_space(3))) float *)(vt + (8 * (v / 4) + v % 4) * L::ROWB + 128 * b + va);
      if constexpr (TAKE == CAREFUL) {
#pragma unroll
        for (int v = 0; v < 16; ++v) plus[v] = minus[v] = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float on = on_bits >> v & 1 ? 1.f : 0.f;
          plus = mfma32f(x[v] == INFINITY || x[v] != x[v] ? 1.f : 0.f, on, plus);
          minus = mfma32f(x[v] == -INFINITY || x[v] != x[v] ? 1.f : 0.f, on, minus);
          if (!(fabsf(x[v]) < INFINITY)) x[v] = 0.f;
        }
        settle(st.o[b]);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) st.o[b] = mfma32f(x[v], p[v], st.o[b]);
    }
  }
}

// O += P V for NB blocks in bf16, whose V fragments are read two groups of products ahead
// (a group: two products, of the 32 rows b of O^T); ahead() reads the first two.
template <int HD, int NB>
struct Weigh {
  using L = Layout<bf16, HD>;
  static constexpr int GROUPS = NB * L::HB;
  const lds_mem *vt;
  uint32_t va;
  s16x4 x[3][4];

  CRF_DEV void read(int i) {
    const lds_mem *v = vt + 32 * (i / L::HB) * L::ROWB;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[i % 3][r] = lds_tr(v + 8 * r * L::ROWB + (va ^ (64 * (i % L::HB))));
  }
  CRF_DEV void ahead(const lds_mem *v, int lane) {
    vt = v;
    va = L::vaddr(lane);
    fresh(va);
    read(0);
    read(1);
    __builtin_amdgcn_sched_barrier(0);
  }
  // Block KB; during(j) is vector work for behind the j-th of its 2 HB products.
  template <int KB, typename F>
  CRF_DEV void add(const float (&p)[16], RowState<HD> &st, F during) {
    bf16x8 pf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[h][e] = f2bf(p[8 * h + e]);
#pragma unroll
    for (int b = 0; b < L::HB; ++b) {
      const int i = KB * L::HB + b;
      if (i + 2 < GROUPS) read(i + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s16x4 f[2] = {x[i % 3][2 * h], x[i % 3][2 * h + 1]};
        st.o[b] = mfma32(__builtin_bit_cast(bf16x8, f), pf[h], st.o[b]);
        during(2 * b + h);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// Up to NB blocks of 32 keys that every row sees; returns how many it has taken.  The
// next one needs another reference for some row, and is taken as below (the code that
// rescales O stays out of the loop over the others).  In bf16 a block's exponentials are
// formed between the products of the one before.
template <typename T, int HD, int NB>
CRF_DEV int whole_blocks(const lds_mem *kt, const lds_mem *vt, const QFrag<T, HD> &q, RowState<HD> &st, float c,
                         int lane) {
  f32x16 s[NB];
  scores<T, HD, NB>(kt, q, lane, s);
  float p[NB][16], sum[NB];
  auto weights = [&](int kb, int v0, int v1) {
#pragma unroll
    for (int v = v0; v < v1; ++v) {
      p[kb][v] = fast_exp2(fmaf(s[kb][v], c, -st.ref));
      sum[kb] = v == 0 ? p[kb][v] : sum[kb] + p[kb][v];
    }
  };
  auto raised = [&](int kb) {  // (also where the sum is no number)
    return __builtin_amdgcn_ballot_w64(!(sum[kb] <= PSUM_MAX)) != 0;
  };
  if constexpr (sizeof(T) == 2) {
    static_assert(NB <= 2, "blocks");
    constexpr int EACH = 16 / (2 * Layout<T, HD>::HB);
    Weigh<HD, NB> w;
    w.ahead(vt, lane);
    weights(0, 0, 16);
    if (raised(0)) return 0;
    st.l += sum[0];
    w.template add<0>(p[0], st, [&](int j) {
      if (NB > 1) weights(NB - 1, EACH * j, EACH * (j + 1));
    });
    if (NB > 1) {
      if (raised(NB - 1)) return 1;
      st.l += sum[NB - 1];
      w.template add<NB - 1>(p[NB - 1], st, [](int) {});
    }
  } else {
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) weights(kb, 0, 16);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
      if (raised(kb)) return 0;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      st.l += sum[kb];
      weigh<T, HD, ALL>(vt + 32 * kb * Layout<T, HD>::ROWB, p[kb], st, lane);
    }
  }
  return NB;
}

// One block of 32 keys, key0 ..: scores, probabilities, O += P V.
template <typename T, int HD, Take TAKE, bool SINKS>
CRF_DEV void block(const lds_mem *kt, const lds_mem *vt, int key0, const QFrag<T, HD> &q, RowState<HD> &st, float c,
                   int lane, const Seen<SINKS> &seen) {
  const float most = TAKE == CAREFUL && (seen.strict >> lane & 1) ? STRICT : PSUM_MAX;
  const int g = lane / 32;
  f32x16 sc[1];
  scores<T, HD, 1>(kt, q, lane, sc);
  f32x16 &s = sc[0];
  if (!seen.all(key0)) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = key0 + 8 * (v / 4) + 4 * g + v % 4;
      if ((key < seen.lo && !(SINKS && key < seen.sinks)) || key > seen.hi) s[v] = -INFINITY;
    }
  }
  if (seen.bad) {
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {  // keys of pages out of range
      const int key = key0 + i;
      if (key < seen.end && seen.pages[div_by(key, seen.ps_div) - seen.first] < 0)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v / 4) + 4 * g + v % 4 == i) s[v] = -INFINITY;
    }
  }
  uint32_t on = 0;
  if constexpr (TAKE == CAREFUL) {
#pragma unroll
    for (int v = 0; v < 16; ++v) on |= (s[v] == -INFINITY ? 0u : 1u) << v;
    fresh(on);  // (one register; else a pair of scalar ones for each bit)
  }
  float p[16], sum = INFINITY;
  if (!__builtin_amdgcn_ballot_w64(st.ref == -INFINITY)) {
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = fast_exp2(fmaf(s[v], c, -st.ref));
      sum += p[v];
    }
  }
  if (__builtin_amdgcn_ballot_w64(!(sum <= most))) {
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
    // only rows that need one: a row's result does not depend on the tile's others
    if (sum == INFINITY && st.ref != -INFINITY) {  // (not formed above, for other rows' sake)
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += fast_exp2(fmaf(s[v], c, -st.ref));
    }
    const float other = __shfl_xor(sum, 32, 64);
    const bool raise = !(sum <= most) || !(other <= most);
    const float ref = raise ? fmaxf(st.ref, mx) : st.ref;
    const float alpha = ref == -INFINITY ? 1.f : fast_exp2(st.ref - ref);
    const float base = ref == -INFINITY ? 0.f : ref;  // (a row that has seen no key yet)
    st.ref = ref;
    if (__builtin_amdgcn_ballot_w64(st.l != 0.f)) {
      st.l *= alpha;
#pragma unroll
      for (int b = 0; b < HD / 32; ++b) {
        if constexpr (TAKE == CAREFUL)  // (an infinity stays one, though alpha be zero)
#pragma unroll
          for (int v = 0; v < 16; ++v) st.o[b][v] *= fabsf(st.o[b][v]) == INFINITY ? 1.f : alpha;
        else
          st.o[b] *= alpha;
      }
    }
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = fast_exp2(fmaf(s[v], c, -base));
      sum += p[v];
    }
  }
  st.l += sum;
  weigh<T, HD, TAKE>(vt, p, st, lane, on);
}

// What O to the reference `from` weighs next to the reference `to`: never zero, so that its
// infinities stay (2^-149 of the largest finite number is 2^-21).
CRF_DEV float rescale(float from, float to) { return fmaxf(fast_exp2(from - to), 0x1p-149f); }

// ---------------------------------------------------------------- keys and values from the pages

// Stages page numbers and loads rows of keys and values, ROWS a wave and tile.
//
// UNI (pages of a multiple of 16 tokens): groups of 16 rows share a page, whose base
// goes into a buffer resource that ends where the sequence does; what lies past it,
// and every row of a page out of range, arrives as zeros.  Else each lane finds its
// own row's page, and the rows that nobody may read come from a block of zeros.
template <typename T, int HD, bool UNI, int ROWS>
struct Pages {
  using L = Layout<T, HD>;
  static constexpr int GRP = ROWS < 16 ? ROWS : 16;
  const PagedBatch &b;
  const char *zeros;
  int *pg;   // LDS, PGCAP numbers: logical page first + i
  int *bad;  // LDS: some page of the unit is out of range
  int first, len, kvh, lds_row0, lane;
  const int32_t *table;

  // A lane's bytes from the first of the rows that load i of a group covers (1 KiB).
  CRF_DEV uint32_t kbytes(int i, uint32_t k0) const {
    return k0 ^ (((i * L::RPI) & (L::CH < 16 ? L::CH - 1 : 15)) * 16);
  }
  // (V's slots repeat every 4 rows: RPI is a multiple of that wherever it has any)
  static_assert(sizeof(T) == 4 || L::RPI % 4 == 0, "V rows of a load");

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

  // Keys key0 .. (a multiple of ROWS): always 2 * ROWS / RPI loads.
  CRF_DEV void load(int key0, const lds_mem *kdst, const lds_mem *vdst) const {
    const int lrow = lane / L::CH;
    uint32_t k0 = lrow * L::ROWB + L::kslot(lds_row0 + lrow, lane % L::CH) * 16;
    uint32_t v0 = lrow * L::ROWB + L::vslot(lrow, lane % L::CH) * 16;
    fresh(k0);
    fresh(v0);
#pragma unroll
    for (int g0 = 0; g0 < ROWS; g0 += GRP) {
      const int kg = key0 + g0;
      const lds_mem *kl = kdst + (lds_row0 + g0) * L::ROWB, *vl = vdst + (lds_row0 + g0) * L::ROWB;
      if constexpr (UNI) {
        const int lp = div_by(kg, b.ps_div), rows = min(len - kg, GRP);
        const int q = rows > 0 ? __builtin_amdgcn_readfirstlane(pg[lp - first]) : -1;
        const int64_t off =
            q < 0 ? 0 : q * b.page_bytes + (int64_t)(kvh * b.page_size + kg - lp * b.page_size) * L::ROWB;
        const uint32_t bytes = q < 0 ? 0 : rows * L::ROWB;
        const u32x4 kr = resource(b.k + off, bytes), vr = resource(b.v + off, bytes);
        constexpr int LOADS = GRP / L::RPI, N = LOADS < 4 ? LOADS : 4;
        static_assert(LOADS == 2 || LOADS % 4 == 0, "loads of a group");
#pragma unroll
        for (int i = 0; i < LOADS; i += N) {
          uint32_t k[4];
#pragma unroll
          for (int j = 0; j < N; ++j) k[j] = kbytes(i + j, k0) + i * 1024;
          dma_page<N>(kr, vr, kl + i * 1024, vl + i * 1024, k, v0 + i * 1024);
        }
      } else {
#pragma unroll
        for (int i = 0; i < GRP / L::RPI; ++i) {
          const int key = kg + i * L::RPI + lrow;
          int q = -1, slot = 0;
          if (key < len) {
            const int lp = div_by(key, b.ps_div);
            q = pg[lp - first];
            slot = key - lp * b.page_size;
          }
          const int64_t o = q * b.page_bytes + (int64_t)(kvh * b.page_size + slot - lrow) * L::ROWB;
          dma_row(q >= 0 ? b.k + o + kbytes(i, k0) : zeros, q >= 0 ? b.v + o + v0 : zeros, kl + i * 1024,
                  vl + i * 1024);
        }
      }
    }
  }
};

}  // namespace
}  // namespace crf
