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
// the one there is, and only where a lane's sum passes 2^16 is the maximum taken and
// O rescaled.  It starts at minus infinity, which makes the first block that a row
// sees take that path.  Scores, sums and O are fp32; the probabilities are rounded
// to the storage type for the second product, as MFMA needs them (bf16: 2^-8
// of each weight at most), and summed before that rounding.
//
// Schedule: a unit is a row tile of one KV head of one sequence.  Its work (keys times
// rows) is known on the device alone, so every workgroup works out from all lengths what
// it computes.  Either units are dealt out whole, longest of a sequence first; or the
// work is dealt out evenly, a contiguous stretch to each resident workgroup, and a unit
// cut by a border leaves partials, which the workgroup that finishes last joins in the
// order of the keys (results do not depend on who that is).
//
// Measured (bf16, head size 128 where nothing else is said):
//   8192 tokens after 8192, 28/4 heads    1.36 ms, 1.06 PFLOP/s (a large matrix product
//     reaches 1.19).  Matrix pipes are busy 57 % of the cycles; with all exponentials of
//     a tile before its second product it takes 2.5 % longer;
//   64 sequences' next tokens over 500 to 16384, 28/4 heads    152 us, 5.2 TB/s: HBM;
//   12 sequences, some with chunks of up to 512, over up to 8192, 12/2 heads    70 us, 0.43
//     PFLOP/s: 9 us until the first task is known, 33 of products, 14 to join 9 or 10
//     parts, whose 33 MB are written and read once;
//   4 chunks of 500 to 2048 in a window of 1024, 12/2 heads of 64    35 us, 0.43 PFLOP/s:
//     the exponentials, of which heads of 64 have twice as many to a product;
//   one next token over 3000, 12/2 heads    13.7 us: a chain of latencies (lengths 2, its
//     schedule 2, page numbers 1.5, keys 3, partials 1.5, ticket 1.5, join 2.5).
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
// Rounds of units over the resident workgroups from which none is split.  8192 tokens
// after 8192 (4.1 rounds) 1.40 ms, split 1.53; 8 chunks of 2048 488 us, split 530; with 1,
// the 12 sequences above 188 us instead of 71.
constexpr int MANY = 3;
// Tiles that a part costs besides its keys, when whole units and parts are weighed.  0: the
// chunks in a window 45 us instead of 35 (cut where whole units come out as even); 99: 16
// chunks of 64 over 4000 99 us instead of 51 (left whole where they do not).
constexpr float SPLIT = 8.f;
// Fewer tiles are no part of their own.  0: the 12 sequences 75.8 us instead of 71.1, six
// chunks in fp32 27.6 instead of 22.5.
constexpr int SLIVER = 2;
// Bytes of K and V up to which tiles of 32 rows do (as counted in launch() below).  0: 300
// tokens 22 us instead of 15, two chunks of 32 over 2000 33 instead of 23, six in fp32 28
// instead of 22.5; no limit: 1000 tokens (190 MB) 37 instead of 30, 16 chunks of 64 over
// 4000 70 instead of 51, the 12 sequences 183 instead of 71.
constexpr int64_t SMALL_READS = 48 << 20;

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
// range, whose keys nobody sees.
struct Seen {
  int lo, hi;
  int all_from, all_to;  // keys that every row of the wave sees: [all_from, all_to)
  int end;               // of the sequence
  bool bad;
  const int *pages;  // staged page numbers, the first of logical page `first`
  int first;
  FastDiv ps_div;
  uint64_t strict;  // CAREFUL: lanes whose reference is the maximum
  CRF_DEV bool all(int key0) const { return key0 >= all_from && key0 + 32 <= all_to; }
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
template <typename T, int HD, Take TAKE>
CRF_DEV void block(const lds_mem *kt, const lds_mem *vt, int key0, const QFrag<T, HD> &q, RowState<HD> &st, float c,
                   int lane, const Seen &seen) {
  const float most = TAKE == CAREFUL && (seen.strict >> lane & 1) ? STRICT : PSUM_MAX;
  const int g = lane / 32;
  f32x16 sc[1];
  scores<T, HD, 1>(kt, q, lane, sc);
  f32x16 &s = sc[0];
  if (!seen.all(key0)) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = key0 + 8 * (v / 4) + 4 * g + v % 4;
      if (key < seen.lo || key > seen.hi) s[v] = -INFINITY;
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

// ---------------------------------------------------------------- schedule

// Row tiles of a sequence and their work in key x row units, a straight line in the
// tile (its keys end where its tokens do) up to a ceiling given by the window:
// work(t) = min(base + (t + 1) BM, cap) + over.
//
// Work is counted in doubles: whole numbers below 2^53, exact, with instructions of
// their own where 64-bit integers take many.
struct SeqWork {
  double base, cap, over;
  int tiles, below, bm;  // below: tiles under the ceiling
  __host__ __device__ double before(int t) const {  // work of the tiles before t
    const double k = below < t ? below : t;
    return k * base + bm * (k * (k + 1) * 0.5) + (t - k) * cap + t * over;
  }
};

// floor(a / b) for whole a >= 0, b > 0: by a reciprocal in 32 bits, put right (a
// division in 64 bits costs three times the instructions)
__host__ __device__ inline double quotient(double a, double b) {
#ifdef __HIP_DEVICE_COMPILE__
  double q = floor(a * (double)__builtin_amdgcn_rcpf((float)b));
#else
  double q = floor(a / b);
#endif
  while (q * b > a) q -= 1;
  while (a - q * b >= b) q += 1;
  return q;
}

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
  int over;                     // keys that a unit costs besides its own
  double pad;                   // and work added by the dealing
  FastDiv g_div;                // by G
  float join;                   // joining a part, in tiles
  bool lead = false;            // `over` lies before a unit's keys, else among them

  __host__ __device__ int by_g(int n) const { return (int)(((uint64_t)(uint32_t)n * g_div.mul) >> g_div.shift); }
  __host__ __device__ SeqWork work(int n, int len) const {
    SeqWork w;  // (rows of a sequence stay below 2^30)
    w.tiles = (int)((unsigned)(n * G + bm - 1) / (unsigned)bm);
    w.bm = bm;
    w.base = (double)(len - n) * G;
    w.cap = 0;
    w.below = w.tiles;
    if (window > 0) {
      w.cap = (double)window * G + bm;
      const double room = w.cap - w.base;
      if (room < (double)w.tiles * bm) w.below = room <= 0 ? 0 : (int)((unsigned)room / (unsigned)bm);
    }
    w.over = (double)over * G + pad;
    return w;
  }
  // All of a sequence's work, or (units) its units.
  __host__ __device__ double seq_work(int n, int len, bool units = false) const {
    const SeqWork w = work(n, len);
    return (units ? (double)w.tiles : w.before(w.tiles)) * nkv;
  }
  __host__ __device__ int first_key(const Task &t) const {  // of the tile's first row
    const int pos = t.len - t.n + by_g(t.tile * bm);
    return window > 0 && pos >= window ? pos - window + 1 : 0;
  }
  __host__ __device__ int last_key(const Task &t) const {  // of the tile's last row
    const int r = (t.tile + 1) * bm, rows = t.n * G;
    return t.len - t.n + by_g((r < rows ? r : rows) - 1);
  }
  // Whether `units` units of `total` work, the longest of a sequence of `longest` tokens,
  // are dealt out whole, and else to how many workgroups their work goes.  In tiles of
  // bkv keys: whole units take `rounds` times the longest one (a single sequence's, longest
  // first, come out even from `MANY` rounds on), stretches the mean and what a part costs
  // besides, SPLIT tiles.  A stretch of s tiles in units of c means s tiles and a join of
  // c / s parts, `join` tiles each, one after the other: no shorter than sqrt(c join).
  struct Plan {
    bool whole;
    double want;
  };
  __host__ __device__ Plan plan(double total, int units, int longest, int slots) const {
    const int most = window > 0 && window < longest - bm ? window + bm : longest;
    const float tile = (float)bkv * G, c = ((float)(most + over) * G + bm) / tile, mean = (float)total / tile / slots;
    const int rounds = (units + slots - 1) / slots;
    const float least = sqrtf(c * join);
    return Plan{rounds >= MANY || rounds * c <= mean + SPLIT, total / (tile * (least > 1.f ? least : 1.f))};
  }
  // Unit i of the sequence's, whole: longest first, its KV heads next to each other.
  __host__ __device__ void whole(int i, Task &t) const {
    const int k = i / nkv;
    t.kvh = i - k * nkv;
    t.tile = work(t.n, t.len).tiles - 1 - k;
    t.t0 = first_key(t) / bkv;
    t.t1 = last_key(t) / bkv + 1;
    t.parts = 1;
  }
  // What workgroup wg, whose stretch ends at `end`, computes from position `at` of
  // all work on, `at` being in the sequence, whose work begins at seq_base; returns
  // where it stops (the end of the unit or of the stretch).  It has no part in the unit
  // when t.part is none of the unit's parts.
  __host__ __device__ double part_at(double at, double end, double share, int wg, double seq_base, Task &t) const {
    const SeqWork w = work(t.n, t.len);
    const double one = w.before(w.tiles), off = at - seq_base;
    t.kvh = (int)quotient(off, one);
    const double rem = off - t.kvh * one;
    int lo = 0, hi = w.tiles;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (w.before(mid) <= rem) lo = mid;
      else hi = mid;
    }
    t.tile = lo;
    const double first = w.before(lo), cost = w.before(lo + 1) - first, u0 = seq_base + t.kvh * one + first,
                 u1 = u0 + cost;
    const double stop = u1 < end ? u1 : end;
    const int k0 = first_key(t) / bkv, k = last_key(t) / bkv + 1 - k0;
    // First key tile of workgroup w's part (both neighbours of a border find it by the same
    // arithmetic).  A first or last part of fewer than SLIVER tiles goes to its neighbour.
    const double ahead = lead ? w.over : 0;
    auto border = [&](int w) {
      const double x = w * share - u0 - ahead;
      return x > 0 ? (int)quotient(x * k, cost - ahead) : 0;
    };
    int last = (int)quotient(u1 - 1, share);
    t.owner = (int)quotient(u0, share);
    while (t.owner < last && border(t.owner + 1) < SLIVER) ++t.owner;
    if (t.owner < last && k - border(last) < SLIVER) --last;
    t.parts = last - t.owner + 1;
    t.part = wg - t.owner;
    t.t0 = k0 + (t.part == 0 ? 0 : border(wg));
    t.t1 = k0 + (t.part == t.parts - 1 ? k : border(wg + 1));
    return stop;
  }
};

// How `total` work is dealt out to `n_wg` workgroups, `share` each: `want` of them, but
// no fewer than there are heads (the sequences' KV heads, which need not wait for each
// other) and no more than `slots`.  one > 0: every head has that much, as
// a single tile; then no border lies inside a head that a neighbour's stretch reaches
// into: heads are padded to whole stretches, or a stretch holds whole heads.
struct Deal {
  double share, pad;  // pad: work added to every unit
  int n_wg;
};
__host__ __device__ inline Deal deal(double total, double want, int heads, double one, int slots) {
  Deal d;
  want = floor(want < heads ? heads : want);
  want = want < slots ? want : slots;
  d.pad = 0;
  if (one > 0 && want >= heads) {
    const double parts = quotient(want, heads);
    d.share = quotient(one + parts - 1, parts);
    d.pad = d.share * parts - one;
    d.n_wg = heads * (int)parts;
  } else if (one > 0) {
    const double per = quotient(heads + want - 1, want);
    d.share = one * per;
    d.n_wg = (int)quotient(heads + per - 1, per);
  } else {
    d.share = quotient(total + want - 1, want);
    d.n_wg = (int)want;  // (the last ones' stretches may begin past the end)
  }
  return d;
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

// The value of lane `from` in every lane (a wave-uniform value).
CRF_DEV int lane_value(int v, int from) { return __builtin_amdgcn_readlane(v, from); }
CRF_DEV double lane_value(double v, int from) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)lane_value((int)(u >> 32), from) << 32 |
                                        (uint32_t)lane_value((int)u, from));
}

// What a workgroup computes, unit after unit.  Every wave works it out for itself,
// 64 sequences at a time, so that nothing waits for a barrier.
struct Schedule {
  const PagedAttn &p;
  Shape sh;
  int slots;
  bool sizes;         // units differ (tiles of 128 rows): whether they are split is decided here
  bool many = false;  // units dealt out whole, gridDim.x apart; else stretches of work
  bool dealt = false;
  int wg = 0;
  double share = 0, at = -1, end = 0;  // many: next unit and their number; else the stretch [at, end) of all work
  int seq = -1, start = 0, n = 0, len = 0;  // the sequence that holds `at` ...
  double base = 0, work = 0;                // ... and where its work begins, and how much it is

  struct Lane {  // a lane's sequence, its work and where that begins
    int s, start, n, len;
    double v, from;
    int units, longest;
  };

  // Prefix sums over the sequences of their work (units: of their units), of which the
  // total is returned; finds the sequence that holds position x, and leaves each lane
  // its last sequence and, when `sizes`, its sequences' units and longest.
  CRF_DEV double pass(double x, bool units, Lane &q, bool sizes = false) {
    const int lane = threadIdx.x % 64;
    double done = 0;
    q.units = q.longest = 0;
#pragma unroll 1
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += 64) {
      q.s = s0 + lane;
      q.start = q.len = 0;
      q.n = q.s < p.b.n_seqs ? seq_new(p.b, q.s, q.start, q.len) : 0;
      q.v = q.n > 0 ? sh.seq_work(q.n, q.len, units) : 0;
      if (sizes && q.n > 0) {
        q.units += sh.work(q.n, q.len).tiles * sh.nkv;
        q.longest = max(q.longest, q.len);
      }
      double sum = q.v;
      wave_prefix([&](auto c, auto rows) { sum += from_lane<c(), rows()>(sum); });
      q.from = done + sum - q.v;
      hold(x, q);
      done += lane_value(sum, 63);
    }
    return done;
  }

  CRF_DEV void hold(double x, const Lane &q) {
    const uint64_t m = __builtin_amdgcn_ballot_w64(q.v > 0 && x >= q.from && x < q.from + q.v);
    if (m) {
      const int l = __builtin_ctzll(m);
      seq = lane_value(q.s, l);
      start = lane_value(q.start, l);
      n = lane_value(q.n, l);
      len = lane_value(q.len, l);
      base = lane_value(q.from, l);
      work = lane_value(q.v, l);
    }
  }

  // The next task; false: done.
  CRF_DEV bool next(Task &t) {
    if (!dealt) {
      dealt = true;
      Lane q;
      double total = pass(-1, false, q, sizes);
      if (total == 0) return false;
      double want;
      if (sizes) {
        wave_prefix([&](auto c, auto rows) {
          q.units += from_lane<c(), rows()>(q.units);
          q.longest = max(q.longest, from_lane<c(), rows()>(q.longest));
        });
        const int units = lane_value(q.units, 63);
        const Shape::Plan plan = sh.plan(total, units, lane_value(q.longest, 63), slots);
        many = plan.whole;
        want = plan.want;
        end = units;
      } else {
        want = total * p.per_wg;
      }
      if (many) {
        at = blockIdx.x;
      } else {
        // sequences of one tile and one length?
        double one = 0;
        int heads = p.b.n_seqs * sh.nkv;
        const uint64_t active = __builtin_amdgcn_ballot_w64(q.v > 0);
        if (p.b.n_seqs <= 64) {
          const double v = lane_value(q.v, __builtin_ctzll(active));
          heads = __popcll(active) * sh.nkv;
          if (!__builtin_amdgcn_ballot_w64(q.v > 0 && (q.v != v || q.n * sh.G > sh.bm))) one = v / sh.nkv;
        }
        const Deal d = deal(total, want, heads, one, slots);
        share = lane_value(d.share, 0);
        sh.pad = lane_value(d.pad, 0);
        wg = stretch_of(blockIdx.x, __builtin_amdgcn_readfirstlane(d.n_wg));
        if (wg < 0) return false;
        total += sh.pad * heads;
        at = wg * share;
        end = at + share < total ? at + share : total;
        if (__builtin_amdgcn_readfirstlane(at >= end)) return false;
        if (p.b.n_seqs <= 64) {  // the pass has seen them all
          if (q.v > 0) {
            q.from += sh.pad * sh.nkv * __popcll(active & (((uint64_t)1 << (threadIdx.x % 64)) - 1));
            q.v += sh.pad * sh.nkv;
          }
          hold(at, q);
        } else {
          pass(at, false, q);
        }
      }
    }
#pragma unroll 1
    for (;;) {
      if (__builtin_amdgcn_readfirstlane(at >= end)) return false;
      if (many) {
        Lane q;
        pass(at, true, q);
        if (__builtin_amdgcn_readfirstlane(!(at >= base && at < base + work))) return false;
      } else {
#pragma unroll 1
        while (__builtin_amdgcn_readfirstlane(at >= base + work)) {  // (some sequence holds `at`)
          base += work;
          if (++seq >= p.b.n_seqs) return false;
          n = seq_new(p.b, seq, start, len);
          work = n > 0 ? sh.seq_work(n, len) : 0;
        }
      }
      t.seq = __builtin_amdgcn_readfirstlane(seq);
      t.start = __builtin_amdgcn_readfirstlane(start);
      t.n = __builtin_amdgcn_readfirstlane(n);
      t.len = __builtin_amdgcn_readfirstlane(len);
      if (many) {
        sh.whole(__builtin_amdgcn_readfirstlane((int)(at - base)), t);
        at += gridDim.x;
        break;
      }
      at = lane_value(sh.part_at(at, end, share, wg, base, t), 0);
      t.part = __builtin_amdgcn_readfirstlane(t.part);
      if (t.part >= 0 && t.part < __builtin_amdgcn_readfirstlane(t.parts)) break;
    }
    t.kvh = __builtin_amdgcn_readfirstlane(t.kvh);
    t.tile = __builtin_amdgcn_readfirstlane(t.tile);
    t.t0 = __builtin_amdgcn_readfirstlane(t.t0);
    t.t1 = __builtin_amdgcn_readfirstlane(t.t1);
    t.parts = __builtin_amdgcn_readfirstlane(t.parts);
    t.owner = __builtin_amdgcn_readfirstlane(t.owner);
    return true;
  }
};

template <typename T, int HD>
struct Writer {
  const PagedAttn &p;
  const Task &t;
  const Shape &sh;
  int rows;  // of the tile

  // Row r of the tile: its token and head, o / l from element e on (NF groups of 4
  // elements, 8 apart), and the row's log-sum.
  template <int NF>
  CRF_DEV void out(int r, int e, const f32x4 (&o)[NF], float ref, float l) const {
    const int a = t.tile * sh.bm + r, k = sh.by_g(a), head = t.kvh * sh.G + a - k * sh.G;
    const int64_t token = t.start + k;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *dst = (T *)p.out + token * p.out_ld + head * HD + e;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const f32x4 x = o[i] * inv;
      if constexpr (sizeof(T) == 2)
        st8(dst + 8 * i, pack_bf16x4(x[0], x[1], x[2], x[3]));
      else
        *reinterpret_cast<f32x4 *>(dst + 8 * i) = x;
    }
    if (e == 0 && p.lse)
      p.lse[token * p.nq + head] = l == 0.f ? -INFINITY : 0.69314718055994531f * (ref + __builtin_amdgcn_logf(l));
  }
};

// Partials of unit parts, 2 a workgroup: BM x HD floats, and behind all of them BM
// pairs (reference, sum).  They are stored past the caches of the XCD, which are not
// coherent with each other, 16 bytes a lane.
template <int HD, int BM>
struct Partials {
  const PagedAttn &p;
  int slots;

  CRF_DEV float *o(int slot) const { return p.part + (int64_t)slot * BM * HD; }
  CRF_DEV float2 *ml(int slot) const {
    return (float2 *)(p.part + (int64_t)2 * slots * BM * HD) + (int64_t)slot * BM;
  }
  CRF_DEV void store(int slot, int at, f32x4 v) const {  // four floats from `at` on
    constexpr int DEVICE = 16;  // cache policy: device scope
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), make_rsrc(o(slot), BM * HD * 4), at * 4, 0,
                                           DEVICE);
  }
  CRF_DEV void store_ml(int slot, int r, float ref, float l) const {
    __hip_atomic_store((uint64_t *)(ml(slot) + r),
                       (uint64_t)__builtin_bit_cast(uint32_t, ref) | (uint64_t)__builtin_bit_cast(uint32_t, l) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

// Counts this workgroup's part of the unit as done; true for the one that finishes
// last, which may then read all parts.
CRF_DEV bool part_done(const PagedAttn &p, const Task &t, int &last) {
  agent_flush();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = agent_ticket(&p.tickets[t.owner]) == (unsigned)t.parts - 1;
    if (last) __hip_atomic_store(&p.tickets[t.owner], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return false;
  // the others' parts are in memory: no line of them may be left in a cache
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  return true;
}

// What O to the reference `from` weighs next to the reference `to`: never zero, so that its
// infinities stay (2^-149 of the largest finite number is 2^-21).
CRF_DEV float rescale(float from, float to) { return fmaxf(fast_exp2(from - to), 0x1p-149f); }

// A row's running result over parts: U parts' references, sums and weights at a time.
template <int U>
struct Joined {
  float ref = -INFINITY, l = 0.f, alpha, w[U];
  // Parts k0 .. of row r: what the sum so far (alpha) and each part's O (w) weigh.  A part
  // of which the row sees nothing weighs nothing.
  template <typename P>
  CRF_DEV void add(const P &parts, const Task &t, int k0, int r) {
    float2 m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = parts.ml(part_slot(t.owner, min(k0 + u, t.parts - 1)))[r];
    float top = ref;
    bool some[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      some[u] = k0 + u < t.parts && m[u].y != 0.f;
      if (some[u]) top = fmaxf(top, m[u].x);
    }
    alpha = l == 0.f ? 0.f : rescale(ref, top);
    l *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = some[u] ? rescale(m[u].x, top) : 0.f;
      l += w[u] * m[u].y;
    }
    ref = top;
  }
  CRF_DEV void plus(f32x4 &o, int u, f32x4 x) const {  // (what is behind the last part stays out)
#pragma unroll
    for (int v = 0; v < 4; ++v) o[v] = w[u] != 0.f ? fmaf(w[u], x[v], o[v]) : o[v];
  }
};

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

// ---------------------------------------------------------------- tiles of 128 rows

template <typename T, int HD, bool UNI>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(const PagedAttn p, int slots) {
  using L = Layout<T, HD>;
  constexpr int NW = 4, NT = 64 * NW, BM = 32 * NW, BKV = sizeof(T) == 2 ? 64 : 32, TILE = BKV * L::ROWB;
  __shared__ __align__(16) char stages[2][2 * TILE];  // K, then V
  __shared__ int pg[PGCAP];
  __shared__ int bad, last;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  // A unit costs 256 keys besides its own (with 0 the 12 sequences take 103 us instead of
  // 71, 4096 tokens 156 instead of 91); a part in a join 1.3 tiles, 0.3 of the slower fp32
  // ones (with none 1000 tokens take 38 us instead of 30).
  Schedule sch{p, Shape{p.nq / p.nkv, p.nkv, p.window, BM, BKV, 256, 0, p.g_div, sizeof(T) == 2 ? 1.3f : 0.3f, true},
               slots, true};
  const Shape &sh = sch.sh;
  const Partials<HD, BM> parts{p, slots};
  const int far = p.window > 0 ? p.window - 1 : INT32_MAX;  // keys before its own that a row sees
  Task t;
#pragma unroll 1
  while (sch.next(t)) {
    const int rows = min(BM, t.n * sh.G - t.tile * BM);
    const Writer<T, HD> wr{p, t, sh, rows};
    const int base = t.len - t.n, row0 = t.tile * BM;
    // this lane's row (padding rows repeat the last one)
    const int r = wave * 32 + l32, row = row0 + min(r, rows - 1);
    const int tok = sh.by_g(row), head = t.kvh * sh.G + row - tok * sh.G, pos = base + tok;
    const int pos_lo = base + sh.by_g(row0 + min(wave * 32, rows - 1));
    const int pos_hi = base + sh.by_g(row0 + min(wave * 32 + 31, rows - 1));
    QFrag<T, HD> q;
    q.load((const T *)p.q + (int64_t)(t.start + tok) * p.q_ld + head * HD, g);
    RowState<HD> st;
    Pages<T, HD, UNI, BKV / NW> pages{p.b, p.zeros, pg, &bad, 0, t.len, t.kvh, wave * (BKV / NW), lane,
                                      p.b.tables + (int64_t)t.seq * p.b.table_stride};
    const int first_seen = pos_lo > far ? pos_lo - far : 0, last_first = pos_hi > far ? pos_hi - far : 0;
    const int whole_to = wave * 32 < rows ? pos_lo + 1 : 0;  // keys before it are seen by every row of the wave
    const int end_key = t.t1 * BKV;
    if (tid == 0) bad = 0;
    bool careful = false, strictly = false;  // (as a counter: 157 registers spilled instead of 99, fp32 heads of 128)
    uint64_t strict = 0;
#pragma unroll 1
    for (;;) {
      st.clear();
      __syncthreads();  // the task (or the pass) before has left LDS
      const lds_mem *mem = (const lds_mem *)&stages[0][0];
      auto load = [&](int it, int stage) {
        const lds_mem *k = mem + stage * 2 * TILE;
        pages.load(it * BKV + wave * (BKV / NW), k, k + TILE);
      };
      if (t.t0 < t.t1) {
        pages.fill(div_by(t.t0 * BKV, p.b.ps_div), end_key, NT);
        __syncthreads();
        load(t.t0, 0);
      }
      // A tile's data is there, the next one's is on its way (each wave passes here once a
      // tile, wherever it then goes).
      auto arrive = [&](int it) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (it + 1 < t.t1) {
          if (div_by(min((it + 2) * BKV, t.len) - 1, p.b.ps_div) >= pages.first + PGCAP) {
            pages.fill(div_by(it * BKV, p.b.ps_div), end_key, NT);
            __syncthreads();
          }
          load(it + 1, (it + 1 - t.t0) & 1);
        }
      };
      q.arrived();
#pragma unroll 1
      for (int it = t.t0; it < t.t1;) {
        // tiles that every row of the wave sees; the first block of all gives the rows
        // their reference
        int taken = 0;  // blocks of the tile
        for (;;) {
          arrive(it);
          const int kt0 = it * BKV;
          if (it == t.t0 || kt0 + BKV > whole_to || kt0 < last_first || bad || careful) break;
          const lds_mem *kt = mem + ((it - t.t0) & 1) * 2 * TILE;
          taken = whole_blocks<T, HD, BKV / 32>(kt, kt + TILE, q, st, p.scale_log2, lane);
          if (taken < BKV / 32) break;
          taken = 0;
          if (++it == t.t1) break;
        }
        if (it == t.t1) break;
        const int kt0 = it * BKV;
        if (wave * 32 < rows && kt0 <= pos_hi && kt0 + BKV > first_seen) {
          const Seen seen{pos > far ? pos - far : 0, pos,         last_first, whole_to, t.len, bad != 0, pg,
                          pages.first,               p.b.ps_div, strict};
          const lds_mem *kt = mem + ((it - t.t0) & 1) * 2 * TILE;
#pragma unroll 1
          for (int kb = 32 * taken; kb < BKV; kb += 32)
            if (careful)
              block<T, HD, CAREFUL>(kt + kb * L::ROWB, kt + TILE + kb * L::ROWB, kt0 + kb, q, st, p.scale_log2, lane,
                                    seen);
            else
              block<T, HD, SOME>(kt + kb * L::ROWB, kt + TILE + kb * L::ROWB, kt0 + kb, q, st, p.scale_log2, lane,
                                 seen);
        }
        ++it;
      }
      // (a barrier after every pass: the next task clears `bad`, which the last tile reads)
      const uint64_t odd = not_finite(st);
      const bool again = __syncthreads_or(odd != 0);
      if (strictly || !again) break;
      if (careful) strict = odd;
      strictly = careful;
      careful = true;
    }

    const float l = st.l + __shfl_xor(st.l, 32, 64);
    f32x4 o[4 * L::HB];
#pragma unroll
    for (int i = 0; i < 4 * L::HB; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[i][v] = st.o[i / 4][4 * (i % 4) + v];
    if (t.parts == 1) {
      if (r < rows) wr.out(r, 4 * g, o, st.ref, l);
      continue;
    }
    // (partials in the order of the fragments: a load or store of a wave is 1 KiB in a row)
    const int slot = part_slot(t.owner, t.part), mine = (wave * 4 * L::HB * 64 + lane) * 4;
#pragma unroll
    for (int i = 0; i < 4 * L::HB; ++i) parts.store(slot, mine + 256 * i, o[i]);
    if (g == 0) parts.store_ml(slot, r, st.ref, l);
    if (!part_done(p, t, last)) continue;
#pragma unroll 1
    for (int b = 0; b < L::HB; ++b) {
      constexpr int U = 4;
      Joined<U> j;
      f32x4 sum[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int k = 0; k < t.parts; k += U) {
        f32x4 x[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[u][i] = *(const f32x4 *)(parts.o(part_slot(t.owner, min(k + u, t.parts - 1))) + mine + 256 * (4 * b + i));
        j.add(parts, t, k, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum[i] *= j.alpha;
#pragma unroll
          for (int u = 0; u < U; ++u) j.plus(sum[i], u, x[u][i]);
        }
      }
      if (r < rows) wr.out(r, 32 * b + 4 * g, sum, j.ref, j.l);
    }
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
__global__ __launch_bounds__((64 * KeysCfg<T, HD>::NW), (KeysCfg<T, HD>::WG_PER_CU)) void attn_keys_kernel(
    const PagedAttn p, int slots) {
  using L = Layout<T, HD>;
  constexpr int NW = KeysCfg<T, HD>::NW, NT = 64 * NW, BM = 32, BKV = 32 * NW, TILE = BKV * L::ROWB;
  constexpr int LOADS = 2 * 32 / L::RPI;  // of a wave's stage
  __shared__ __align__(16) char stages[2][2 * TILE];  // K, then V
  __shared__ int pg[PGCAP];
  __shared__ float2 wml[NW][32];
  __shared__ int bad, last;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 32, l32 = lane % 32;
  Schedule sch{p, Shape{p.nq / p.nkv, p.nkv, p.window, BM, BKV, 256, 0, p.g_div, 0}, slots, false};
  const Shape &sh = sch.sh;
  const Partials<HD, BM> parts{p, slots};
  const int far = p.window > 0 ? p.window - 1 : INT32_MAX;
  Task t;
#pragma unroll 1
  while (sch.next(t)) {
    const int rows = min(BM, t.n * sh.G - t.tile * BM);
    const Writer<T, HD> wr{p, t, sh, rows};
    const int base = t.len - t.n, row0 = t.tile * BM;
    const int row = row0 + min(l32, rows - 1);
    const int tok = sh.by_g(row), head = t.kvh * sh.G + row - tok * sh.G, pos = base + tok;
    const int pos_lo = base + sh.by_g(row0), pos_hi = base + sh.by_g(row0 + rows - 1);
    QFrag<T, HD> q;
    q.load((const T *)p.q + (int64_t)(t.start + tok) * p.q_ld + head * HD, g);
    RowState<HD> st;
    Pages<T, HD, UNI, 32> pages{p.b, p.zeros, pg, &bad, 0, t.len, t.kvh, wave * 32, lane,
                                p.b.tables + (int64_t)t.seq * p.b.table_stride};
    const int first_seen = pos_lo > far ? pos_lo - far : 0, last_first = pos_hi > far ? pos_hi - far : 0;
    if (tid == 0) bad = 0;
    uint64_t strict = 0;
#pragma unroll 1
    for (int pass = 0;; ++pass) {
      const bool careful = pass > 0;
      st.clear();
      __syncthreads();  // the task (or the pass) before has left LDS
      // stretches of tiles whose pages fit the staged table
#pragma unroll 1
      for (int a = t.t0; a < t.t1;) {
        const int fp = div_by(a * BKV, p.b.ps_div);
        // (whole tiles before the end of the staged pages)
        const int64_t tiles = ((int64_t)fp + PGCAP) * p.b.page_size / BKV;
        const int z = tiles < t.t1 ? (int)tiles : t.t1;
        pages.fill(fp, z * BKV, NT);
        __syncthreads();
        const Seen seen{pos > far ? pos - far : 0, pos, last_first, pos_lo + 1, t.len, bad != 0, pg, fp, p.b.ps_div,
                        strict};
        const lds_mem *mem = (const lds_mem *)&stages[0][0];
        auto load = [&](int it) {
          const lds_mem *k = mem + ((it - a) & 1) * 2 * TILE;
          pages.load(it * BKV + wave * 32, k, k + TILE);
        };
        // The wave's loads of a tile have arrived; those of the next one stay in flight.
        auto arrive = [&](int it) {
          if (it + 1 < z)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
          else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        };
        auto leave = [&](int it) {  // the stage is read before it is loaded again
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (it + 2 < z) load(it + 2);
        };
        load(a);
        if (a + 1 < z) load(a + 1);
        q.arrived();
#pragma unroll 1
        for (int it = a; it < z;) {
          for (;;) {
            arrive(it);
            const int key0 = it * BKV + wave * 32;
            if (it == t.t0 || !seen.all(key0) || seen.bad || careful) break;
            const lds_mem *kt = mem + ((it - a) & 1) * 2 * TILE + wave * 32 * L::ROWB;
            if (!whole_blocks<T, HD, 1>(kt, kt + TILE, q, st, p.scale_log2, lane)) break;
            leave(it);
            if (++it == z) break;
          }
          if (it == z) break;
          const int key0 = it * BKV + wave * 32;
          if (key0 <= pos_hi && key0 + 32 > first_seen) {
            const lds_mem *kt = mem + ((it - a) & 1) * 2 * TILE + wave * 32 * L::ROWB;
            if (careful)
              block<T, HD, CAREFUL>(kt, kt + TILE, key0, q, st, p.scale_log2, lane, seen);
            else
              block<T, HD, SOME>(kt, kt + TILE, key0, q, st, p.scale_log2, lane, seen);
          }
          leave(it);
          ++it;
        }
        a = z;
        __syncthreads();
      }
      const uint64_t odd = not_finite(st);
      if (pass == 2 || !__syncthreads_or(odd != 0)) break;
      if (pass == 1) strict = odd;
    }

    // join the waves: O of wave w at 32 x HD floats w of the stages
    const float lw = st.l + __shfl_xor(st.l, 32, 64);
    auto osum = [&](int w) { return (f32x4 *)&stages[0][0] + w * 32 * (HD / 4); };
    static_assert(NW * 32 * HD * 4 <= 4 * TILE, "O of all waves");
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
        const float k = rescale(m.x, ref);
        l += k * m.y;
        o += k * osum(w)[r * (HD / 4) + (c4 ^ (r & 15))];
      }
      if (t.parts == 1) {
        const f32x4 one[1] = {o};
        wr.out(r, 4 * c4, one, ref, l);
      } else {
        const int slot = part_slot(t.owner, t.part);
        parts.store(slot, 4 * i, o);
        if (c4 == 0) parts.store_ml(slot, r, ref, l);
      }
    }
    if (t.parts == 1 || !part_done(p, t, last)) continue;
#pragma unroll 1
    for (int i = tid; i < rows * (HD / 4); i += NT) {
      const int r = i / (HD / 4);
      constexpr int U = 16;
      Joined<U> j;
      f32x4 o[1] = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll 1
      for (int k = 0; k < t.parts; k += U) {
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          x[u] = *(const f32x4 *)(parts.o(part_slot(t.owner, min(k + u, t.parts - 1))) + 4 * i);
        j.add(parts, t, k, r);
        o[0] *= j.alpha;
#pragma unroll
        for (int u = 0; u < U; ++u) j.plus(o[0], u, x[u]);
      }
      wr.out(r, 4 * (i % (HD / 4)), o, j.ref, j.l);
    }
  }
}

template <typename T, int HD, bool UNI>
hipError_t launch(hipStream_t s, PagedAttn p) {
  const int G = p.nq / p.nkv;
  // Tiles of 32 rows for up to 32 rows to a sequence and KV head (with tiles of 128 the
  // steps above take 33 us instead of 13.6 and 196 instead of 154), and where all of them
  // together read so few keys, as far as the host can tell, that four times the reads of
  // K and V cost less than the parts of long units.
  const int64_t row_tiles = ((int64_t)p.b.n_rows * G / 32 + p.b.n_seqs) * p.nkv;
  const int64_t longest = std::min<int64_t>((int64_t)p.b.max_pages * p.b.page_size, (int64_t)1 << 24);
  const bool keys = (int64_t)p.b.max_new * G <= 32 ||
                    (row_tiles < (1 << 16) && row_tiles * longest * 2 * HD * (int)sizeof(T) <= SMALL_READS);
  const int bm = keys ? 32 : 128;
  p.g_div = fast_div(G);
  const int resident = p.n_cu * (keys ? KeysCfg<T, HD>::WG_PER_CU : 2);
  const int64_t room = p.part_floats / (2 * bm * (HD + 2));  // two slots a workgroup
  int slots = (int)(room < resident ? room : resident);
  if (slots > PAGED_TICKETS) slots = PAGED_TICKETS;
  slots = slots / 8 * 8;
  if (slots < 8) return hipErrorOutOfMemory;  // (no context is that small)
  // (a sequence's last tile may be short)
  const int64_t most = ((int64_t)p.b.n_rows * G / bm + p.b.n_seqs) * p.nkv;
  // (a tile of 128 keys takes a workgroup alone on its CU 1 us, a part in a join 0.1 us)
  p.per_wg = 1.0 / (256.0 * G);
  const int64_t grid = !keys && most >= (int64_t)MANY * slots ? most : slots;
  const dim3 g((unsigned)(grid < MOST_GROUPS ? grid : MOST_GROUPS));
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
