// How paged attention's launches are planned, walked on the host: a window that no
// sequence reaches plans as none does; and over ragged batches, tiles of 32 rows with
// many to a sequence among them, the plan's choice (whole units, or stretches of work
// over a grid of as many workgroups as there are slots, or as a launch has row tiles)
// computes every key tile of every unit once.  Compiled with -fwrapv: integers wrap, as
// on the device.  Prints the number of plans and batches checked.
#include <climits>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2609_30884_amd/csrc/paged_attn.hip"

using namespace crf;

static std::mt19937 rng(11);
static int upto(int n) { return (int)(rng() % (unsigned)(n + 1)); }

static int windows(int &checked) {
  for (int it = 0; it < 3000; ++it) {
    const int G = 1 + upto(15), bm = it % 2 ? 32 : 128, slots = 8 * (1 + upto(63));
    const int longest = 1 + upto(upto(1) ? 4000 : 1 << 30), units = 1 + upto(4000);
    const double total = (double)units * (1 + upto(1 << 20));
    auto plan = [&](int window) {
      const Shape sh{G, 2, window, bm, bm == 32 ? 128 : 64, 256, 0, fast_div(G), 1.3f, true};
      return sh.plan(total, units, longest, slots);
    };
    const Shape::Plan none = plan(0);
    for (int window : {INT32_MAX, INT32_MAX - 1, INT32_MAX - 31, INT32_MAX - 128, INT32_MAX - 129, longest}) {
      if (window < longest) continue;
      const Shape::Plan p = plan(window);
      if (p.whole != none.whole || p.want != none.want) {
        std::printf("window %d, %d tokens: whole %d, want %g; without it %d, %g\n", window, longest, p.whole, p.want,
                    none.whole, none.want);
        return 1;
      }
      ++checked;
    }
  }
  return 0;
}

static int batches(int &checked, int &whole, int &wide) {
  for (int it = 0; it < 1500; ++it) {
    const int nkv = 1 + upto(7), G = 1 + upto(8), bm = it % 2 ? 32 : 128, slots = 8 * (1 + upto(it % 7 ? 63 : 3));
    const int window = upto(2) ? 0 : upto(1) ? INT32_MAX - upto(200) : 1 + upto(3000);
    Shape sh{G, nkv, window, bm, bm == 32 ? 128 : 64, 256, 0, fast_div(G), upto(1) ? 1.3f : 0.3f, bm == 128};
    const int seqs = 1 + upto(20);
    std::vector<int> n(seqs), len(seqs), first(seqs);
    double total = 0;
    int units = 0, longest = 0, rows = 0;
    for (int s = 0; s < seqs; ++s) {
      n[s] = upto(5) ? 1 + upto(1 + upto(700)) : 0;
      len[s] = n[s] + upto(upto(2) ? 600 : 20000);
      rows += n[s];
      first[s] = units;
      if (n[s] == 0) continue;
      total += sh.seq_work(n[s], len[s]);
      units += sh.work(n[s], len[s]).tiles * nkv;
      longest = std::max(longest, len[s]);
    }
    if (units == 0) continue;
    rows += upto(3) ? 0 : 100000;  // rows of nobody, which the host cannot tell from others
    const int64_t most = ((int64_t)rows * G / bm + seqs) * nkv;
    const int grid = most >= (int64_t)MANY * slots ? (int)most : slots;
    std::vector<std::vector<char>> seen(units);
    auto unit = [&](const Task &t, int &k0, int &k1) -> std::vector<char> & {
      const int64_t r0 = (int64_t)t.tile * bm, r1 = std::min<int64_t>(r0 + bm, (int64_t)t.n * G) - 1;
      const int64_t p0 = t.len - t.n + r0 / G, p1 = t.len - t.n + r1 / G;
      k0 = (int)((window ? std::max<int64_t>(0, p0 - window + 1) : 0) / sh.bkv);
      k1 = (int)(p1 / sh.bkv) + 1;
      std::vector<char> &u = seen[first[t.seq] + t.kvh * sh.work(t.n, t.len).tiles + t.tile];
      u.resize(k1);
      return u;
    };
    auto take = [&](const Task &t) {
      int k0, k1;
      if (t.kvh < 0 || t.kvh >= nkv || t.tile < 0 || (int64_t)t.tile * bm >= (int64_t)t.n * G) return 1;
      std::vector<char> &u = unit(t, k0, k1);
      if (t.t0 < k0 || t.t1 > k1 || t.t0 > t.t1) return 2;
      for (int k = t.t0; k < t.t1; ++k)
        if (u[k]++) return 3;
      return 0;
    };
    auto holds = [&](double at, bool by_units, double &base) {
      base = 0;
      for (int s = 0; s < seqs; ++s) {
        const double w = n[s] > 0 ? sh.seq_work(n[s], len[s], by_units) : 0;
        if (at < base + w) return s;
        base += w;
      }
      return -1;
    };
    const Shape::Plan plan = sh.plan(total, units, longest, slots);
    int wrong = 0;
    if (plan.whole && bm == 128) {  // (tiles of 32 rows are always dealt as stretches)
      ++whole;
      for (int bid = 0; bid < grid; ++bid)
        for (double at = bid; at < units && !wrong; at += grid) {
          double base;
          const int s = holds(at, true, base);
          Task t{};
          t.seq = s, t.n = n[s], t.len = len[s];
          sh.whole((int)(at - base), t);
          wrong = take(t);
        }
    } else {
      wide += grid > slots;
      const double want = bm == 32 ? total / (256.0 * G) : plan.want;
      const Deal d = deal(total, want, seqs * nkv, 0, slots);
      int stretches = 0;
      for (int bid = 0; bid < grid && !wrong; ++bid) {
        const int wg = stretch_of(bid, d.n_wg);
        if (wg < 0) continue;
        ++stretches;
        const double end = std::min((wg + 1) * d.share, total);
        for (double at = wg * d.share; at < end && !wrong;) {
          double base;
          const int s = holds(at, false, base);
          Task t{};
          t.seq = s, t.n = n[s], t.len = len[s];
          const double stop = sh.part_at(at, end, d.share, wg, base, t);
          if (stop <= at) wrong = 4;
          at = stop;
          if (t.part < 0 || t.part >= t.parts) continue;
          if (t.owner < 0 || t.owner + t.parts > slots) wrong = 5;
          if (!wrong) wrong = take(t);
        }
      }
      if (!wrong && stretches != d.n_wg) wrong = 6;
    }
    for (int s = 0; s < seqs && !wrong; ++s)
      for (int h = 0; n[s] > 0 && h < nkv; ++h)
        for (int i = 0; i < sh.work(n[s], len[s]).tiles && !wrong; ++i) {
          Task t{};
          t.seq = s, t.n = n[s], t.len = len[s], t.kvh = h, t.tile = i;
          int k0, k1;
          std::vector<char> &u = unit(t, k0, k1);
          for (int k = k0; k < k1; ++k)
            if (u[k] != 1) wrong = 7;
        }
    if (wrong) {
      std::printf("batch %d: %d\n", it, wrong);
      return 1;
    }
    ++checked;
  }
  return 0;
}

int main() {
  int checked = 0, whole = 0, wide = 0;
  if (windows(checked) || batches(checked, whole, wide)) return 1;
  if (whole < 50 || wide < 50) {
    std::printf("%d batches of whole units, %d of stretches over more workgroups than slots\n", whole, wide);
    return 1;
  }
  std::printf("ok %d\n", checked);
  return 0;
}
