// The decomposition of paged attention into workgroups, walked on the host: over
// many ragged batches every key tile of every unit is computed exactly once, a
// unit's parts are those that its owner counts, and no two partials share a slot.
// Prints the number of batches checked.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "../../paper_2609_30884_amd/csrc/paged_attn.hip"

using namespace crf;

static int fail(const char *what, int batch) {
  std::printf("batch %d: %s\n", batch, what);
  return 1;
}

int main() {
  std::mt19937 rng(7);
  auto upto = [&](int n) { return (int)(rng() % (unsigned)(n + 1)); };
  int checked = 0;
  for (int it = 0; it < 4200; ++it) {
    const int nkv = 1 + upto(7), G = 1 + upto(8), bm = it % 2 ? 32 : 128;
    const int window = upto(3) ? 0 : 1 + upto(3000);
    Shape sh{G, nkv, window, bm, bm == 32 ? 128 : 64, upto(600), 0, fast_div(G), 1.f, it % 3 == 0};
    const int slots = 8 * (1 + upto(63)), seqs = 1 + upto(40);
    const int most_new = bm == 32 ? (32 / G > 0 ? 32 / G : 1) : 1 + upto(1 + upto(2000));
    std::vector<int> n(seqs), len(seqs);
    double total = 0;
    int64_t units = 0;
    for (int s = 0; s < seqs; ++s) {
      n[s] = upto(9) ? upto(most_new) : 0;
      len[s] = n[s] + upto(upto(3) ? 500 : 20000);
      if (it % 5 == 0) len[s] = len[0] - n[0] + n[s], n[s] = n[s] ? n[0] : 0;  // alike, some idle
      if (it % 5 == 0 && n[s]) len[s] = len[0];
      if (n[s] == 0) continue;
      total += sh.seq_work(n[s], len[s]);
      units += (int64_t)sh.work(n[s], len[s]).tiles * nkv;
    }
    auto rows_keys = [&](const Task &t, int &k0, int &k1) {
      const int64_t r0 = (int64_t)t.tile * bm, r1 = std::min<int64_t>(r0 + bm, (int64_t)t.n * G) - 1;
      const int p0 = t.len - t.n + (int)(r0 / G), p1 = t.len - t.n + (int)(r1 / G);
      k0 = (window ? std::max(0, p0 - window + 1) : 0) / sh.bkv;
      k1 = p1 / sh.bkv + 1;
    };
    // whole units
    int64_t seen = 0;
    for (int s = 0; s < seqs; ++s) {
      if (n[s] == 0) continue;
      std::set<std::pair<int, int>> got;
      for (int64_t i = 0; i < (int64_t)sh.work(n[s], len[s]).tiles * nkv; ++i, ++seen) {
        Task t{};
        t.n = n[s];
        t.len = len[s];
        sh.whole(i, t);
        int k0, k1;
        rows_keys(t, k0, k1);
        if (t.kvh < 0 || t.kvh >= nkv || t.tile < 0 || (int64_t)t.tile * bm >= (int64_t)n[s] * G)
          return fail("whole unit out of range", it);
        if (t.t0 != k0 || t.t1 != k1 || !got.insert({t.kvh, t.tile}).second) return fail("whole unit's keys", it);
      }
    }
    if (seen != units) return fail("number of units", it);
    if (total == 0) continue;
    // dealt out
    double one = 0;
    int heads = 0;
    bool alike = true;
    for (int s = 0; s < seqs; ++s) {
      if (n[s] == 0) continue;
      heads += nkv;
      alike &= n[s] * G <= bm && (one == 0 || sh.seq_work(n[s], len[s]) == one * nkv);
      one = sh.seq_work(n[s], len[s]) / nkv;
    }
    const Deal d = deal(total, total / (1.0 + upto(600)) / G, heads, alike ? one : 0, slots);
    const double share = d.share;
    const int n_wg = d.n_wg;
    sh.pad = d.pad;
    total += d.pad * heads;
    if (n_wg < 1 || n_wg > slots) return fail("more workgroups than slots", it);
    if (n_wg * share < total) return fail("work that nobody gets", it);
    std::set<int> stretches;
    for (int b = 0; b < slots; ++b) {
      const int wg = stretch_of(b, n_wg);
      if (wg >= 0 && !stretches.insert(wg).second) return fail("a stretch twice", it);
    }
    if ((int)stretches.size() != n_wg) return fail("a stretch that nobody takes", it);
    std::map<std::tuple<int, int, int>, std::vector<Task>> unit;
    std::set<int> slot, owner;
    for (int wg = 0; wg < n_wg; ++wg) {
      double at = wg * share;
      const double end = std::min(at + share, total);
      while (at < end) {
        double base = 0;
        int s = 0;
        for (;; ++s) {
          const double w = n[s] > 0 ? sh.seq_work(n[s], len[s]) : 0;
          if (at < base + w) break;
          base += w;
        }
        Task t{};
        t.seq = s;
        t.n = n[s];
        t.len = len[s];
        const double stop = sh.part_at(at, end, share, wg, base, t);
        if (stop <= at || stop > end) return fail("no progress", it);
        at = stop;
        if (t.part < 0 || t.part >= t.parts) continue;  // a sliver, which a neighbour takes
        unit[{s, t.kvh, t.tile}].push_back(t);
        if (t.owner < 0 || t.owner + t.parts > n_wg) return fail("part number", it);
        if (t.parts > 1) {
          const int sl = part_slot(t.owner, t.part);
          if (sl < 0 || sl >= 2 * slots || !slot.insert(sl).second) return fail("two partials in a slot", it);
          if (t.part == 0 && !owner.insert(t.owner).second) return fail("two units count at one owner", it);
        }
      }
    }
    if ((int64_t)unit.size() != units) return fail("a unit that nobody computes", it);
    for (auto &[key, parts] : unit) {
      int k0, k1, at;
      rows_keys(parts[0], k0, k1);
      at = k0;
      if ((int)parts.size() != parts[0].parts) return fail("number of parts", it);
      for (size_t i = 0; i < parts.size(); ++i) {
        if (parts[i].part != (int)i || parts[i].t0 != at || parts[i].t1 < at) return fail("keys of a part", it);
        at = parts[i].t1;
      }
      if (at != k1) return fail("keys left out", it);
    }
    ++checked;
  }
  // the division that finds a key's page
  for (int d = 1; d < 5000; d = d < 70 ? d + 1 : d * 2 + 1) {
    const FastDiv f = fast_div(d);
    for (int i = 0; i < 2000; ++i) {
      const int x = i < 300 ? i : i < 600 ? INT32_MAX - (i - 300) : (int)(rng() >> 1);
      if ((int)(((uint64_t)(uint32_t)x * f.mul) >> f.shift) != x / d) return fail("division", d);
    }
  }
  std::printf("ok %d\n", checked);
  return 0;
}
