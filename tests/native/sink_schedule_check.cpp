// Attention with sinks: how its work is dealt out, walked on the host.  Over ragged batches
// every key tile that holds a key that some row of a unit sees (its window's, the sinks'
// before it) is computed exactly once, those between are not, and a unit's parts follow each
// other.  Prints the number of batches checked.
#include <climits>
#include <cstdio>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "../../paper_2609_30884_amd/csrc/paged_attn.hip"

using namespace crf;

static std::mt19937 rng(5);
static int upto(int n) { return (int)(rng() % (unsigned)(n + 1)); }

int main() {
  int checked = 0, between = 0, split = 0;
  for (int it = 0; it < 3000; ++it) {
    const int nkv = 1 + upto(5), G = 1 + upto(8), bm = it % 2 ? 32 : 128;
    const int window = it % 7 ? 1 + upto(1 + upto(3000)) : INT_MAX - upto(5);
    const int sinks = it % 5 ? upto(upto(2) ? 300 : 6000) : it % 3 ? INT_MAX - upto(5) : 1;
    Shape sh{G, nkv, window, bm, bm == 32 ? 128 : 64, 256, 0, fast_div(G), 1.f, it % 2 == 0, sinks};
    const int slots = 8 * (1 + upto(63)), seqs = 1 + upto(12);
    std::vector<int> n(seqs), len(seqs);
    double total = 0;
    int units = 0, longest = 0;
    for (int s = 0; s < seqs; ++s) {
      n[s] = upto(5) ? 1 + upto(bm == 32 ? 32 / G : 1 + upto(700)) : 0;
      len[s] = n[s] + upto(upto(2) ? 600 : 20000);
      if (n[s] == 0) continue;
      total += sh.seq_work(n[s], len[s]);
      units += sh.work(n[s], len[s]).tiles * nkv;
      longest = std::max(longest, len[s]);
    }
    if (units == 0) continue;
    std::map<std::tuple<int, int, int>, std::multiset<int>> got;  // key tiles of each unit
    auto take = [&](int s, const Task &t) {
      for (int x = t.t0; x < t.t1; ++x) {
        const bool first = x < t.k0;  // as the kernels take them
        got[{s, t.kvh, t.tile}].insert(first ? x - t.gap : x);
      }
    };
    if (it % 4 == 0) {  // whole units
      for (int s = 0; s < seqs; ++s)
        for (int i = 0; n[s] && i < sh.work(n[s], len[s]).tiles * nkv; ++i) {
          Task t{};
          t.n = n[s], t.len = len[s];
          sh.whole(i, t);
          take(s, t);
        }
    } else {
      const Shape::Plan plan = sh.plan(total, units, longest, slots);
      const Deal d = deal(total, plan.want, seqs * nkv, 0, slots);
      std::map<std::tuple<int, int, int>, int> last;
      for (int wg = 0; wg < d.n_wg; ++wg) {
        double at = wg * d.share;
        const double end = std::min(at + d.share, total);
        while (at < end) {
          double base = 0;
          int s = 0;
          for (;; ++s) {
            const double w = n[s] > 0 ? sh.seq_work(n[s], len[s]) : 0;
            if (at < base + w) break;
            base += w;
          }
          Task t{};
          t.seq = s, t.n = n[s], t.len = len[s];
          at = sh.part_at(at, end, d.share, wg, base, t);
          if (t.part < 0 || t.part >= t.parts) continue;
          split += t.parts > 1;
          auto &l = last[{s, t.kvh, t.tile}];
          if (t.part && l != t.t0) return std::printf("batch %d: a part does not begin where the one before ends\n", it), 1;
          l = t.t1;
          take(s, t);
        }
      }
    }
    if ((int)got.size() != units) return std::printf("batch %d: %zu units of %d\n", it, got.size(), units), 1;
    for (auto &[unit, tiles] : got) {
      const int s = std::get<0>(unit), tile = std::get<2>(unit);
      const int64_t r0 = (int64_t)tile * bm, r1 = std::min<int64_t>(r0 + bm, (int64_t)n[s] * G) - 1;
      const int64_t p0 = len[s] - n[s] + r0 / G, p1 = len[s] - n[s] + r1 / G;
      std::multiset<int> want;
      const int64_t lo = std::max<int64_t>(0, p0 - window + 1);
      for (int64_t x = 0; x * sh.bkv <= p1; ++x) {
        const bool seen = (x + 1) * sh.bkv > lo || x * sh.bkv < sinks;
        if (seen) want.insert((int)x);
        between += !seen;
      }
      if (tiles != want) return std::printf("batch %d: key tiles of sequence %d, tile %d\n", it, s, tile), 1;
    }
    ++checked;
  }
  if (between == 0 || split == 0) return std::printf("nothing between, or nothing split\n"), 1;
  std::printf("ok %d\n", checked);
  return 0;
}
