// Host-side check of how attention over the 8-bit cache is cut into shares and merged (kvq_shares.h), with the kernels' own arithmetic.
//   * merge: for units of 1 .. 512 parts that arrive in any order, every maximum and sum that a merge reads was written, on that level, by a workgroup that has
//     published it; every part is merged exactly once; a counter serves one group; the last merge covers the unit.
//   * shares: the parts of every unit of random batches follow each other without gap or overlap, one for each workgroup from the first to the last that the
//     kernel computes.
// Prints "ok <cases>" or the first violation.  With arguments (wide Hkv G n_max max_pages, then context and rows of every sequence) it prints the parts
// and rows of every unit that is cut, as "parts:rows".
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <utility>
#include <vector>
#include "../../paper_2605_08862_amd/csrc/kvq_shares.h"

constexpr int kLevels = 5, kMost = 2 * kCUs;              // as the workspace has them
static long cases = 0;
#define FAIL(...) do { std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } while (0)

// ---- merge
struct Word { int lo = -1, hi = -1, owner = -1; bool published = false; };       // parts [lo, hi) are in it
static void check_merge(int n, int log_f, std::mt19937& rng) {
  std::vector<std::vector<Word>> ml(kLevels, std::vector<Word>(n));
  std::vector<std::vector<int>> counter(kLevels, std::vector<int>(n, 0)), size(kLevels, std::vector<int>(n, 0));
  std::vector<int> order(n);
  for (int i = 0; i < n; ++i) order[i] = i;
  std::shuffle(order.begin(), order.end(), rng);
  int done = 0;
  for (int w : order) {
    ml[0][w] = Word{w, w + 1, w, false};
    merge_levels(w, n, log_f,
                 [&](int level, int i0, int count) {
                   if (level >= kLevels) FAIL("n=%d: level %d", n, level);
                   if (size[level][i0] && size[level][i0] != count) FAIL("n=%d: two groups at level %d, part %d", n, level, i0);
                   size[level][i0] = count;
                   for (auto& l : ml) for (auto& x : l) if (x.owner == w) x.published = true;
                   return ++counter[level][i0] == count;
                 },
                 [&](int level, int i0, int stride, int count, int lone, bool last) {
                   int lo = i0, hi = i0;
                   for (int u = 0; u < count; ++u) {
                     const int i = i0 + u * stride, at = u == count - 1 ? lone : level;
                     if (i >= n || at < 0 || at > level) FAIL("n=%d F=%d: part %d on level %d", n, 1 << log_f, i, at);
                     const Word& x = ml[at][i];
                     if (x.lo < 0 || !x.published) FAIL("n=%d F=%d: part %d is read on level %d, where nobody has published it", n, 1 << log_f, i, at);
                     if (x.lo != hi) FAIL("n=%d F=%d: part %d on level %d holds %d .. %d, not %d ..", n, 1 << log_f, i, at, x.lo, x.hi, hi);
                     hi = x.hi;
                   }
                   if (hi - lo != least_of(n - lo, stride << log_f)) FAIL("n=%d F=%d: a merge of %d .. %d", n, 1 << log_f, lo, hi);
                   if (last) { if (lo != 0 || hi != n) FAIL("n=%d F=%d: the last merge covers %d .. %d", n, 1 << log_f, lo, hi); ++done; }
                   else if (level + 1 >= kLevels) FAIL("n=%d: no level behind %d", n, level);
                   else ml[level + 1][i0] = Word{lo, hi, w, false};
                 });
  }
  if (n > 1 && done != 1) FAIL("n=%d F=%d: merged %d times", n, 1 << log_f, done);
  ++cases;
}

// ---- shares
struct Seq { int c, n; };
struct Cut { int parts, rows; };
template <bool WIDE>
static std::vector<Cut> check_shares(const std::vector<Seq>& seqs, int Hkv, int g, int n_max, int max_pages) {
  const Group G = make_group(g);
  std::vector<Unit<WIDE>> units;
  int at = 0;
  for (const Seq& s : seqs)
    for (int h = 0; s.n > 0 && h < Hkv; ++h)
      for (int qb = 0; qb * kBlock<WIDE> < s.n * g; ++qb) {
        Unit<WIDE> u{};
        u.n = s.n; u.c = s.c; u.qb = qb; u.first = at;
        fill_unit<WIDE>(u, G);
        const int seen = s.c + least_of(s.n, ((qb + 1) * kBlock<WIDE> - 1) / g + 1);      // tokens that its last row sees
        if (seen > kStep * u.steps || seen <= kStep * (u.steps - 1)) FAIL("a unit of %d steps for %d tokens", u.steps, seen);
        at = u.end();
        units.push_back(u);
      }
  std::vector<Cut> cuts;
  if (!at) return cuts;
  const Shares sh = make_shares(at, share_grid(WIDE, (int)seqs.size(), Hkv, (long long)n_max * g, max_pages));
  std::vector<std::vector<std::pair<int, std::pair<int, int>>>> parts(units.size());
  size_t u0 = 0;
  for (int w = 0; w < sh.W; ++w) {
    const int p0 = sh.bound(w), p1 = sh.bound(w + 1);
    if (p0 >= p1) FAIL("an empty share");
    while (units[u0].end() <= p0) ++u0;
    int s_lo = units[u0].cut(p0), from = 0, on = 0;
    for (size_t k = u0;; ++k, s_lo = 0) {
      const Unit<WIDE>& u = units[k];
      const bool last = u.end() >= p1;
      const int s_hi = last ? u.cut(p1) : u.steps;
      if (s_lo < s_hi) {
        parts[k].push_back({w, {s_lo, s_hi}});
        from += s_lo > 0;
        on += s_lo == 0 && s_hi < u.steps;
        if (!(s_lo == 0 && s_hi == u.steps)) {            // as part_of does
          const int f = s_lo == 0 ? w : u.first_share(sh), l = s_hi == u.steps ? w : u.last_share(sh);
          if (f > w || l < w || f == l) FAIL("share %d is not of %d .. %d", w, f, l);
        }
      }
      if (last) break;
    }
    if (from > 1 || on > 1) FAIL("workgroup %d has %d and %d parts of cut units", w, from, on);
  }
  for (size_t k = 0; k < units.size(); ++k) {
    const auto& p = parts[k];
    const Unit<WIDE>& u = units[k];
    if (p.empty() || p.front().second.first != 0 || p.back().second.second != u.steps) FAIL("a unit of %d steps is not covered", u.steps);
    for (size_t i = 0; i + 1 < p.size(); ++i)
      if (p[i].second.second != p[i + 1].second.first || p[i].first + 1 != p[i + 1].first) FAIL("a gap between the parts of a unit");
    if (p.size() > 1) {
      for (const auto& x : p)
        if ((x.second.first > 0 && u.first_share(sh) != p.front().first) || (x.second.second < u.steps && u.last_share(sh) != p.back().first))
          FAIL("workgroups %d .. %d have a unit, not %d .. %d", p.front().first, p.back().first, u.first_share(sh), u.last_share(sh));
      if ((int)p.size() > kMost) FAIL("%zu parts", p.size());
      cuts.push_back({(int)p.size(), least_of(u.n * g - u.qb * kBlock<WIDE>, kBlock<WIDE>)});
    }
  }
  ++cases;
  return cuts;
}

int main(int argc, char** argv) {
  if (argc > 5) {
    std::vector<Seq> seqs;
    for (int i = 6; i + 1 < argc; i += 2) seqs.push_back({std::atoi(argv[i]), std::atoi(argv[i + 1])});
    const int Hkv = std::atoi(argv[2]), g = std::atoi(argv[3]), n_max = std::atoi(argv[4]), pages = std::atoi(argv[5]);
    if (runs_wide((int)seqs.size(), Hkv, (long long)n_max * g, pages) != (std::atoi(argv[1]) != 0)) FAIL("the other kernel");
    for (const Cut& c : std::atoi(argv[1]) ? check_shares<true>(seqs, Hkv, g, n_max, pages) : check_shares<false>(seqs, Hkv, g, n_max, pages)) std::printf("%d:%d ", c.parts, c.rows);
    std::printf("\n");
    return 0;
  }
  std::mt19937 rng(1);
  for (int n = 1; n <= 512; ++n)
    for (int log_f : {2, 3})
      for (int r = 0; r < 4; ++r) check_merge(n, log_f, rng);
  auto upto = [&](double hi) { return (int)std::exp(std::uniform_real_distribution<double>(0, std::log(hi + 0.99))(rng)); };
  const int groups[] = {1, 3, 6, 7, 8, 14, 128};
  for (int r = 0; r < 3000; ++r) {
    const int B = upto(300), Hkv = upto(8), g = groups[rng() % 7], n_max = r % 3 == 0 ? 1 : r % 3 == 1 ? 17 : upto(600), most = upto(r % 5 ? 4000 : 60000);
    std::vector<Seq> seqs;
    int longest = 1;
    for (int b = 0; b < B; ++b) {
      seqs.push_back({(int)(rng() % most), rng() % 9 == 0 ? 0 : 1 + (int)(rng() % n_max)});
      longest = most_of(longest, seqs.back().c + seqs.back().n);
    }
    const int pages = (longest + kPage - 1) / kPage + (r % 2 ? 0 : (int)(rng() % 500));
    if ((long long)B * Hkv * (pages / 2 + 1) > ((long long)1 << 24) / ((long long)n_max * g / 128 + 1)) continue;      // refused (kvq_attention_counts)
    check_shares<false>(seqs, Hkv, g, n_max, pages);
    check_shares<true>(seqs, Hkv, g, n_max, pages);
  }
  std::printf("ok %ld\n", cases);
  return 0;
}
