// The integer logic of paged calls with trees (csrc/burst_paged.h, the same code as on the device) on the host: bits and depths of masks against
// loops over single bits, and over random batches that every key that a token sees lies in its block's range, and every unit of every item in
// exactly one run.  Built with the address and undefined-behaviour sanitizers by tests/test_paged_tree_work.py.
#include <cstdio>
#include <map>
#include <tuple>
#include <vector>
#include "burst_paged.h"
using namespace burst;

static int bad = 0, g_case = 0;
#define CHECK(x) do { if (!(x)) { if (bad++ < 10) std::printf("line %d: %s (case %d)\n", __LINE__, #x, g_case); } } while (0)
static std::vector<int> g_starts, g_lengths;
struct HostRead {
  static int at(const int* p, int i) { return (p == g_starts.data() ? g_starts : g_lengths).at((size_t)i); }   // (throws outside)
};
typedef PagedCursor<HostRead, true> Cursor;

static unsigned long long g_seed = 1;
static unsigned long long next() { return (g_seed = g_seed * 6364136223846793005ULL + 1442695040888963407ULL) >> 16; }
static int rnd(int n) { return n > 0 ? (int)((next() >> 15) % (unsigned)n) : 0; }
static unsigned long long word() { return next() << 40 ^ next() << 20 ^ next(); }
static int wild() { const int w[] = {-1, 0, 1, 0x7fffffff, -0x7fffffff - 1, 1 << 30, -5, 64}; return rnd(2) ? w[rnd(8)] : rnd(3000) - 100; }

static bool bit(const std::vector<unsigned long long>& m, long long j) { return j >= 0 && j < 64 * (long long)m.size() && (m[j >> 6] >> (j & 63) & 1) != 0; }

static void masks() {
  const int words = 1 + rnd(4), n = rnd(64 * words + 1), off = rnd(500) - 200, lo = rnd(200) - 100, hi = rnd(200) - 100;
  std::vector<unsigned long long> m(words);
  for (auto& w : m) w = rnd(3) ? word() : rnd(2) ? 0 : ~0ull;
  const unsigned long long got = tree_bits(m.data(), words, off), range = bit_range(lo, hi);
  int depth = -1;
  for (int i = 0; i < n; i++) depth += bit(m, i);
  CHECK(tree_depth(m.data(), words, n) == depth);
  for (int i = 0; i < 64; i++) {
    CHECK((got >> i & 1) == (unsigned long long)bit(m, off + (long long)i));
    CHECK((range >> i & 1) == (unsigned long long)(i >= lo && i <= hi));
  }
  CHECK(bit_range(-0x7fffffff, 0x7fffffff) == ~0ull && bit_range(64, 0x7fffffff) == 0 && bit_range(-0x7fffffff, -1) == 0);
}

static void batch(bool anything) {
  const int S = 1 + rnd(6), page_shift = 4 + rnd(4), width = rnd(40), cap = width << page_shift, group = 1 + rnd(20), item_rows = rnd(2) ? 16 : 128;
  g_starts.assign(S + 1, 0);
  g_lengths.assign(S, 0);
  for (int s = 0; s < S; s++) {
    g_lengths[s] = anything ? wild() : rnd(cap + 40);
    g_starts[s + 1] = g_starts[s] + (rnd(4) ? rnd(70) : rnd(400));
  }
  const int rows = g_starts[S] + rnd(3);
  if (anything)
    for (int s = 1; s <= S; s++) g_starts[s] = g_starts[s - 1] + (rnd(3) ? rnd(90) : (g_starts[s - 1] < 1 << 20 ? rnd(1 << 20) : 0));
  const int words = 1 + rnd(4);
  PagedWork w = {};
  w.starts = g_starts.data(); w.lengths = g_lengths.data(); w.sequences = S; w.rows = rows; w.cap = cap;
  w.tokens = group <= item_rows ? item_rows / group : 1;
  w.parts = 1 + rnd(3);
  w.causal = 1;
  w.window = rnd(2) ? 0 : rnd(2) ? 1 + rnd(100) : 1 << 30;
  w.item_cost = rnd(3);
  w.unit_shift = 5 + rnd(2);
  w.tree = 64 * words;
  // what tokens see lies in their blocks' ranges
  for (int s = 0; s < S; s++) {
    const PagedSeq q = Cursor::load(w, s);
    if (q.n <= 0 || !w.is_tree(q)) continue;
    for (int t = 0; t < q.n; t++) {
      std::vector<unsigned long long> m(words);
      for (auto& x : m) x = rnd(2) ? word() : 0;
      int k0, k1;
      w.keys<true>(q, t / w.tokens, k0, k1);
      CHECK(0 <= k0 && k0 <= k1 && k1 <= q.len);
      const int depth = tree_depth(m.data(), words, q.n), base = q.at < q.len ? q.at : q.len;
      const long long first = w.window > 0 ? (long long)q.at + depth - w.window + 1 : 0;
      if (first < base && base > 0) CHECK(k0 <= (first > 0 ? first : 0) && k1 >= base);
      for (int j = 0; j < q.n; j++)
        if (bit(m, j) && q.at + j >= 0 && q.at + j < q.len) CHECK(k0 <= q.at + j && q.at + j < k1);
    }
  }
  // every unit of every item once
  PagedTotals all = {0, 0, 0, 0};
  std::vector<PagedTotals> each;
  for (int s = 0; s < S; s++) {
    const PagedSeq q = Cursor::load(w, s);
    PagedTotals t = w.totals<true>(q, w.blocks(q), 0, 1);
    t.pair = w.pair<true>(q, w.blocks(q), t.most);
    for (int b = 0; b + 1 < w.blocks(q); b++) CHECK(w.cost<true>(q, w.block_at(b, w.blocks(q))) + w.cost<true>(q, w.block_at(b + 1, w.blocks(q))) <= t.pair);
    all.units += t.units * w.parts; all.items += t.items * w.parts;
    all.most = t.most > all.most ? t.most : all.most;
    all.pair = t.pair > all.pair ? t.pair : all.pair;
    each.push_back(t);
  }
  const int runs = 1 + rnd(40);
  const PagedDeal deal = paged_deal(all, runs, rnd(10), rnd(2) * rnd(9));
  const int total = deal.by_items ? all.items : all.units;
  std::map<std::tuple<int, int, int>, std::vector<int>> covered;
  for (long long begin = 0; begin < total; begin += deal.each) {
    auto one = [&](int s) { return deal.by_items ? each[s].items : each[s].units; };
    int before = 0, s = 0;
    while (begin >= before + one(s) * w.parts) before += one(s++) * w.parts;
    Cursor cur;
    if (!cur.place(w, s, Cursor::load(w, s), one(s), (int)begin - before, deal, deal.each < total - begin ? deal.each : (int)(total - begin),
                   [](int&, int) { return 0; })) continue;
    do {
      const PagedSegment& g = cur.g;
      std::vector<int>& c = covered[std::make_tuple(cur.s, g.part, g.block)];
      c.resize(g.hi - g.lo);
      CHECK(g.lo <= g.from && g.from < g.to && g.to <= g.hi);
      for (int u = g.from; u < g.to; u++) c[u - g.lo]++;
      int first, end, k0, k1;
      segment_tiles<true>(w, g, w.unit_shift, first, end);
      w.keys<true>(g.q, g.block, k0, k1);
      CHECK(first < end && (k1 <= k0 || end <= ((k1 - 1) >> w.unit_shift) + 1 || end == first + 1));
    } while (cur.next(w));
  }
  int items = 0;
  for (int s = 0; s < S; s++) items += w.blocks(Cursor::load(w, s)) * w.parts;
  CHECK((int)covered.size() == items);
  for (const auto& c : covered)
    for (const int n : c.second) CHECK(n == 1);
}

int main() {
  for (g_case = 0; g_case < 20000; g_case++) masks();
  for (g_case = 0; g_case < 600; g_case++) batch(g_case % 4 == 3);
  std::printf("tree checks failed: %d\n", bad);
  return bad != 0;
}
