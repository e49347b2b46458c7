// The integer logic of a paged call (csrc/burst_paged.h, the same code as on the device) on the host, over random batches: ordinary
// ones, and arrays that hold anything.  Checks that every unit of every item belongs to exactly one run, that no key
// outside the table or the pages is named, and that the parts of a cut item are joined once, from the slots that they were written
// to.  Built with the address and undefined-behaviour sanitizers by tests/test_paged_work.py.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <set>
#include <tuple>
#include <vector>
#include "burst_paged.h"
using namespace burst;

static int bad = 0;
#define CHECK(x) do { if (!(x)) { if (bad++ < 10) std::printf("line %d: %s (case %d)\n", __LINE__, #x, g_case); } } while (0)
static int g_case = 0;
static long long by_items = 0, by_units = 0, ordered = 0, disordered = 0;

static std::vector<int> g_starts, g_lengths;
struct HostRead {
  static int at(const int* p, int i) {
    const std::vector<int>& v = p == g_starts.data() ? g_starts : g_lengths;
    return v.at((size_t)i);                        // (throws outside)
  }
};
typedef PagedCursor<HostRead> Cursor;

static unsigned long long g_seed = 1;
static int rnd(int n) {
  g_seed = g_seed * 6364136223846793005ULL + 1442695040888963407ULL;
  return n > 0 ? (int)((g_seed >> 33) % (unsigned)n) : 0;
}
static int wild() { const int w[] = {-1, 0, 1, 0x7fffffff, -0x7fffffff - 1, 1 << 30, -5, 64}; return rnd(2) ? w[rnd(8)] : rnd(3000) - 100; }

// As the kernels' start_run does it, whose lanes share the blocks of a sequence, or go past them 64 at a time.
static bool locate(const PagedWork& w, int runs, int slack, int few, int run, Cursor& cur, PagedDeal& deal, long long& bound) {
  PagedTotals all = {0, 0, 0, 0};
  std::vector<PagedTotals> each;
  for (int s = 0; s < w.sequences; s++) {
    const PagedSeq q = Cursor::load(w, s);
    PagedTotals t = w.totals(q, w.blocks(q), 0, 1), shared = {0, 0, 0, 0};
    for (int lane = 0; lane < 64; lane++) {
      const PagedTotals x = w.totals(q, w.blocks(q), lane, 64);
      shared.items = x.items; shared.units += x.units;
      if (x.most > shared.most) shared.most = x.most;
    }
    CHECK(t.units == shared.units && t.items == shared.items && t.most == shared.most);
    t.pair = w.pair(q, w.blocks(q), t.most);
    each.push_back(t);
    if (!PagedWork::in_order(g_starts[s], g_starts[s + 1])) return false;
    all.units += each[s].units * w.parts;
    all.items += each[s].items * w.parts;
    if (each[s].most > all.most) all.most = each[s].most;
    if (each[s].pair > all.pair) all.pair = each[s].pair;
  }
  deal = paged_deal(all, runs, slack, few);
  if (all.units <= (long long)few * runs) runs = (runs + 1) / 2;
  const long long per = deal.each, even = (all.units + runs - 1) / runs;
  bound = (per >> 1) * all.pair + (per & 1) * all.most;
  if (deal.by_items) CHECK(bound <= even + even / 16 + slack);
  const int total = deal.by_items ? all.items : all.units;
  const long long begin = (long long)deal.each * run;
  if (begin >= total) return false;
  auto one = [&](int s) { return deal.by_items ? each[s].items : each[s].units; };
  int before = 0, s = 0;
  while (begin >= before + one(s) * w.parts) before += one(s++) * w.parts;
  return cur.place(w, s, Cursor::load(w, s), one(s), (int)begin - before, deal, deal.each < total - begin ? deal.each : total - (int)begin,
                   [&](int& rem, int n) {
                     int place = 0;
                     const PagedSeq q = Cursor::load(w, s);
                     for (; n - place > 8; place += 64) {
                       int sum = 0;
                       for (int i = 0; i < 64 && place + i < n; i++) {
                         const int c = w.cost(q, w.block_at(place + i, n));
                         if (rem < sum + c) { rem -= sum; return place + i; }
                         sum += c;
                       }
                       rem -= sum;
                     }
                     return place;
                   });
}

static void batch(bool anything) {
  const int S = 1 + rnd(9), page_shift = 4 + rnd(4), width = rnd(40), cap = width << page_shift, pages = 1 + rnd(50);
  const int group = 1 + rnd(20), item_rows = rnd(2) ? 16 : 128, heads = 1 + rnd(3);
  g_starts.assign(S + 1, 0);
  g_lengths.assign(S, 0);
  for (int s = 0; s < S; s++) {
    g_lengths[s] = anything ? wild() : rnd(4) ? rnd(cap + 1) : rnd(2);
    g_starts[s + 1] = g_starts[s] + (rnd(4) ? rnd(4) : rnd(rnd(20) ? 200 : 3000));
  }
  const int rows = g_starts[S] + rnd(3);
  bool order = true;
  if (anything) {
    for (int& x : g_starts) x = rnd(2) ? x : wild();
    if (rnd(4)) std::sort(g_starts.begin(), g_starts.end());
    for (int s = 0; s < S; s++) order = order && g_starts[s] <= g_starts[s + 1];
    (order ? ordered : disordered)++;
  }
  std::vector<int> table((size_t)S * width);
  for (int& x : table) x = anything || rnd(20) == 0 ? wild() : rnd(pages);
  PagedWork w = {};
  w.starts = g_starts.data(); w.lengths = g_lengths.data();
  w.sequences = S; w.rows = rows; w.cap = cap;
  w.tokens = group <= item_rows ? item_rows / group : 1;
  const int each_head = (group + item_rows - 1) / item_rows;
  w.parts = heads * each_head;
  w.causal = rnd(3) != 0;
  w.window = rnd(3) ? 0 : rnd(2) ? 1 + rnd(100) : 1 << 30;
  w.item_cost = rnd(4);
  w.unit_shift = rnd(4) ? 5 + rnd(2) : 7 + rnd(3);
  const int runs = 1 + rnd(40), slack = rnd(3) ? rnd(10) : rnd(2) * 100000, few = rnd(2) * rnd(9);

  typedef std::tuple<int, int, int> Item;          // sequence, part, block
  std::map<Item, std::vector<int>> covered;
  std::map<Item, std::vector<int>> slots;          // of the parts, in the order of their keys
  std::set<int> used;
  std::map<Item, int> joins;
  for (int run = 0; run < runs; run++) {
    Cursor cur;
    PagedDeal deal;
    long long bound = 0;
    if (!locate(w, runs, slack, few, run, cur, deal, bound)) continue;
    CHECK(order);
    bool first = true;
    long long length = 0;                          // no run of whole items is longer than the deal's bound on it
    do {
      const PagedSegment& g = cur.g;
      const Item item(cur.s, g.part, g.block);
      CHECK(cur.s >= 0 && cur.s < S && g.part >= 0 && g.part < w.parts && g.block >= 0 && g.block < w.blocks(g.q));
      CHECK(g.lo <= g.from && g.from < g.to && g.to <= g.hi);
      CHECK(g.q.first >= 0 && g.q.n > 0 && g.q.first + g.q.n <= rows && g.q.len >= 0 && g.q.len <= cap);
      std::vector<int>& c = covered[item];
      c.resize(g.hi - g.lo);
      for (int u = g.from; u < g.to; u++) c[u - g.lo]++;
      by_items += deal.by_items;
      by_units += !deal.by_items;
      if (!g.whole()) {
        CHECK(!deal.by_items);
        CHECK(used.insert(partial_slot(g, run)).second);
        CHECK(partial_slot(g, run) < 2 * runs);
        slots[item].push_back(partial_slot(g, run));
      }
      int k0, k1;
      w.keys(g.q, g.block, k0, k1);
      for (int shift = 4; shift <= kTileShift && shift <= w.unit_shift; shift++) {   // what the kernels fetch: 16 keys at a time, in one page
        int t, end;
        segment_tiles(w, g, shift, t, end);
        CHECK(t < end);
        const int lo = g.from << w.unit_shift, hi = g.to << w.unit_shift;
        for (int key = lo > k0 ? lo : k0; key < (hi < k1 ? hi : k1); key++) CHECK(key >= t << shift && key < end << shift);
        for (; t < end; t++)
          for (int key = t << shift; key < (t + 1) << shift; key += 16) {
            const int entry = table_entry(key, g.q.len, page_shift);
            CHECK(entry >= -1 && entry < width);
            if (entry < 0) continue;
            const int page = checked_page(table.at((size_t)cur.s * width + entry), pages);
            CHECK(page >= -1 && page < pages);
            CHECK((key & ((1 << page_shift) - 1)) + 16 <= 1 << page_shift);
          }
      }
      if (first && run > 0) {
        const int n = parts_to_join(g, deal.each);
        if (n > 0) {
          joins[item]++;
          for (int i = 0; i < n; i++) slots[Item(-1 - cur.s, g.part, g.block)].push_back(2 * (run - 1 + i) + (i == 0 ? 1 : 0));
        }
      }
      first = false;
      length += g.hi - g.lo + w.item_cost;
    } while (cur.next(w));
    CHECK(cur.left <= w.item_cost);
    if (deal.by_items) CHECK(length <= bound);
  }
  if (!order) return;                              // (nothing is done)
  for (int s = 0; s < S; s++) {
    const PagedSeq q = Cursor::load(w, s);
    if (q.n <= 0) continue;
    for (int part = 0; part < w.parts; part++)
      for (int b = 0; b < w.blocks(q); b++) {
        int lo, hi;
        w.units(q, b, lo, hi);
        const std::vector<int>& c = covered[Item(s, part, b)];
        CHECK((int)c.size() == hi - lo);
        for (int x : c) CHECK(x == 1);
        const std::vector<int>&parts = slots[Item(s, part, b)], &joined = slots[Item(-1 - s, part, b)];
        CHECK(joins[Item(s, part, b)] == (parts.empty() ? 0 : 1));
        CHECK(parts == joined);
      }
  }
  size_t items = 0;
  for (auto& x : covered) items += !x.second.empty();
  size_t want = 0;
  for (int s = 0; s < S; s++) {
    const PagedSeq q = Cursor::load(w, s);
    if (q.n > 0) want += (size_t)w.parts * w.blocks(q);
  }
  CHECK(items == want);
}

// every run with work has one workgroup, run 0 the first one, and no XCD has more than its share
static void placement() {
  const int runs = rnd(3) ? 8 * (1 + rnd(128)) : 1 + rnd(8), active = rnd(runs + 1);
  std::vector<int> seen(runs), xcd(8);
  for (int bid = 0; bid < runs; bid++) {
    const int run = run_of(bid, runs, active);
    CHECK(run >= -1 && run < active);
    if (run < 0) continue;
    seen[run]++;
    xcd[bid % 8]++;
    CHECK((run == 0) == (bid == 0));
  }
  for (int run = 0; run < active; run++) CHECK(seen[run] == 1);
  if (runs % 8 == 0)
    for (int n : xcd) CHECK(n <= (active + 7) / 8);
}

int main() {
  for (g_case = 0; g_case < 6000; g_case++) { batch(g_case % 3 == 2); placement(); }
  if (by_items < 1000 || by_units < 1000 || ordered < 500 || disordered < 100) bad++;   // all of them have been seen
  std::printf("work checks failed: %d\n", bad);
  return bad != 0;
}
