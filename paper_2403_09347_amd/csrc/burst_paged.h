// How a call of burst_paged_fwd is dealt out: what a sequence, an item, a unit and a run are, and which page a key lies in.
// Integer logic alone, the same code on the device and (tests) on the host: every array that a caller fills on the device
// (starts, lengths, the page table) is clamped here, so that no value in it leads to an access outside the tensors.
#pragma once
#include <stdint.h>
#ifdef __HIPCC__
#define BURST_HD __host__ __device__ __forceinline__
#else
#define BURST_HD inline
#endif

namespace burst {

// A sequence of the batch: rows [first, first + n) of the packed tokens, keys [0, len).  Token t has position at + t; a sequence that has
// outgrown its row of the table has tokens at positions from `cap` on, which have no place among the keys.
constexpr int kMostTokens = 1 << 30;               // of a sequence: every position is below
struct PagedSeq { int first, n, len, at; };
BURST_HD PagedSeq paged_seq(int start, int end, int length, int rows, int cap) {
  PagedSeq q;
  q.first = start < 0 ? 0 : start < rows ? start : rows;
  const int e = end < q.first ? q.first : end < rows ? end : rows;
  q.n = e - q.first;
  const int all = length < 0 ? 0 : length < kMostTokens ? length : kMostTokens;
  q.len = all < cap ? all : cap;
  q.at = all - q.n;
  return q;
}

// An item: a block of `tokens` tokens of a sequence with the query heads of one part of a key/value head's group.  Groups of more
// heads than a block has rows are cut into parts of so many heads (and then a block has one token).
// A unit: 1 << unit_shift keys of an item (32, bf16 chunks 64, more only where a call could have 2^31 units).  An item has the units that
// some row of it sees, and at least one, so that rows that see nothing are written too.
constexpr int kTileShift = 6, kTileShiftF32 = 5;   // tiles of the chunk kernels; units are not smaller
struct PagedTotals { int units, items, most, pair; };   // units of the largest item, and of two that follow one another
struct PagedWork {
  const int* starts; const int* lengths;
  int sequences, rows, cap;          // rows of the packed tensors; keys that a row of the table has pages for
  int tokens, parts;                 // of an item; parts of all key/value heads
  int causal, window;                // window: 0 = none
  int unit_shift;
  int item_cost;                     // what the beginning of an item costs, in units: it counts in a run's length
  BURST_HD int blocks(const PagedSeq& q) const { return (q.n + tokens - 1) / tokens; }
  // keys [lo, hi) that the rows of a block see between them
  BURST_HD void keys(const PagedSeq& q, int block, int& lo, int& hi) const {
    const int t0 = block * tokens, t1 = (q.n - t0 < tokens ? q.n : t0 + tokens) - 1;
    lo = 0; hi = q.len;
    if (causal && q.at + t1 + 1 < hi) hi = q.at + t1 + 1;
    if (window > 0) {
      const int first = q.at + t0 - window + 1;   // (all of them at most 2^30)
      if (first > 0) lo = first < hi ? first : hi;
    }
    if (hi < lo) hi = lo;
  }
  // Under a causal mask blocks see more the later they are: they are taken from both ends in turn, so that every two that follow one another
  // see about the same.
  BURST_HD bool in_turn() const { return causal && window == 0; }
  BURST_HD int block_at(int place, int n) const { return !in_turn() ? place : place & 1 ? n - 1 - (place >> 1) : place >> 1; }
  BURST_HD void units(const PagedSeq& q, int block, int& lo, int& hi) const {
    int k0, k1;
    keys(q, block, k0, k1);
    lo = k0 >> unit_shift;
    hi = k1 > k0 ? ((k1 - 1) >> unit_shift) + 1 : lo + 1;
  }
  BURST_HD int cost(const PagedSeq& q, int block) const {   // units, an item's beginning among them
    int lo, hi;
    units(q, block, lo, hi);
    return hi - lo + item_cost;
  }
  // blocks from, from + step .. of the n of a sequence, for one part of a head: all blocks' number, these ones' units, and those of the largest
  BURST_HD PagedTotals totals(const PagedSeq& q, int n, int from, int step) const {
    PagedTotals t = {0, n, 0, 0};
    for (int b = from; b < n; b += step) {
      const int c = cost(q, b);
      t.units += c;
      if (c > t.most) t.most = c;
    }
    return t;
  }
  // units of two blocks that follow one another, at most; most: of the largest block.  (Blocks of a sequence that has outgrown its table all
  // see its last keys: the ends are no more than those between.)
  BURST_HD int pair(const PagedSeq& q, int n, int most) const {
    return in_turn() && n > 1 && q.at + q.n <= q.len ? cost(q, 0) + cost(q, n - 1) + (tokens >> unit_shift) + 2 : 2 * most;   // (rounded up)
  }
  // Whether a sequence ends behind its start.  Where one does not, rows could belong to several sequences, and there could be more units than
  // 32 bits hold: such a call does nothing.
  static BURST_HD bool in_order(int start, int end) { return start <= end; }
};

// How the parts, blocks and units of all sequences (sequence, part, place of the block, unit, the last one fastest) are dealt out to runs:
// `each` units a run (the items' beginnings among them: a run that ends within one leaves the item to the next), or, where that costs
// less, `each` whole items, of which nothing has to be joined.  `slack`: the units that a run may have more for that.
struct PagedDeal { int each, by_items; };
// few: where a run would have no more units than this, half as many runs have twice as many.
BURST_HD PagedDeal paged_deal(const PagedTotals& t, int runs, int slack, int few) {
  PagedDeal d;
  if (t.units <= (long long)few * runs) runs = (runs + 1) >> 1;
  const int each = (int)(((unsigned)t.units + runs - 1) / (unsigned)runs), per = (int)(((unsigned)t.items + runs - 1) / (unsigned)runs);
  d.by_items = (long long)(per >> 1) * t.pair + (per & 1) * t.most <= each + each / 16 + slack;
  d.each = d.by_items ? per : each;
  if (d.each < 1) d.each = 1;
  return d;
}
// A run's part of one item.
struct PagedSegment {
  PagedSeq q;
  int part, block;
  int lo, hi;                        // the item's units
  int from, to;                      // those of this segment
  BURST_HD bool whole() const { return from == lo && to == hi; }
};
// Where a run is.  Read: element i of one of the caller's arrays (device: by a scalar load).
template <typename Read>
struct PagedCursor {
  PagedSegment g;
  int s, at;                         // sequence; place of the block
  int left;                          // units (items) from the beginning of the item behind the segment to the end of the run
  int by_items;
  static BURST_HD PagedSeq load(const PagedWork& w, int s) {
    return paged_seq(Read::at(w.starts, s), Read::at(w.starts, s + 1), Read::at(w.lengths, s), w.rows, w.cap);
  }
  // the place `rem` units (items) into sequence s, which has more of them (`one` for each part of a head); false: the run, of `run`
  // units, ends within the beginning of an item.  Skip: (part's units, blocks) -> the place of a block that is not behind the one sought, and
  // takes the units before it away.
  template <typename Skip>
  BURST_HD bool place(const PagedWork& w, int seq, const PagedSeq& q, int one, int rem, const PagedDeal& d, int run, const Skip& skip) {
    by_items = d.by_items;
    s = seq;
    g.q = q;
    g.part = (int)((unsigned)rem / (unsigned)one);
    rem -= g.part * one;
    const int n = w.blocks(g.q);
    for (at = by_items ? rem : skip(rem, n);; at++) {
      g.block = w.block_at(at, n);
      w.units(g.q, g.block, g.lo, g.hi);
      if (by_items || rem < g.hi - g.lo + w.item_cost) break;
      rem -= g.hi - g.lo + w.item_cost;
    }
    left = by_items ? run : rem + run;
    return cut(w, by_items || rem < w.item_cost ? 0 : rem - w.item_cost);
  }
  // the segment of the item that `left` reaches into; false: not as far as its first unit
  BURST_HD bool cut(const PagedWork& w, int skip) {
    g.from = g.lo + skip;
    g.to = g.hi;
    if (!by_items && left - w.item_cost < g.hi - g.lo) g.to = g.lo + left - w.item_cost;
    left -= by_items ? 1 : g.hi - g.lo + w.item_cost;
    return g.to > g.from;
  }
  // the run's next segment; false: there is none
  BURST_HD bool next(const PagedWork& w) {
    if (left <= 0) return false;
    if (++at >= w.blocks(g.q)) {
      at = 0;
      if (++g.part >= w.parts) {
        g.part = 0;
        do {
          if (++s >= w.sequences) return false;
          g.q = load(w, s);
        } while (g.q.n <= 0);
      }
    }
    g.block = w.block_at(at, w.blocks(g.q));
    w.units(g.q, g.block, g.lo, g.hi);
    return cut(w, 0);
  }
};
// The tiles of 1 << shift keys (shift <= unit_shift) of a segment that hold a key which some row of its item sees: [first, end).  A segment
// without any has one tile all the same (its rows are written), the only one that may begin at the end of the sequence or behind it.
BURST_HD void segment_tiles(const PagedWork& w, const PagedSegment& g, int shift, int& first, int& end) {
  int k0, k1;
  w.keys(g.q, g.block, k0, k1);
  const int u = w.unit_shift - shift, e = (k1 + (1 << shift) - 1) >> shift;
  first = k0 >> shift > g.from << u ? k0 >> shift : g.from << u;
  end = e < g.to << u ? e : g.to << u;
  if (end <= first) end = first + 1;
}
// The run of a workgroup, -1: none.  Workgroup ids go to the eight XCDs in turn: the runs that have work (`active` of them) are spread over all
// XCDs, and neighbouring ones, which share keys, lie on one.  (us a call, laid out as if all had work / so: one token over 32768 keys 38.1 /
// 37.0, 8 over 200 to 1500 17.8 / 16.5, a window of 1024 at d = 64, 300 runs of 512, 37.9 / 36.3; 8 x 8 tokens fp32 46.0 / 48.4.)
BURST_HD int run_of(int bid, int runs, int active) {
  if (runs % 8 != 0) return bid < active ? bid : -1;
  const int each = (active + 7) >> 3, run = (bid & 7) * each + (bid >> 3);
  return bid >> 3 < each && run < active ? run : -1;
}
// Where a run leaves the partial results of an item that is not all its own: the first part of an item is its run's last segment, every
// other part its run's first one.
BURST_HD int partial_slot(const PagedSegment& g, int run) { return 2 * run + (g.from == g.lo ? 1 : 0); }
// The number of parts (from run - 1 on) of the item that a run's first segment `g` belongs to, if this run is the first one that starts inside
// it; else 0.
BURST_HD int parts_to_join(const PagedSegment& g, int run_units) {
  const int before = g.from - g.lo;
  if (before == 0 || before > run_units) return 0;
  return 2 + (g.hi - g.from - 1) / run_units;
}

// An entry of the page table, or -1 if it is no page.
BURST_HD int checked_page(int page, int pages) { return page >= 0 && page < pages ? page : -1; }
// The entry of a table row to read for the 16 keys from `key` on; -1: none, they are behind the sequence's end.
BURST_HD int table_entry(int key, int len, int page_shift) { return key < len ? key >> page_shift : -1; }

}  // namespace burst
