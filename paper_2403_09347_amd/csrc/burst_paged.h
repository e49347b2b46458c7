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

// A sequence of the batch: rows [first, first + n) of the packed tokens, keys [0, len).  Token t has position len - n + t.
struct PagedSeq { int first, n, len; };
BURST_HD PagedSeq paged_seq(int start, int end, int length, int rows, int cap) {
  PagedSeq q;
  q.first = start < 0 ? 0 : start < rows ? start : rows;
  const int e = end < q.first ? q.first : end < rows ? end : rows;
  q.n = e - q.first;
  q.len = length < 0 ? 0 : length < cap ? length : cap;
  return q;
}

// An item: a block of `tokens` tokens of a sequence with the query heads of one part of a key/value head's group.  Groups of more
// heads than a block has rows are cut into parts of so many heads (and then a block has one token).
// A unit: kUnit keys of an item.  An item has the units that some row of it sees, and at least one, so that rows that
// see nothing are written too.
constexpr int kUnitShift = 6, kUnit = 1 << kUnitShift;
struct PagedWork {
  const int* starts; const int* lengths;
  int sequences, rows, cap;          // rows of the packed tensors; keys that a row of the table has pages for
  int tokens, parts;                 // of an item; parts of all key/value heads
  int least, most;                   // sequences of fewer or more new tokens are another launch's
  int causal;
  long long window;
  BURST_HD bool mine(const PagedSeq& q) const { return q.n > 0 && q.n >= least && q.n <= most; }
  BURST_HD int blocks(const PagedSeq& q) const { return (q.n + tokens - 1) / tokens; }
  // keys [lo, hi) that the rows of a block see between them
  BURST_HD void keys(const PagedSeq& q, int block, int& lo, int& hi) const {
    const int t0 = block * tokens, t1 = (q.n - t0 < tokens ? q.n : t0 + tokens) - 1;
    lo = 0; hi = q.len;
    if (causal && q.len - q.n + t1 + 1 < hi) hi = q.len - q.n + t1 + 1;
    if (window > 0) {
      const long long first = (long long)(q.len - q.n + t0) - window + 1;
      if (first > 0) lo = first < hi ? (int)first : hi;
    }
    if (hi < lo) hi = lo;
  }
  BURST_HD void units(const PagedSeq& q, int block, int& lo, int& hi) const {
    int k0, k1;
    keys(q, block, k0, k1);
    lo = k0 >> kUnitShift;
    hi = k1 > k0 ? ((k1 - 1) >> kUnitShift) + 1 : lo + 1;
  }
  // units of all blocks of a sequence, for one part of a head
  BURST_HD long long cost(const PagedSeq& q) const {
    if (!mine(q)) return 0;
    long long sum = 0;
    const int n = blocks(q);
    for (int b = 0; b < n; b++) {
      int lo, hi;
      units(q, b, lo, hi);
      sum += hi - lo;
    }
    return sum;
  }
};

// A run: the units [at, at + left) of the sequence that the parts, blocks and units of all sequences make (sequence, part, block, unit,
// the last one fastest).  Runs of a launch have the same length, the last one excepted.
BURST_HD long long run_length(long long total, int runs) {
  const long long n = (total + runs - 1) / runs;
  return n > 0 ? n : 1;
}
// A run's part of one item.
struct PagedSegment {
  PagedSeq q;
  int s, part, block;
  int lo, hi;                        // the item's units
  int from, to;                      // those of this segment
  BURST_HD bool whole() const { return from == lo && to == hi; }
};
// Read: element i of one of the caller's arrays (device: by a scalar load).
template <typename Read>
struct PagedCursor {
  PagedSegment g;
  long long left;
  int skip;                          // units of the item before the segment
  BURST_HD PagedSeq load(const PagedWork& w, int s) const {
    return paged_seq(Read::at(w.starts, s), Read::at(w.starts, s + 1), Read::at(w.lengths, s), w.rows, w.cap);
  }
  // the place `rem` units into sequence s (rem < its units)
  BURST_HD void place(const PagedWork& w, int s, long long rem, long long run) {
    g.s = s;
    g.q = load(w, s);
    const long long one = w.cost(g.q);
    g.part = (int)(rem / one);
    rem -= g.part * one;
    g.block = 0;
    for (;;) {
      w.units(g.q, g.block, g.lo, g.hi);
      if (rem < g.hi - g.lo) break;
      rem -= g.hi - g.lo;
      g.block++;
    }
    skip = (int)rem;
    left = run;
    cut();
  }
  BURST_HD void cut() {
    g.from = g.lo + skip;
    g.to = left < g.hi - g.from ? g.from + (int)left : g.hi;
    left -= g.to - g.from;
  }
  // the run's next segment; false: there is none
  BURST_HD bool next(const PagedWork& w) {
    if (left <= 0) return false;
    if (++g.block >= w.blocks(g.q)) {
      g.block = 0;
      if (++g.part >= w.parts) {
        g.part = 0;
        do {
          if (++g.s >= w.sequences) return false;
          g.q = load(w, g.s);
        } while (!w.mine(g.q));
      }
    }
    w.units(g.q, g.block, g.lo, g.hi);
    skip = 0;
    cut();
    return true;
  }
};

// The tiles of 1 << shift keys (shift <= kUnitShift) of a segment that hold a key which some row of its item sees: [first, end).  All of them
// begin before the end of the sequence, and so within the pages of its table row.
BURST_HD void segment_tiles(const PagedWork& w, const PagedSegment& g, int shift, int& first, int& end) {
  int k0, k1;
  w.keys(g.q, g.block, k0, k1);
  const int u = kUnitShift - shift, e = (k1 + (1 << shift) - 1) >> shift;
  first = k0 >> shift > g.from << u ? k0 >> shift : g.from << u;
  end = e < g.to << u ? e : g.to << u;
}
// Where a run leaves the partial results of an item that is not all its own: the first part of an item is its run's last segment, every
// other part its run's first one.
BURST_HD int partial_slot(const PagedSegment& g, int run) { return 2 * run + (g.from == g.lo ? 1 : 0); }
// The number of parts (from run - 1 on) of the item that a run's first segment `g` belongs to, if this run is the first one that starts inside
// it; else 0.
BURST_HD int parts_to_join(const PagedSegment& g, long long run_units) {
  const int before = g.from - g.lo;
  if (before == 0 || before > run_units) return 0;
  return 2 + (int)((g.hi - g.from - 1) / run_units);
}

// An entry of the page table, or -1 if it is no page.
BURST_HD int checked_page(int page, int pages) { return page >= 0 && page < pages ? page : -1; }

}  // namespace burst
