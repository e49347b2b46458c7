// The books of a paged cache: what the calls of a step read, made from the lengths of its sequences (burst_cache_plan), and the rows of
// drafted tokens that are kept, moved together (burst_cache_keep).
// Bound by latency: nearly nothing is read, but one thing tells where the next one is.  Measured: a plan of 256 single tokens, a few of which start a
// page, 7.2 us (again, with nothing to give, 5.1), of 400 sequences with trees and prompts, 20 of them ended, 87 thousand rows, 20.6 + 4 (again 10.8 + 4); where pages
// or rows do not suffice 33 and 73 + 5; the kept rows of 96 trees in 24 layers, 8 heads, 37 us.
#include "burst_paged_kernels.h"
#include "burst_plan.h"

namespace burst {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// Exclusive sum over the workgroup's threads; `all`: the sum of all.  (side: kPlanWaves integers, free before and after.)
__device__ __forceinline__ int block_scan(int x, int& all, int* side) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, scan = wave_scan(x);
  if (lane == 63) side[wave] = scan;
  __syncthreads();
  const int part = wave_scan(lane < kPlanWaves ? side[lane] : 0);
  all = __builtin_amdgcn_readlane(part, kPlanWaves - 1);
  const int before = wave == 0 ? 0 : __shfl(part, wave - 1);
  __syncthreads();
  return before + scan - x;
}
// The last i in [0, n) with at[i] <= x; at[0] = 0 and x is not negative.
__device__ __forceinline__ int last_at(const int* at, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Slot, position and mask of a row, but for trees of up to 64 tokens (see fill_tree): of theirs only the slot.  start: of all sequences, in LDS;
// before(s, n): the tokens that a sequence of n new ones had.
template <typename Before>
__device__ __forceinline__ void fill_row(const PlanArgs& a, int row, const int* start, const Before& before) {
  long long slot = -1, pos = -1;
  unsigned long long* const mask = a.parents != nullptr ? a.tree + (size_t)row * a.words : nullptr;
  int word = a.words - 1;                          // the next of the mask's words to be written
  bool small = false;
  if (a.sequences > 0 && row < start[a.sequences]) {
    const int s = last_at(start, a.sequences, row), t = row - start[s], n = start[s + 1] - start[s], base = before(s, n), place = base + t;
    const int page = checked_page(a.table[(long long)s * a.table_stride + (place >> a.page_shift)], a.pages);
    if (page >= 0) slot = (long long)page << a.page_shift | (place & ((1 << a.page_shift) - 1));
    pos = place;
    small = mask != nullptr && n <= 64;
    if (mask != nullptr && !small && n <= 64 * a.words) {   // up the branch: numbers get smaller, so words are done one after the other
      const int* const parents = a.parents + (long long)s * a.parents_stride;
      unsigned long long bits = 0;
      int depth = -1;
      for (int at = t; at >= 0; depth++) {
        for (; word > at >> 6; word--) {
          mask[word] = bits;
          bits = 0;
        }
        if (depth + 1 < a.window) bits |= 1ull << (at & 63);
        const int up = at < a.most ? parents[at] : -1;
        at = up < at ? up : -1;                    // (negative: a root; one that is not before the token is taken for none)
      }
      mask[word--] = bits;
      pos = base + depth;
    }
  }
  a.slots[row] = slot;
  if (small) return;
  if (mask != nullptr)
    for (; word >= 0; word--) mask[word] = 0;
  a.positions[row] = pos;
}
// The highest n of the bits that are set (n >= 1): those from the highest b on above which so many are.
__device__ __forceinline__ unsigned long long highest_bits(unsigned long long x, int n) {
  int b = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1)
    if (__builtin_popcountll(x >> (b + step)) >= n) b += step;
  return x >> b << b;
}
// Positions and masks of a tree of n <= 64 tokens, by a wavefront: every token takes over what the token that it has come to sees, and goes on to where that one
// has come to, twice as far each time.  (Going up branch by branch, a load each step, the rows of 400 sequences took 12.8 us; so 6.3, of which the rest is rows of chunks.)
__device__ __forceinline__ void fill_tree(const PlanArgs& a, int s, int first, int n, int base) {
  const int t = threadIdx.x & 63, up = t < n && t < a.most ? a.parents[(long long)s * a.parents_stride + t] : -1;
  int at = up >= 0 && up < t ? up : -1;
  unsigned lo = t < 32 ? 1u << t : 0u, hi = t < 32 ? 0u : 1u << (t - 32);
  while (__builtin_amdgcn_ballot_w64(at >= 0) != 0) {
    const int from = at >= 0 ? at : t;
    lo |= __shfl(lo, from);
    hi |= __shfl(hi, from);
    const int next = __shfl(at, from);
    at = at >= 0 ? next : -1;
  }
  if (t >= n) return;
  const size_t row = (size_t)first + t;
  a.positions[row] = base + __builtin_popcount(lo) + __builtin_popcount(hi) - 1;
  unsigned long long* const mask = a.tree + row * a.words;
  const unsigned long long branch = (unsigned long long)hi << 32 | lo;
  mask[0] = a.window < 64 ? highest_bits(branch, a.window) : branch;
  for (int w = 1; w < a.words; w++) mask[w] = 0;
}

// One workgroup: pages that go back, who is served, pages that are missing.
// Sequences in order are served while there are rows and pages for them; where there is enough of both, which a sum over all says, nobody is looked at
// one by one.  The entries of the table in which new tokens lie are numbered through all sequences, and the threads share them, so that a long
// prompt takes no longer than many sequences.
__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(PlanArgs a) {
  __shared__ int start[kPlanSequences + 1], base[kPlanSequences], flat[kPlanSequences + 1];   // exclusive sums of new tokens and of entries
  __shared__ unsigned passed[kPlanSequences / 32];
  __shared__ int side[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), S = a.sequences;
  int left = *a.count;                             // pages on the stack
  left = left < 0 ? 0 : left < a.pages ? left : a.pages;

  for (int i = tid; i < kPlanSequences / 32; i += kPlanThreads) passed[i] = 0;
  int mine = 0;
  for (int s = tid; s < S; s += kPlanThreads) mine |= a.added[s] < 0;
  if (__syncthreads_or(mine)) {                    // sequences that have ended: their pages go back, in order
    int n = 0;                                     // flat: which they are, start: how many pages each has
    for (int s0 = 0; s0 < S; s0 += kPlanThreads) {
      const int s = s0 + tid, ended = s < S && a.added[s] < 0;
      int all;
      const int at = block_scan(ended, all, side);
      if (ended) flat[n + at] = s;
      n += all;
    }
    __syncthreads();
    constexpr int kAtOnce = 8;
    for (int e = wave; e < n; e += kPlanWaves) {
      const int* const row = a.table + (long long)flat[e] * a.table_stride;
      int pages = 0;
      bool holds = false;                          // anything but -1
      for (int c0 = 0; c0 < a.width; c0 += 64 * kAtOnce) {
        int page[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; k++) page[k] = c0 + 64 * k + lane < a.width ? row[c0 + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < kAtOnce; k++) {
          pages += __builtin_popcountll(__builtin_amdgcn_ballot_w64(checked_page(page[k], a.pages) >= 0));
          holds = holds || page[k] != -1;
        }
      }
      if (__builtin_amdgcn_ballot_w64(holds) == 0) flat[e] = -1;   // (there is nothing to do)
      if (lane == 0) start[e] = pages;
    }
    __syncthreads();
    int back = 0;
    for (int e0 = 0; e0 < n; e0 += kPlanThreads) {
      int all;
      const int at = block_scan(e0 + tid < n ? start[e0 + tid] : 0, all, side);
      if (e0 + tid < n) start[e0 + tid] = back + at;
      back += all;
    }
    __syncthreads();
    for (int e = wave; e < n; e += kPlanWaves) {
      if (flat[e] < 0) continue;
      int* const row = a.table + (long long)flat[e] * a.table_stride;
      int to = left + start[e];
      for (int c0 = 0; c0 < a.width; c0 += 64 * kAtOnce) {
        int page[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; k++) page[k] = c0 + 64 * k + lane < a.width ? row[c0 + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < kAtOnce; k++) {
          const int c = c0 + 64 * k + lane;
          const bool is = checked_page(page[k], a.pages) >= 0;
          const unsigned long long bal = __builtin_amdgcn_ballot_w64(is);
          const int at = to + __builtin_popcountll(bal & ((1ull << lane) - 1));
          if (is && (unsigned)at < (unsigned)a.pages) a.free_pages[at] = page[k];   // (a page that several entries name can come back more often than there is room)
          if (c < a.width && page[k] != -1) row[c] = -1;
          to += __builtin_popcountll(bal);
        }
      }
    }
    left = left + back < a.pages ? left + back : a.pages;
    __syncthreads();
  }

  const int cap = a.width << a.page_shift;
  auto asked = [&](int s, int& before, int& entries) __attribute__((always_inline)) {   // new tokens, tokens before them, entries of the table that they lie in
    const int added = a.added[s], length = a.lengths[s];
    before = added < 0 || length < 0 ? 0 : length < kMostTokens ? length : kMostTokens;
    int n = added < 0 ? 0 : added;
    if (n > a.rows || before > cap - n || (passed[s >> 5] >> (s & 31) & 1) != 0) n = 0;
    entries = n > 0 ? ((before + n - 1) >> a.page_shift) + 1 - (before >> a.page_shift) : 0;
    return n;
  };
  // those of `each` entries from number `from` on that have no page; with a page for each of them, the first one of which is next(): they get one
  constexpr int kMostEach = 8;
  auto missing = [&](int from, int each, int entries, auto&& give) __attribute__((always_inline)) {
    unsigned none = 0;
    if (from < entries) {
      int s = last_at(flat, S, from);
      long long at[kMostEach];
      int page[kMostEach];
#pragma unroll
      for (int k = 0; k < kMostEach; k++) {
        at[k] = -1;
        if (k >= each || from + k >= entries) continue;
        while (from + k >= flat[s + 1]) s++;
        at[k] = (long long)s * a.table_stride + (base[s] >> a.page_shift) + (from + k - flat[s]);
      }
#pragma unroll
      for (int k = 0; k < kMostEach; k++) page[k] = at[k] >= 0 ? a.table[at[k]] : 0;
#pragma unroll
      for (int k = 0; k < kMostEach; k++) none |= at[k] >= 0 && checked_page(page[k], a.pages) < 0 ? 1u << k : 0u;
      give(none, at);
    }
    return __builtin_popcount(none);
  };
  int rows, entries, each, need;
#pragma unroll 1
  for (int round = 0;; round++) {
    rows = entries = 0;
    for (int s0 = 0; s0 < S; s0 += kPlanThreads) {
      const int s = s0 + tid;
      int before = 0, e = 0, all, n = s < S ? asked(s, before, e) : 0;
      const int at = block_scan(n, all, side);
      if (s < S) { start[s] = rows + at; base[s] = before; }
      rows += all;
      const int from = block_scan(e, all, side);
      if (s < S) flat[s] = entries + from;
      entries += all;
    }
    if (tid == 0) { start[S] = rows; flat[S] = entries; }
    __syncthreads();
    each = (entries + kPlanThreads - 1) / kPlanThreads;
    each = each < kMostEach ? each : kMostEach;
    need = 0;
    if ((unsigned)rows <= (unsigned)a.rows)
      for (int e0 = 0; e0 < entries; e0 += each * kPlanThreads) {
        int all;
        block_scan(missing(e0 + tid * each, each, entries, [](unsigned, const long long (&)[kMostEach]) {}), all, side);
        need += all;
      }
    if (((unsigned)rows <= (unsigned)a.rows && need <= left) || round == 1) break;
    // Not enough: one sequence after the other, those that do not fit are passed over.  (start, flat: rows and pages that each needs.)  A thread reads all of a
    // sequence's entries, and one goes through all sequences: 8 sequences of 8000 new tokens 19 us (8.6 where there are pages for all), 256 single tokens 33 (7.2),
    // 400 with trees and prompts 73 (20.6), 4096 of two tokens 557 (18).
    __syncthreads();
    for (int s = tid; s < S; s += kPlanThreads) {
      int before, e, pages = 0;
      const int n = asked(s, before, e);
      const int* const row = a.table + (long long)s * a.table_stride + (before >> a.page_shift);
#pragma unroll 8
      for (int k = 0; k < e; k++) pages += checked_page(row[k], a.pages) < 0;
      start[s] = n; flat[s] = pages;
    }
    __syncthreads();
    if (tid == 0) {
      int rows_left = a.rows, pages_left = left;
      for (int s = 0; s < S; s++) {
        const bool fits = start[s] <= rows_left && flat[s] <= pages_left;
        if (!fits) { passed[s >> 5] |= 1u << (s & 31); continue; }
        rows_left -= start[s]; pages_left -= flat[s];
      }
    }
    __syncthreads();
  }
  if (need > 0) {
    int given = 0;
    for (int e0 = 0; e0 < entries; e0 += each * kPlanThreads) {
      const int from = e0 + tid * each;
      unsigned none = 0;
      long long at[kMostEach];
      const int count = missing(from, each, entries, [&](unsigned m, const long long (&w)[kMostEach]) {
        none = m;
#pragma unroll
        for (int k = 0; k < kMostEach; k++) at[k] = w[k];
      });
      int all, p = left - 1 - given;
      p -= block_scan(count, all, side);
#pragma unroll
      for (int k = 0; k < kMostEach; k++)
        if ((none >> k & 1) != 0) {
          if (p >= 0) a.table[at[k]] = a.free_pages[p];
          p--;
        }
      given += all;
    }
  }
  if (tid == 0) { *a.count = left - need; a.starts[S] = rows; }
  for (int s = tid; s < S; s += kPlanThreads) {
    a.starts[s] = start[s];
    a.totals[s] = base[s] + start[s + 1] - start[s];
  }
  if (a.rows > kPlanRows) return;                  // (another launch's)
  __syncthreads();
  for (int row = tid; row < a.rows; row += kPlanThreads) fill_row(a, row, start, [&](int s, int) { return base[s]; });
  if (a.parents != nullptr)
    for (int s = wave; s < S; s += kPlanWaves) {
      const int n = start[s + 1] - start[s];
      if (n > 0 && n <= 64) fill_tree(a, s, start[s], n, base[s]);
    }
}

// The rows of a call of many, and behind them the trees.
constexpr int kFillRows = 256;                     // of a workgroup: one a thread (87 thousand rows: four a thread 16.7 us a call, two 14.6, so 13.7)
__global__ void __launch_bounds__(kFillRows)
plan_rows_kernel(PlanArgs a, int row_blocks) {
  if ((int)blockIdx.x >= row_blocks) {             // a sequence a wavefront
    const int s = ((int)blockIdx.x - row_blocks) * 4 + (threadIdx.x >> 6);
    if (s >= a.sequences) return;
    const int first = a.starts[s], n = a.starts[s + 1] - first;
    if (n > 0 && n <= 64) fill_tree(a, s, first, n, a.totals[s] - n);
    return;
  }
  __shared__ int start[kPlanSequences + 1];
  for (int s = threadIdx.x; s <= a.sequences; s += kFillRows) start[s] = a.starts[s];
  __syncthreads();
  const int row = blockIdx.x * kFillRows + threadIdx.x;
  if (row < a.rows) fill_row(a, row, start, [&](int s, int n) { return a.totals[s] - n; });
}

int launch_plan(const PlanArgs& a, hipStream_t s) {
  BURST_LAUNCH(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  if (a.rows > kPlanRows) {
    const int blocks = (a.rows + kFillRows - 1) / kFillRows, trees = a.parents != nullptr ? (a.sequences + 3) / 4 : 0;
    BURST_LAUNCH(plan_rows_kernel, dim3((unsigned)(blocks + trees)), dim3(kFillRows), 0, s, a, blocks);
  }
  return launch_status();
}

// ------------------------------------------------------------------------------- keep
// A thread has one granule of one head in one layer's keys or values, and moves it for all of a sequence's kept tokens, which come in increasing order to
// places that are not behind their own: eight at a time are read before they are written, and threads have nothing to do with one another.
template <typename V>
__global__ void __launch_bounds__(256)
keep_kernel(KeepArgs a, int granules, int shift) {   // granules of a row; elements of one: 1 << shift
  constexpr int kMost = 256, kAtOnce = 8;
  __shared__ long long from[kMost], to[kMost];     // of the tokens that move: granules from a head's beginning
  __shared__ int counts[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = blockIdx.y;
  const PagedSeq q = paged_seq(a.starts[s], a.starts[s + 1], a.lengths[s], a.rows, a.cap);
  int kept = a.counts[s];
  kept = kept < 0 ? 0 : kept;
  kept = min(kept, min(a.most, q.n));
  if (blockIdx.x == 0 && tid == 0) a.out[s] = max(q.at + kept, 0);
  const int column = blockIdx.x * 256 + tid, row = column / granules, g = column - row * granules, pool = row / a.heads, h = row - pool * a.heads;
  const bool active = pool < a.pools;
  V* const at = active ? (V*)a.pool[pool] + (((long long)h * a.p_head) >> shift) + g : nullptr;
  auto place = [&](int p) __attribute__((always_inline)) {
    if (p < 0 || p >= a.cap) return -1LL;
    const int page = checked_page(a.table[(long long)s * a.table_stride + (p >> a.page_shift)], a.pages);
    return page < 0 ? -1LL : (page * a.p_page + (long long)(p & ((1 << a.page_shift) - 1)) * a.p_row) >> shift;
  };
  for (int j0 = 0; j0 < kept; j0 += kMost) {
    const int j = j0 + tid;
    const int k = j < kept ? a.kept[(long long)s * a.kept_stride + j] : -1;
    long long f = -1, t = -1;
    if (k > j && k < q.n) {                        // (one that is where it belongs stays there; one that is not among the new tokens is not moved)
      f = place(q.at + k);
      t = place(q.at + j);
    }
    const bool moves = f >= 0 && t >= 0;
    const unsigned long long bal = __builtin_amdgcn_ballot_w64(moves);
    if (j0 > 0) __syncthreads();                   // (the list before this one has been read)
    if (lane == 0) counts[wave] = __builtin_popcountll(bal);
    __syncthreads();
    int n = 0, mine = 0;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      if (w == wave) mine = n;
      n += counts[w];
    }
    mine += __builtin_popcountll(bal & ((1ull << lane) - 1));
    if (moves) { from[mine] = f; to[mine] = t; }
    __syncthreads();
    if (active)
      for (int i = 0; i < n; i += kAtOnce) {
        V v[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; e++)
          if (i + e < n) v[e] = at[from[i + e]];
#pragma unroll
        for (int e = 0; e < kAtOnce; e++)
          if (i + e < n) at[to[i + e]] = v[e];
      }
  }
}

int launch_keep(const KeepArgs& a, int size, hipStream_t s) {
  auto fits = [&](int bytes) {
    const int g = bytes / size;
    bool ok = a.d % g == 0 && a.p_page % g == 0 && a.p_head % g == 0 && a.p_row % g == 0;
    for (int i = 0; i < a.pools && ok; i++) ok = reinterpret_cast<uintptr_t>(a.pool[i]) % bytes == 0;
    return ok;
  };
  const int bytes = fits(16) ? 16 : size, shift = bytes == size ? 0 : size == 2 ? 3 : 2, granules = a.d >> shift;
  const long long columns = (long long)a.pools * a.heads * granules, blocks = columns > 0 ? (columns + 255) / 256 : 1;
  if (blocks > 1 << 22) return BURST_ERR_SHAPE;
  const dim3 grid((unsigned)blocks, (unsigned)a.sequences), block(256);
  if (bytes == 16) BURST_LAUNCH((keep_kernel<i32x4>), grid, block, 0, s, a, granules, shift);
  else if (bytes == 4) BURST_LAUNCH((keep_kernel<int>), grid, block, 0, s, a, granules, shift);
  else BURST_LAUNCH((keep_kernel<short>), grid, block, 0, s, a, granules, shift);
  return launch_status();
}

}  // namespace burst
