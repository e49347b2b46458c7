// What the kernels of burst_paged_fwd share with its entry point: their arguments, and a run's place in the work.
#pragma once
#include "burst_common.h"
#include "burst_paged.h"
#include "burst_rows.h"

namespace burst {

struct PagedArgs {
  const void* Q; void* O; float* lse;
  const void* K; const void* V;      // the pages
  const int* table;
  long long table_stride;
  long long q_row, q_head, o_row, o_head;          // element strides
  long long p_page, p_head, p_row;
  float* part;                       // partial results: [2 runs][rows_of_item][d] columns, m, l
  struct PagedJoin* join;            // [runs]
  PagedWork w;
  int heads, group, d, pages, page_shift;
  int parts_each, part_heads;        // parts of a key/value head, query heads of a part
  int runs, slack, few, o_f32;       // slack, few: see paged_deal
  int full_p;                        // see paged_chunk_kernel's TERMS
  float scale;
  const unsigned long long* tree;    // masks of the rows, tree_row words apart; nullptr: no trees
  long long tree_row;
  int words;
};
// What a run tells the merging launch: the item that is joined from the parts of n runs, from the run before it on (n = 0: none); run 0, which
// cuts none: the number of runs that have work, in n.
struct PagedJoin { int n, first, count, part, block, pad[3]; };   // first, count: the sequence's rows
static_assert(sizeof(PagedJoin) == 32, "one load");
constexpr int kShortRows = 16, kChunkRows = 128;   // rows of an item
constexpr int kShortLds = 32768;                   // bytes of a wavefront's ring of tiles

int launch_paged_short(const PagedArgs& a, int dtype, hipStream_t s);
int launch_paged_chunk(const PagedArgs& a, int dtype, hipStream_t s);
int launch_paged_merge(const PagedArgs& a, int rows_of_item, hipStream_t s);

#ifdef __HIPCC__
// Element i (the same in every lane) of an array that no kernel in flight writes, by a scalar load: it waits for no vector load.
template <typename I>
__device__ __forceinline__ int scalar_at(const int* p, I i) {
  return ((const int __attribute__((address_space(4)))*)p)[i];
}
struct ScalarRead { static __device__ __forceinline__ int at(const int* p, int i) { return scalar_at(p, __builtin_amdgcn_readfirstlane(i)); } };
template <bool TREE>
using DeviceCursor = PagedCursor<ScalarRead, TREE>;

__device__ __forceinline__ int wave_scan(int x) {  // inclusive
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);    // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // row_bcast:15 to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);    // row_bcast:31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_most(int x) {  // of numbers that are not negative; in every lane
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
// A workgroup's run and its start, by a wavefront: every lane adds up a sequence.  False: there is none for it.  The merging launch is told
// what the run's start has cut (`tell`).
// Of sequences with many blocks the lanes share the blocks where there are few such sequences: going through them takes as long as
// the longest has blocks, sharing about four blocks' time for every 64.  (us a call, lanes by themselves / so: 131072 tokens with a window of
// 1024, 8 heads over one, 1361 / 817; 16384 tokens causal 657 / 591; 4096, 32 heads over 8, 158 / 152; single tokens 0.1 more.)
template <bool TREE>
__device__ __forceinline__ bool start_run(const PagedArgs& a, int bid, int lane, bool tell, DeviceCursor<TREE>& cur, int& run) {
  const PagedWork& w = a.w;
  PagedSeq q;
  PagedTotals mine = {0, 0, 0, 0}, all = {0, 0, 0, 0};
  unsigned long long disorder = 0;
  auto totals = [&](int s) __attribute__((always_inline)) {
    q = PagedSeq{0, 0, 0, 0};
    bool bad = false;
    if (s < w.sequences) {
      const int start = w.starts[s], end = w.starts[s + 1];
      bad = !PagedWork::in_order(start, end);
      q = paged_seq(start, end, w.lengths[s], w.rows, w.cap);
    }
    disorder |= __builtin_amdgcn_ballot_w64(bad);
    const int n = w.blocks(q);
    unsigned long long longer = __builtin_amdgcn_ballot_w64(n > 8);
    if (longer != 0) {
      const int most = wave_most(n);
      if (4LL * __builtin_popcountll(longer) * ((most + 63) / 64) >= most) longer = 0;
    }
    if (((longer >> lane) & 1) == 0) mine = w.totals<TREE>(q, n, 0, 1);
#pragma unroll 1
    for (; longer != 0; longer &= longer - 1) {
      const int at = __builtin_ctzll(longer);
      const PagedSeq there = {0, __builtin_amdgcn_readlane(q.n, at), __builtin_amdgcn_readlane(q.len, at), __builtin_amdgcn_readlane(q.at, at)};
      PagedTotals t = w.totals<TREE>(there, __builtin_amdgcn_readlane(n, at), lane, 64);
      t.units = __builtin_amdgcn_readlane(wave_scan(t.units), 63);
      t.most = wave_most(t.most);
      if (lane == at) mine = t;
    }
    mine.pair = w.pair<TREE>(q, n, mine.most);
  };
#pragma unroll 1
  for (int base = 0; base < w.sequences; base += 64) {
    totals(base + lane);
    all.units += __builtin_amdgcn_readlane(wave_scan(mine.units), 63) * w.parts;
    all.items += __builtin_amdgcn_readlane(wave_scan(mine.items), 63) * w.parts;
    all.most = max(all.most, wave_most(mine.most));
    all.pair = max(all.pair, wave_most(mine.pair));
  }
  const PagedDeal deal = paged_deal(all, a.runs, a.slack, a.few);
  const int total = disorder != 0 ? 0 : deal.by_items ? all.items : all.units;
  const int active = (int)(((unsigned)total + deal.each - 1) / (unsigned)deal.each);
  run = run_of(bid, a.runs, active);
  bool some = run >= 0;
  const long long from = (long long)deal.each * run;
  if (some) {
    const int begin = (int)from;
    int before = 0, scan = 0, own = 0, base = 0;
#pragma unroll 1
    for (;; base += 64) {
      if (w.sequences > 64) totals(base + lane);
      own = (deal.by_items ? mine.items : mine.units) * w.parts;
      scan = wave_scan(own);
      const int here = __builtin_amdgcn_readlane(scan, 63);
      if (begin < before + here) break;
      before += here;
    }
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(begin < before + scan));
    const PagedSeq there = {__builtin_amdgcn_readlane(q.first, at), __builtin_amdgcn_readlane(q.n, at), __builtin_amdgcn_readlane(q.len, at),
                            __builtin_amdgcn_readlane(q.at, at)};
    const int one = __builtin_amdgcn_readlane(deal.by_items ? mine.items : mine.units, at);
    some = cur.place(w, base + at, there, one, begin - (before + __builtin_amdgcn_readlane(scan - own, at)), deal, min(deal.each, total - begin),
                     [&](int& rem, int n) __attribute__((always_inline)) {   // 64 blocks at a time
                       int place = 0;
#pragma unroll 1
                       for (; n - place > 8; place += 64) {
                         const int c = place + lane < n ? w.cost<TREE>(there, w.block_at(place + lane, n)) : 0, sum = wave_scan(c);
                         if (rem < __builtin_amdgcn_readlane(sum, 63)) {
                           const int i = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rem < sum));
                           rem -= __builtin_amdgcn_readlane(sum - c, i);
                           return place + i;
                         }
                         rem -= __builtin_amdgcn_readlane(sum, 63);
                       }
                       return place;
                     });
  }
  if (tell && a.join != nullptr && (run >= 0 || bid == 0)) {
    PagedJoin j = {0, 0, 0, 0, 0, {0, 0, 0}};
    if (some && !deal.by_items) j = PagedJoin{parts_to_join(cur.g, deal.each), cur.g.q.first, cur.g.q.n, cur.g.part, cur.g.block, {0, 0, 0}};
    if (bid == 0) j.n = active;
    a.join[bid == 0 ? 0 : run] = j;
  }
  return some;
}
#endif

}  // namespace burst
