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
  PagedWork w;
  int heads, group, d, pages, page_shift;
  int parts_each, part_heads;        // parts of a key/value head, query heads of a part
  int runs, o_f32;
  float scale;
};
constexpr int kShortRows = 16, kChunkRows = 128;   // rows of an item
constexpr int kShortLds = 32768;                   // bytes of a wavefront's ring

int launch_paged_short(const PagedArgs& a, int dtype, hipStream_t s);
int launch_paged_chunk(const PagedArgs& a, hipStream_t s);
int launch_paged_merge(const PagedArgs& a, int rows_of_item, hipStream_t s);

#ifdef __HIPCC__
// Element i (the same in every lane) of an array that no kernel in flight writes, by a scalar load: it waits for no vector load.
template <typename I>
__device__ __forceinline__ int scalar_at(const int* p, I i) {
  return ((const int __attribute__((address_space(4)))*)p)[i];
}
struct ScalarRead { static __device__ __forceinline__ int at(const int* p, int i) { return scalar_at(p, __builtin_amdgcn_readfirstlane(i)); } };
struct DeviceCursor : PagedCursor<ScalarRead> { long long run; };

// Workgroup -> run: an XCD (ids go to the eight in turn) gets neighbouring runs, which share keys.
__device__ __forceinline__ int run_of(int bid, int runs) {
  return runs % 8 == 0 ? (bid & 7) * (runs / 8) + (bid >> 3) : bid;
}
__device__ __forceinline__ long long wave_scan(long long x, int lane) {   // inclusive
  for (int off = 1; off < 64; off <<= 1) {
    const long long y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  return x;
}
__device__ __forceinline__ long long lane_value64(long long x, int lane) {
  return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) |
                     (unsigned)__builtin_amdgcn_readlane((int)x, lane));
}
// The start of run `run`, by a wavefront: every lane adds up the units of a sequence.  False: the run has none.
__device__ __forceinline__ bool locate_run(const PagedArgs& a, int run, int lane, DeviceCursor& cur) {
  const PagedWork& w = a.w;
  auto units = [&](int s) -> long long {
    if (s >= w.sequences) return 0;
    return w.cost(paged_seq(w.starts[s], w.starts[s + 1], w.lengths[s], w.rows, w.cap)) * w.parts;
  };
  long long total = 0, mine = 0, scan = 0;
  for (int base = 0; base < w.sequences; base += 64) {
    mine = units(base + lane);
    scan = wave_scan(mine, lane);
    total += lane_value64(scan, 63);
  }
  cur.run = run_length(total, a.runs);
  const long long begin = cur.run * run;
  if (begin >= total) return false;
  long long before = 0;
  int base = 0;
  for (;; base += 64) {
    if (w.sequences > 64) {
      mine = units(base + lane);
      scan = wave_scan(mine, lane);
    }
    const long long all = lane_value64(scan, 63);
    if (begin < before + all) break;
    before += all;
  }
  const unsigned long long bal = __builtin_amdgcn_ballot_w64(begin < before + scan);
  const int at = __builtin_ctzll(bal);
  const long long rem = begin - (before + lane_value64(scan - mine, at));
  cur.place(w, base + at, rem, min(cur.run, total - begin));
  return true;
}
#endif

}  // namespace burst
