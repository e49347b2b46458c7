// Arguments of the launches that keep the books of a paged cache (burst_plan.hip), filled by the entry points.
#pragma once
#include "burst_common.h"
#include "burst_paged.h"

namespace burst {

constexpr int kPlanSequences = 4096;               // most of a call: what a sequence has is in LDS
constexpr int kPlanMostRows = (1 << 20) - 1;       // and of rows: sums over all sequences fit 32 bits, whatever the sequences ask for
constexpr int kPlanRows = 2048;                    // calls of up to so many rows are one launch
struct PlanArgs {
  const int* added; const int* lengths;
  int* table; int* free_pages; int* count;
  const int* parents;                              // nullptr: no trees
  int* starts; int* totals; long long* slots; long long* positions; unsigned long long* tree;
  long long table_stride, parents_stride;
  int sequences, rows, pages, page_shift, width, words, most;
  int window;                                      // tokens of a branch that a mask names, at most
};
int launch_plan(const PlanArgs& a, hipStream_t s);

constexpr int kMaxKeepPools = 400;                 // of a launch: they travel in its arguments, which hold 4 KB
struct KeepArgs {
  const int* starts; const int* lengths; const int* table; const int* kept; const int* counts;
  int* out;
  long long table_stride, kept_stride, p_page, p_head, p_row;   // elements
  int sequences, rows, cap, pages, page_shift, most;
  int heads, d, pools;
  void* pool[kMaxKeepPools];
};
static_assert(sizeof(KeepArgs) <= 4000, "kernel arguments");
int launch_keep(const KeepArgs& a, int size, hipStream_t s);   // size: bytes of an element

}  // namespace burst
