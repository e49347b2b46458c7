// Arguments of the launches that normalise rows (burst_norm.hip), filled by the entry points.
#pragma once
#include "burst_common.h"
#include "burst_paged.h"

namespace burst {

constexpr int kNormRows = 16;                      // most rows of a workgroup
constexpr int kMaxNormItems = 12;                  // of a launch: they travel in its arguments, which hold 4 KB
constexpr int kMaxNormWeights = 64;                // of the launch that adds up their gradients
struct NormItem {
  const void* x; void* y;                          // backward: y is the gradient of x, nullptr = not wanted
  const void* g;                                   // backward: the gradient of the result
  const void* w;                                   // weights of the columns, nullptr = 1
  const long long* positions;                      // nullptr: the row's number
  long long positions_stride, offset;
  long long xs_b, xs_h, xs_r, ys_b, ys_h, ys_r;    // element strides; paged: those of y are page, head, row of a page
  long long gs_b, gs_h, gs_r;
  int B, heads, rows;
  int part;                                        // backward: row of `part` that its first block leaves its sums in, -1 = dw not wanted
  short normed, rotated, paged, w_f32;
  int first_block, row_tiles, head_tiles;          // set_tiles'
  short lanes_shift, rows_shift;                   // of a workgroup's 256 threads: lanes of a row, rows; the others take other heads
};
struct NormArgs {
  NormItem it[kMaxNormItems];
  int n, d;
  int granule;                                     // elements of a load
  float eps;
  const double* turns;
  int dims, interleaved;                           // dims = 0: not rotated
  float amplitude;
  int first;                                       // block that the launch begins with
  int heads_each;                                  // of a thread
  int tiles_each;                                  // backward: of a block
  float* part;
  // packed tokens of sequences (cached): where they go
  int cached;
  const long long* slots; const long long* places; // of the rows; nullptr: by the arrays below
  const int* starts; const int* lengths; const int* table; const long long* offsets;
  long long table_stride;
  int sequences, tokens, cap, pages, page_shift;
};
static_assert(sizeof(NormArgs) <= 4000, "kernel arguments");
struct NormSum { void* dw; int first, count, f32; };   // rows of `part` that make up a weight's gradient
struct NormSums { NormSum s[kMaxNormWeights]; const float* part; int d; };
// Granules, and the tiles of the items; returns the number of blocks of the launch, -1: more than 2^30.
long long set_tiles(NormArgs& a, int dtype, bool backward);
int launch_norm(NormArgs& a, int dtype, long long blocks, hipStream_t s);   // as set_tiles has laid it out
int launch_norm_bwd(NormArgs& a, int dtype, long long blocks, hipStream_t s);
int launch_norm_sums(const NormSums& a, int weights, hipStream_t s);

}  // namespace burst
