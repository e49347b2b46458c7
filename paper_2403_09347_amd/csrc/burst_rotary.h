// Arguments of the row-rotating launches (burst_rotary.hip), filled by the entry points.
#pragma once
#include "burst_common.h"
#include "burst_paged.h"

namespace burst {

constexpr int kRotateRows = 16;                    // most rows of a workgroup
constexpr int kMaxRotateSize = 0x7fffff00;         // of a dimension: rows and heads of a workgroup are counted past the last one in 32 bits
constexpr int kMaxRotateItems = 20;                // of a launch: they travel in its arguments, which hold 4 KB
struct RotateItem {
  const void* x; void* y;
  const long long* positions;                      // nullptr: the row's number
  long long positions_stride, offset;
  long long xs_b, xs_h, xs_r, ys_b, ys_h, ys_r;    // element strides; paged: those of y are page, head, row of a page
  int B, heads, rows, d;
  int rotated, paged;                              // rotated = 0: copied
  int first_block, row_tiles, head_tiles, heads_each;   // launch_rotate's
};
struct RotateArgs {
  RotateItem it[kMaxRotateItems];
  int n;
  const double* turns;
  int dims, interleaved, inverse;
  float amplitude;
  int rows_each;
  int first;                                       // block that the launch begins with
  // packed tokens of sequences (starts != nullptr): rows behind the last sequence and at negative positions are left out
  const int* starts; const int* lengths; const int* table; const long long* offsets;
  long long table_stride;
  int sequences, tokens, cap, pages, page_shift;
};
static_assert(sizeof(RotateArgs) <= 4000, "kernel arguments");
int launch_rotate(RotateArgs& a, int dtype, hipStream_t s);

}  // namespace burst
