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

#ifdef __HIPCC__
// cos and sin of 2 pi x, in 64 bits: the nearest quarter turn taken off (exactly), and Taylor's series within pi/4 of it (terms up to x^12 and
// x^11: the next ones are below 2^-41 and 2^-37).  Rounded to 32 bits by the caller, once.
__device__ __forceinline__ void cos_sin_turns(double x, double& c, double& s) {
  const double q = rint(4 * x);
  const double t = (x - 0.25 * q) * 6.283185307179586, u = t * t;
  const double cs = 1 + u * (-0.5 + u * (1. / 24 + u * (-1. / 720 + u * (1. / 40320 + u * (-1. / 3628800 + u * (1. / 479001600))))));
  const double sn = t + t * u * (-1. / 6 + u * (1. / 120 + u * (-1. / 5040 + u * (1. / 362880 - u * (1. / 39916800)))));
  const int n = (int)q & 3;
  c = n == 0 ? cs : n == 1 ? -sn : n == 2 ? -cs : sn;
  s = n == 0 ? sn : n == 1 ? cs : n == 2 ? -sn : -cs;
}
#endif

}  // namespace burst
