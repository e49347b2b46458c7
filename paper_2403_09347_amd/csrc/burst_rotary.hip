// Rotation of rows by their positions (burst_rotate), and the same on the way into a paged cache (burst_cache_append).
// A pair of columns (a, b) of a row at position p becomes (a cos - b sin, b cos + a sin) x amplitude, with the angle
// 2 pi frac(p x turns[pair]): the angle, its cos and sin in 64 bits (at position 10^6 a product in 32 bits is 0.06 off), which are rounded to
// 32; the products with a and b in 32.  The gradient is the rotation by the negative angle.
// Bound by HBM: every row is read and written once.  A workgroup takes some rows of some heads, and computes the angles of
// its rows once, into LDS, for all of those heads.  Measured: 32 + 32 heads of 4096 rows, d = 128, bf16 (134 MB in and out), 27 us, 4.9 TB/s;
// appending 7 prompts of 300 to 4096 tokens with their queries, 32 heads over 8 (272 MB), 53 us, 5.1 TB/s.  A device copy moves 5.0 TB/s.
#include "burst_rotary.h"

namespace burst {

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

constexpr int kRowsThreads = 256;

// Slots: the units of work of a row.  Half layout, VEC: 16 bytes of the first half of a pair's columns with the 16 bytes that
// belong to them; interleaved, VEC: 16 bytes; else a pair.  Columns past the rotated ones are copied, 16 bytes (a column) a slot.
// A thread keeps to one slot of one row (its cos and sin stay in registers) and goes through the heads.
template <typename T, bool VEC, bool INTER>
__global__ void __launch_bounds__(kRowsThreads)
rotate_kernel(RotateArgs a) {
  constexpr int E = VEC ? 16 / sizeof(T) : 1;      // elements of a granule
  constexpr int P = VEC ? (INTER ? E / 2 : E) : 1; // pairs of a slot
  typedef __attribute__((ext_vector_type(E))) T vec;
  __shared__ float2 turn[kRotateRows * 64];
  __shared__ long long at[kRotateRows], to[kRotateRows];   // position; where the row goes (elements of y), -1: nowhere
  const int tid = threadIdx.x, lane = tid & 63;
  const int bid = a.first + (int)blockIdx.x;
  int i = 0;
  while (i + 1 < a.n && bid >= a.it[i + 1].first_block) i++;
  const RotateItem& it = a.it[i];
  int blk = bid - it.first_block;
  const int ht = blk % it.head_tiles;
  blk /= it.head_tiles;
  const int rt = blk % it.row_tiles, b = blk / it.row_tiles;
  const int row0 = rt * a.rows_each, rows = min(a.rows_each, it.rows - row0);
  const int h0 = ht * it.heads_each, h1 = min(h0 + it.heads_each, it.heads);
  const int pairs = it.rotated ? a.dims / 2 : 0;

  const int rot_slots = pairs / P, slots = rot_slots + (it.d - 2 * pairs) / E;
  const int mine = tid % (slots * a.rows_each), sub = tid / (slots * a.rows_each), subs = kRowsThreads / (slots * a.rows_each);
  const int r = mine / slots, slot = mine - r * slots;
  const bool active = sub < subs && r < rows;
  const bool turned = slot < rot_slots;
  const int c1 = turned ? (INTER ? (VEC ? slot * E : 2 * slot) : slot * E) : 2 * pairs + (slot - rot_slots) * E;
  const int c2 = INTER ? c1 + 1 : c1 + pairs;       // (interleaved granules hold both)
  constexpr bool TWO = !(VEC && INTER);            // a slot has a second granule

  if (a.starts != nullptr) {                       // packed tokens: the sequence of every row, its position and its place in the cache
    for (int k = tid >> 6; k < rows; k += kRowsThreads / 64) {
      const int row = row0 + k;
      int s = -1;                                  // the last sequence that starts at or before the row
      for (int base = 0; base < a.sequences; base += 64) {
        const int start = base + lane < a.sequences ? a.starts[base + lane] : 0x7fffffff;
        const unsigned long long bal = __builtin_amdgcn_ballot_w64(start <= row);
        if (bal != 0) s = base + 63 - __builtin_clzll(bal);
      }
      long long pos = 0, dst = -1;
      if (s >= 0) {
        const PagedSeq q = paged_seq(a.starts[s], a.starts[s + 1], a.lengths[s], a.tokens, a.cap);
        const int p = q.at + (row - q.first);
        if (row - q.first < q.n && p >= 0) {
          pos = p + (a.offsets != nullptr ? a.offsets[s] : 0);
          if (!it.paged) {
            dst = (long long)row * it.ys_r;
          } else if (p < a.cap) {                  // (no entry of the table is behind its row)
            const int page = checked_page(a.table[(long long)s * a.table_stride + (p >> a.page_shift)], a.pages);
            if (page >= 0) dst = page * it.ys_b + (long long)(p & ((1 << a.page_shift) - 1)) * it.ys_r;
          }
        }
      }
      if (lane == 0) { at[k] = pos; to[k] = dst; }
    }
  } else if (tid < rows) {
    const long long* const p = it.positions;
    at[tid] = it.offset + (p != nullptr ? p[b * it.positions_stride + row0 + tid] : row0 + tid);
    to[tid] = b * it.ys_b + (row0 + tid) * it.ys_r;
  }
  __syncthreads();
  for (int k = tid; k < rows * pairs; k += kRowsThreads) {
    const int row = k / pairs;
    const double p = (double)at[row], t = a.turns[k - row * pairs];
    double c, s;
    cos_sin_turns(__builtin_fma(p, t, -rint(p * t)), c, s);   // (the product's own rounding does not come in)
    turn[k] = make_float2((float)(c * a.amplitude), (float)((a.inverse ? -s : s) * a.amplitude));
  }
  __syncthreads();
  if (!active) return;
  const long long dst = to[r];
  if (dst < 0) return;
  float cs[P], sn[P];
#pragma unroll
  for (int k = 0; k < P; k++) {
    const float2 v = turned ? turn[r * pairs + slot * P + k] : make_float2(1.f, 0.f);
    cs[k] = v.x; sn[k] = v.y;
  }
  const T* const x = (const T*)it.x + b * it.xs_b + (row0 + r) * it.xs_r;
  T* const y = (T*)it.y + dst;
#pragma unroll 4
  for (int h = h0 + sub; h < h1; h += subs) {
    const T* const xh = x + h * it.xs_h;
    T* const yh = y + h * it.ys_h;
    vec u = *reinterpret_cast<const vec*>(xh + c1);
    if (turned) {
      if constexpr (TWO) {
        vec v = *reinterpret_cast<const vec*>(xh + c2), o1, o2;
#pragma unroll
        for (int k = 0; k < E; k++) {
          const float f = (float)u[k], g = (float)v[k];
          o1[k] = (T)(f * cs[k] - g * sn[k]);
          o2[k] = (T)(g * cs[k] + f * sn[k]);
        }
        *reinterpret_cast<vec*>(yh + c1) = o1;
        *reinterpret_cast<vec*>(yh + c2) = o2;
      } else {
        vec o;
#pragma unroll
        for (int k = 0; k < P; k++) {
          const float f = (float)u[2 * k], g = (float)u[2 * k + 1];
          o[2 * k] = (T)(f * cs[k] - g * sn[k]);
          o[2 * k + 1] = (T)(g * cs[k] + f * sn[k]);
        }
        *reinterpret_cast<vec*>(yh + c1) = o;
      }
    } else {
      *reinterpret_cast<vec*>(yh + c1) = u;
    }
  }
}

template <typename T>
static void enqueue(const RotateArgs& a, bool vec, long long blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(kRowsThreads);
  if (vec && a.interleaved) BURST_LAUNCH((rotate_kernel<T, true, true>), grid, block, 0, s, a);
  else if (vec) BURST_LAUNCH((rotate_kernel<T, true, false>), grid, block, 0, s, a);
  else if (a.interleaved) BURST_LAUNCH((rotate_kernel<T, false, true>), grid, block, 0, s, a);
  else BURST_LAUNCH((rotate_kernel<T, false, false>), grid, block, 0, s, a);
}

// The items of `a` (all but their tiles, which are laid out here) in one launch (more only of more than 8 million blocks).
int launch_rotate(RotateArgs& a, int dtype, hipStream_t s) {
  const int E = dtype == BURST_BF16 ? 8 : 4;
  // 16-byte accesses: every granule of a row starts on 16 bytes, and no pair is cut by one
  bool vec = a.dims % (a.interleaved ? E : 2 * E) == 0;
  int d = 0;
  for (int i = 0; i < a.n; i++) {
    const RotateItem& it = a.it[i];
    d = it.d;
    vec = vec && it.d % E == 0 && (reinterpret_cast<uintptr_t>(it.x) | reinterpret_cast<uintptr_t>(it.y)) % 16 == 0;
    for (long long v : {it.xs_b, it.xs_h, it.xs_r, it.ys_b, it.ys_h, it.ys_r}) vec = vec && v % E == 0;
  }
  const int rotated = vec ? (a.interleaved ? a.dims / E : a.dims / 2 / E) + (d - a.dims) / E : a.dims / 2 + (d - a.dims);
  const int copied = vec ? d / E : d;              // slots of a row that is not rotated
  bool copies = false;
  for (int i = 0; i < a.n; i++) copies = copies || !a.it[i].rotated;
  const int slots = copies ? copied : rotated;     // (the larger number)
  double all = 0;                                  // rows x heads
  for (int i = 0; i < a.n; i++) all += (double)a.it[i].B * a.it[i].rows * a.it[i].heads;
  a.rows_each = kRotateRows;
  while (a.rows_each > 1 && a.rows_each * slots > kRowsThreads) a.rows_each /= 2;
  // Few rows: smaller blocks, so that every CU has some
  while (a.rows_each > 1 && all < 2048. * a.rows_each) a.rows_each /= 2;
  const int heads_each = 8;
  long long blocks = 0;
  for (int i = 0; i < a.n; i++) {
    RotateItem& it = a.it[i];
    it.first_block = (int)blocks;
    it.row_tiles = (it.rows + a.rows_each - 1) / a.rows_each;
    it.heads_each = heads_each;
    it.head_tiles = (it.heads + heads_each - 1) / heads_each;
    if (blocks + (double)it.B * it.row_tiles * it.head_tiles > 0x7fffffff) return BURST_ERR_SHAPE;
    blocks += (long long)it.B * it.row_tiles * it.head_tiles;
  }
  constexpr long long kMost = 1 << 23;             // blocks of a launch: it can have 2^32 threads
  for (long long first = 0; first < blocks; first += kMost) {
    a.first = (int)first;
    const long long n = blocks - first < kMost ? blocks - first : kMost;
    if (dtype == BURST_BF16) enqueue<bf16>(a, vec, n, s);
    else enqueue<float>(a, vec, n, s);
    const int e = launch_status();
    if (e != BURST_OK) return e;
  }
  return BURST_OK;
}

}  // namespace burst
