// Rows normalised by their root mean square, weighted column by column, and rotated by their positions, in one pass
// (burst_norm_rotate, burst_cache_store), and the gradient of that (burst_norm_rotate_bwd).
//   r = (mean of x^2 + eps)^(-1/2);  n = x r w;  y = R(position) n,  R as in burst_rotary.hip
//   h = R^T g;  dw = sum over the rows of h x r;  u = h w;  dx = r (u - x r^2 (sum of u x) / d)
// All of it in 32 bits (angles in 64), rounded once; sums over a row by the lanes that hold it, in a fixed order.
// Bound by HBM: the forward reads and writes every row once, the backward reads x and g and writes dx; r is computed again, which costs
// nothing beside x, which the gradient needs anyway.  Measured, d = 128, bf16: 40 heads of 8192 rows forward 44 us, 3.8 TB/s, backward 56 us and its sums
// 4, 4.2 TB/s (a device copy moves 5.1); fp32, 20 heads of 4096 rows, 19, 30 and 4 us.  Where the loads of all workgroups and their stores take turns
// (5 a CU do these sizes in one or two rounds) nothing overlaps the arithmetic, 8 us of the first of these.
#include <type_traits>

#include "burst_norm.h"
#include "burst_rotary.h"

namespace burst {

constexpr int kNormThreads = 256;

// Sum over groups of 1 << shift neighbouring lanes, in every lane of them.
__device__ __forceinline__ float group_sum(float x, int shift) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (shift > 0) x += dpp(x, std::integral_constant<int, 0xb1>());    // quad_perm: neighbours
  if (shift > 1) x += dpp(x, std::integral_constant<int, 0x4e>());    // quad_perm: pairs
  if (shift > 2) x += dpp(x, std::integral_constant<int, 0x141>());   // row_half_mirror
  if (shift > 3) x += dpp(x, std::integral_constant<int, 0x140>());   // row_mirror
  if (shift > 4) x += __shfl_xor(x, 16);
  if (shift > 5) x += __shfl_xor(x, 32);
  return x;
}

// What a thread does: the slots of a row that it holds.  Half layout: a granule of the first half of the pairs' columns with the granule
// that belongs to it; interleaved (and columns past the rotated ones): one granule.  Single elements: two slots a lane.
template <int E, bool INTER>
struct NormSlots {
  static constexpr int N = E == 1 ? 2 : 1;         // slots of a lane
  static constexpr int P = E > 1 && INTER ? E / 2 : E;   // pairs of a slot
  static constexpr bool TWO = E == 1 || !INTER;
  int c1[N], c2[N], pair[N];                       // columns; first pair
  bool there[N], turned[N];
  __device__ __forceinline__ void set(int lane, int lanes_shift, int pairs, int d) {
    const int rot = pairs / P, all = rot + (d - 2 * pairs) / E;
#pragma unroll
    for (int k = 0; k < N; k++) {
      const int slot = lane + (k << lanes_shift);
      there[k] = slot < all;
      turned[k] = slot < rot;
      c1[k] = turned[k] ? (INTER ? (E > 1 ? slot * E : 2 * slot) : slot * E) : 2 * pairs + (slot - rot) * E;
      c2[k] = INTER ? c1[k] + 1 : c1[k] + pairs;   // (interleaved granules hold both)
      pair[k] = slot * P;
    }
  }
};
template <typename T, int E>
struct Granule { typedef __attribute__((ext_vector_type(E))) T vec; };
// sum + the squares of a granule (bf16: two at a time, no conversions).
template <typename T, int E>
__device__ __forceinline__ float add_squares(const typename Granule<T, E>::vec& x, float sum) {
  if constexpr (sizeof(T) == 2 && E > 1) {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const bf16x2 p = {x[e], x[e + 1]};
      sum = __builtin_amdgcn_fdot2_f32_bf16(p, p, sum, false);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; e++) sum = __builtin_fmaf((float)x[e], (float)x[e], sum);
  }
  return sum;
}
// Weights of a granule's columns.
template <typename T, int E>
__device__ __forceinline__ void load_weights(float (&out)[E], const NormItem& it, int c, bool there) {
  typedef typename Granule<T, E>::vec vec;
  typedef typename Granule<float, E>::vec fvec;
  if (it.w == nullptr || !there) {
#pragma unroll
    for (int e = 0; e < E; e++) out[e] = 1.f;
  } else if (it.w_f32) {
    const fvec v = *reinterpret_cast<const fvec*>((const float*)it.w + c);
#pragma unroll
    for (int e = 0; e < E; e++) out[e] = v[e];
  } else {
    const vec v = *reinterpret_cast<const vec*>((const T*)it.w + c);
#pragma unroll
    for (int e = 0; e < E; e++) out[e] = (float)v[e];
  }
}

// Positions of a block's rows, and where they go (elements of y; -1: nowhere).
__device__ __forceinline__ void find_rows(const NormArgs& a, const NormItem& it, int b, int row0, int rows, long long* at, long long* to) {
  const int tid = threadIdx.x, lane = tid & 63;
  if (!a.cached) {
    if (tid < rows) {
      const long long* const p = it.positions;
      at[tid] = it.offset + (p != nullptr ? p[b * it.positions_stride + row0 + tid] : row0 + tid);
      to[tid] = b * it.ys_b + (row0 + tid) * it.ys_r;
    }
    return;
  }
  auto in_pages = [&](long long slot) __attribute__((always_inline)) {
    const long long page = slot >> a.page_shift;
    return slot < 0 || page >= a.pages ? -1 : page * it.ys_b + (slot & ((1LL << a.page_shift) - 1)) * it.ys_r;
  };
  if (a.slots != nullptr && a.places != nullptr) {
    if (tid < rows) {
      const int row = row0 + tid;
      const long long pos = a.places[row], dst = it.paged ? in_pages(a.slots[row]) : (long long)row * it.ys_r;
      at[tid] = pos;
      to[tid] = pos >= 0 ? dst : -1;
    }
    return;
  }
  for (int k = tid >> 6; k < rows; k += kNormThreads / 64) {   // the sequence of every row
    const int row = row0 + k;
    int s = -1;                                    // the last sequence that starts at or before the row
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
        pos = a.places != nullptr ? a.places[row] : p + (a.offsets != nullptr ? a.offsets[s] : 0);
        if (!it.paged) {
          dst = (long long)row * it.ys_r;
        } else if (a.slots != nullptr) {
          dst = in_pages(a.slots[row]);
        } else if (p < a.cap) {                    // (no entry of the table is behind its row)
          const int page = checked_page(a.table[(long long)s * a.table_stride + (p >> a.page_shift)], a.pages);
          if (page >= 0) dst = page * it.ys_b + (long long)(p & ((1 << a.page_shift) - 1)) * it.ys_r;
        }
        if (a.places != nullptr && pos < 0) dst = -1;
      }
    }
    if (lane == 0) { at[k] = pos; to[k] = dst; }
  }
}
// cos and sin of a block's rows.
__device__ __forceinline__ void find_turns(const NormArgs& a, int pairs, int rows, const long long* at, float2* turn) {
  for (int k = threadIdx.x; k < rows * pairs; k += kNormThreads) {
    const int row = k / pairs;
    const double p = (double)at[row], t = a.turns[k - row * pairs];
    double c, s;
    cos_sin_turns(__builtin_fma(p, t, -rint(p * t)), c, s);   // (the product's own rounding does not come in)
    turn[k] = make_float2((float)(c * a.amplitude), (float)(s * a.amplitude));
  }
}
struct NormTile { int b, row0, rows, h0; };
__device__ __forceinline__ NormTile tile_of(const NormArgs& a, const NormItem& it, int tile) {
  NormTile t;
  const int ht = tile % it.head_tiles;
  tile /= it.head_tiles;
  const int rt = tile % it.row_tiles;
  t.b = tile / it.row_tiles;
  t.row0 = rt << it.rows_shift;
  t.rows = min(1 << it.rows_shift, it.rows - t.row0);
  t.h0 = ht * ((kNormThreads >> (it.lanes_shift + it.rows_shift)) * a.heads_each);
  return t;
}

// A workgroup takes up to 16 rows of some heads; a thread keeps to its columns of one row (cos, sin and weights stay in registers) and takes
// NH heads, all of which are asked for before anything else is done.
template <typename T, int E, bool INTER, int NH>
__global__ void __launch_bounds__(kNormThreads)
norm_kernel(NormArgs a) {
  typedef NormSlots<E, INTER> Slots;
  typedef typename Granule<T, E>::vec vec;
  constexpr int N = Slots::N, P = Slots::P;
  constexpr bool TWO = Slots::TWO;
  __shared__ float2 turn[kNormRows * 64];
  __shared__ long long at[kNormRows], to[kNormRows];
  const int tid = threadIdx.x, bid = a.first + (int)blockIdx.x;
  int i = 0;
  while (i + 1 < a.n && bid >= a.it[i + 1].first_block) i++;
  const NormItem& it = a.it[i];
  const NormTile t = tile_of(a, it, bid - it.first_block);
  const int lanes = 1 << it.lanes_shift, pairs = it.rotated ? a.dims / 2 : 0;
  const int r = (tid >> it.lanes_shift) & ((1 << it.rows_shift) - 1), sub = tid >> (it.lanes_shift + it.rows_shift);
  const int subs = kNormThreads >> (it.lanes_shift + it.rows_shift);
  Slots s;
  s.set(tid & (lanes - 1), it.lanes_shift, pairs, a.d);
  const bool row_there = r < t.rows;

  const T* xh = (const T*)it.x + t.b * it.xs_b + (t.row0 + (row_there ? r : 0)) * it.xs_r + (t.h0 + sub) * it.xs_h;
  vec u[NH][N], v[NH][N];
#pragma unroll
  for (int j = 0; j < NH; j++, xh += subs * it.xs_h) {
    const int h = t.h0 + sub + j * subs;
#pragma unroll
    for (int k = 0; k < N; k++) {
      u[j][k] = v[j][k] = (vec)(T)0.f;
      if (row_there && h < it.heads && s.there[k]) {
        u[j][k] = *reinterpret_cast<const vec*>(xh + s.c1[k]);
        if (TWO && s.turned[k]) v[j][k] = *reinterpret_cast<const vec*>(xh + s.c2[k]);
      }
    }
  }
  float w1[N][E], w2[N][E];
#pragma unroll
  for (int k = 0; k < N; k++) {
    load_weights<T, E>(w1[k], it, s.c1[k], s.there[k]);
    load_weights<T, E>(w2[k], it, s.c2[k], TWO && s.there[k] && s.turned[k]);
  }
  find_rows(a, it, t.b, t.row0, t.rows, at, to);
  __syncthreads();
  if (pairs > 0) find_turns(a, pairs, t.rows, at, turn);
  __syncthreads();
  float cs[N][P], sn[N][P];
#pragma unroll
  for (int k = 0; k < N; k++)
#pragma unroll
    for (int p = 0; p < P; p++) {
      const bool some = row_there && s.turned[k];
      const float2 cv = turn[some ? r * pairs + s.pair[k] + p : 0];
      cs[k][p] = some ? cv.x : 1.f; sn[k][p] = some ? cv.y : 0.f;
    }
  // (the weights go into cos and sin, which all heads share: r (x (w cos) - x' (w' sin)))
  float wc1[N][E], wc2[N][E], ws1[N][E], ws2[N][E];
#pragma unroll
  for (int k = 0; k < N; k++)
#pragma unroll
    for (int e = 0; e < E; e++) {
      const int p = TWO ? e : e / 2, o = TWO ? e : e ^ 1;
      wc1[k][e] = w1[k][e] * cs[k][p]; ws1[k][e] = (TWO ? w2[k][e] : w1[k][o]) * sn[k][p];
      if (TWO) { wc2[k][e] = w2[k][e] * cs[k][p]; ws2[k][e] = w1[k][e] * sn[k][p]; }
    }
  const long long dst = row_there ? to[r] : -1;
  T* yh = (T*)it.y + dst + (t.h0 + sub) * it.ys_h;
#pragma unroll
  for (int j = 0; j < NH; j++, yh += subs * it.ys_h) {
    const int h = t.h0 + sub + j * subs;
    float f = 1.f;
    if (it.normed) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < N; k++) {
        sum = add_squares<T, E>(u[j][k], sum);
        if (TWO) sum = add_squares<T, E>(v[j][k], sum);
      }
      f = 1.f / sqrtf(group_sum(sum, it.lanes_shift) / (float)a.d + a.eps);
    }
    if (dst < 0 || h >= it.heads) continue;
#pragma unroll
    for (int k = 0; k < N; k++) {
      if (!s.there[k]) continue;
      vec o1, o2;
      if (!s.turned[k]) {
        o1 = u[j][k];
        if (it.normed)
#pragma unroll
          for (int e = 0; e < E; e++) o1[e] = (T)((float)u[j][k][e] * f * w1[k][e]);
        *reinterpret_cast<vec*>(yh + s.c1[k]) = o1;
      } else if constexpr (TWO) {
#pragma unroll
        for (int e = 0; e < E; e++) {
          const float p = (float)u[j][k][e], q = (float)v[j][k][e];
          o1[e] = (T)(f * (p * wc1[k][e] - q * ws1[k][e]));
          o2[e] = (T)(f * (q * wc2[k][e] + p * ws2[k][e]));
        }
        *reinterpret_cast<vec*>(yh + s.c1[k]) = o1;
        *reinterpret_cast<vec*>(yh + s.c2[k]) = o2;
      } else {
#pragma unroll
        for (int e = 0; e < P; e++) {
          const float p = (float)u[j][k][2 * e], q = (float)u[j][k][2 * e + 1];
          o1[2 * e] = (T)(f * (p * wc1[k][2 * e] - q * ws1[k][2 * e]));
          o1[2 * e + 1] = (T)(f * (q * wc1[k][2 * e + 1] + p * ws1[k][2 * e + 1]));
        }
        *reinterpret_cast<vec*>(yh + s.c1[k]) = o1;
      }
    }
  }
}

// The gradient.  Tiles as above with one head a thread; a workgroup takes several, one after the other: the next one's rows are asked for before this one's
// are worked on, and neighbouring tiles are other heads of the same rows, whose cos and sin stay.  It keeps the sums of dw over all of its tiles:
// its rows' lanes each have a part of them, which are added up in LDS at the end and left in `part`, a row for every workgroup.
template <typename T, int E, bool INTER>
__global__ void __launch_bounds__(kNormThreads, 3)
norm_bwd_kernel(NormArgs a) {
  typedef NormSlots<E, INTER> Slots;
  typedef typename Granule<T, E>::vec vec;
  constexpr int N = Slots::N, P = Slots::P;
  constexpr bool TWO = Slots::TWO;
  constexpr int kSums = 2 * kNormThreads * (E == 1 ? 2 : E);   // (lanes of a row hold its columns, two granules each at most)
  __shared__ union { float2 turn[kNormRows * 64]; float sums[kSums]; float two[2][128]; } sh;
  __shared__ long long at[kNormRows], to[kNormRows];
  const int tid = threadIdx.x, bid = a.first + (int)blockIdx.x;
  int i = 0;
  while (i + 1 < a.n && bid >= a.it[i + 1].first_block) i++;
  const NormItem& it = a.it[i];
  const int lanes = 1 << it.lanes_shift, pairs = it.rotated ? a.dims / 2 : 0;
  const int rs = tid >> it.lanes_shift, r = rs & ((1 << it.rows_shift) - 1), sub = rs >> it.rows_shift;
  const int first = (bid - it.first_block) * a.tiles_each, tiles = min(a.tiles_each, it.B * it.row_tiles * it.head_tiles - first);
  const int heads = kNormThreads >> (it.lanes_shift + it.rows_shift);   // of a tile
  Slots s;
  s.set(tid & (lanes - 1), it.lanes_shift, pairs, a.d);
  // the tile whose rows are asked for: its heads' number ht of the rows' number rt of batch entry b
  vec u[N], v[N], gu[N], gv[N];
  int ht = first % it.head_tiles, rt = first / it.head_tiles, b = rt / it.row_tiles;
  rt -= b * it.row_tiles;
  const T *x, *g;
  int rows;
  auto enter = [&]() __attribute__((always_inline)) {   // the first of some rows' tiles
    const int row0 = rt << it.rows_shift;
    rows = min(1 << it.rows_shift, it.rows - row0);
    const long long row = row0 + (r < rows ? r : 0), h = ht * heads + sub;
    x = (const T*)it.x + b * it.xs_b + row * it.xs_r + h * it.xs_h;
    g = (const T*)it.g + b * it.gs_b + row * it.gs_r + h * it.gs_h;
  };
  auto fetch = [&]() __attribute__((always_inline)) {
    const bool there = r < rows && ht * heads + sub < it.heads;
#pragma unroll
    for (int k = 0; k < N; k++) {
      u[k] = v[k] = gu[k] = gv[k] = (vec)(T)0.f;
      if (there && s.there[k]) {
        u[k] = *reinterpret_cast<const vec*>(x + s.c1[k]);
        gu[k] = *reinterpret_cast<const vec*>(g + s.c1[k]);
        if (TWO && s.turned[k]) {
          v[k] = *reinterpret_cast<const vec*>(x + s.c2[k]);
          gv[k] = *reinterpret_cast<const vec*>(g + s.c2[k]);
        }
      }
    }
  };
  enter();
  fetch();
  float w1[N][E], w2[N][E], d1[N][E], d2[N][E], cs[N][P], sn[N][P];
#pragma unroll
  for (int k = 0; k < N; k++) {
    load_weights<T, E>(w1[k], it, s.c1[k], s.there[k]);
    load_weights<T, E>(w2[k], it, s.c2[k], TWO && s.there[k] && s.turned[k]);
#pragma unroll
    for (int e = 0; e < E; e++) d1[k][e] = d2[k][e] = 0.f;
  }
  const float inv_d = 1.f / (float)a.d;
  bool other = true;                               // other rows than those that cos and sin are of
  T* y = nullptr;
#pragma unroll 1
  for (int tile = 0; tile < tiles; tile++) {
    const int h = ht * heads + sub;
    const bool row_there = r < rows, store = it.y != nullptr && row_there && h < it.heads;
    if (other) {
      __syncthreads();                             // (the rows before have been read)
      find_rows(a, it, b, rt << it.rows_shift, rows, at, to);
      __syncthreads();
      if (pairs > 0) {
        find_turns(a, pairs, rows, at, sh.turn);
        __syncthreads();
      }
      y = (T*)it.y + (row_there ? to[r] : 0) + h * it.ys_h;
#pragma unroll
      for (int k = 0; k < N; k++)
#pragma unroll
        for (int p = 0; p < P; p++) {
          const bool some = row_there && s.turned[k];
          const float2 cv = sh.turn[some ? r * pairs + s.pair[k] + p : 0];
          cs[k][p] = some ? cv.x : 1.f; sn[k][p] = some ? cv.y : 0.f;
        }
    }
    vec x1[N], x2[N];
    float h1[N][E], h2[N][E], ss = 0.f, ux = 0.f;  // R^T g; sums of x^2 and of u x
#pragma unroll
    for (int k = 0; k < N; k++) {
      x1[k] = u[k]; x2[k] = v[k];
      if constexpr (TWO) {
#pragma unroll
        for (int e = 0; e < E; e++) {
          const float p = (float)gu[k][e], q = (float)gv[k][e];
          h1[k][e] = p * cs[k][e] + q * sn[k][e];
          h2[k][e] = s.turned[k] ? q * cs[k][e] - p * sn[k][e] : 0.f;   // (p may be infinite: sn = 0 does not keep it out)
        }
      } else {
#pragma unroll
        for (int e = 0; e < P; e++) {
          const float p = (float)gu[k][2 * e], q = (float)gu[k][2 * e + 1];
          h1[k][2 * e] = s.turned[k] ? p * cs[k][e] + q * sn[k][e] : p;   // (as above)
          h1[k][2 * e + 1] = s.turned[k] ? q * cs[k][e] - p * sn[k][e] : q;
        }
      }
    }
    other = ht + 1 == it.head_tiles;
    if (tile + 1 < tiles) {
      if (other) {
        ht = 0;
        if (++rt == it.row_tiles) { rt = 0; b++; }
        enter();
      } else {
        ht++;
        x += heads * it.xs_h;
        g += heads * it.gs_h;
      }
      fetch();
    }
#pragma unroll
    for (int k = 0; k < N; k++) {
      ss = add_squares<T, E>(x1[k], ss);
      if (TWO) ss = add_squares<T, E>(x2[k], ss);
#pragma unroll
      for (int e = 0; e < E; e++) {
        ux = __builtin_fmaf(h1[k][e] * (float)x1[k][e], w1[k][e], ux);
        if (TWO) ux = __builtin_fmaf(h2[k][e] * (float)x2[k][e], w2[k][e], ux);
      }
    }
    const float f = 1.f / sqrtf(group_sum(ss, it.lanes_shift) / (float)a.d + a.eps);
    const float c = group_sum(ux, it.lanes_shift) * inv_d * f * f;
#pragma unroll
    for (int k = 0; k < N; k++) {
      vec o1, o2;
#pragma unroll
      for (int e = 0; e < E; e++) {
        const float f1 = (float)x1[k][e];
        d1[k][e] = __builtin_fmaf(h1[k][e] * f1, f, d1[k][e]);
        o1[e] = (T)(f * (h1[k][e] * w1[k][e] - f1 * c));
        if (TWO) {
          const float f2 = (float)x2[k][e];
          d2[k][e] = __builtin_fmaf(h2[k][e] * f2, f, d2[k][e]);
          o2[e] = (T)(f * (h2[k][e] * w2[k][e] - f2 * c));
        }
      }
      if (store && s.there[k]) {
        *reinterpret_cast<vec*>(y + s.c1[k]) = o1;
        if (TWO && s.turned[k]) *reinterpret_cast<vec*>(y + s.c2[k]) = o2;
      }
    }
    y += heads * it.ys_h;
  }
  if (it.part < 0) return;
  __syncthreads();                                 // (the last tile's cos and sin have been read)
#pragma unroll
  for (int k = 0; k < N; k++) {
    if (!s.there[k]) continue;
#pragma unroll
    for (int e = 0; e < E; e++) {
      sh.sums[rs * a.d + s.c1[k] + e] = d1[k][e];
      if (TWO && s.turned[k]) sh.sums[rs * a.d + s.c2[k] + e] = d2[k][e];
    }
  }
  __syncthreads();
  const int c = tid & 127, half = tid >> 7, all = kNormThreads >> it.lanes_shift;
  float sum = 0.f;
  if (c < a.d)
    for (int q = half; q < all; q += 2) sum += sh.sums[q * a.d + c];
  __syncthreads();
  sh.two[half][c] = sum;
  __syncthreads();
  if (half == 0 && c < a.d) a.part[(size_t)(it.part + (bid - it.first_block)) * a.d + c] = sum + sh.two[1][c];
}

// A weight's gradient from its rows of `part`: 32 columns a workgroup, 32 rows at a time, in a fixed order.
__global__ void __launch_bounds__(1024)
norm_sums_kernel(NormSums a) {
  __shared__ float side[32][33];
  const NormSum w = a.s[blockIdx.x];
  const int col = threadIdx.x & 31, row = threadIdx.x >> 5, c = blockIdx.y * 32 + col;
  float sum = 0.f;
  if (c < a.d) {
    const float* const p = a.part + (size_t)w.first * a.d + c;
#pragma unroll 8
    for (int i = row; i < w.count; i += 32) sum += p[(size_t)i * a.d];
  }
  side[row][col] = sum;
  __syncthreads();
  const float v = side[col][row];                  // (transposed: the rows of column `row` in 32 neighbouring lanes)
  const float all = group_sum(v, 5);
  if (col == 0 && blockIdx.y * 32 + row < a.d) {
    const int at = blockIdx.y * 32 + row;
    if (w.f32) ((float*)w.dw)[at] = all;
    else ((bf16*)w.dw)[at] = (bf16)all;
  }
}

constexpr int kBackBlocks = 768;                   // workgroups of a backward launch: three a CU, as many as are there at once
long long set_tiles(NormArgs& a, int dtype, bool backward) {
  const int size = dtype == BURST_BF16 ? 2 : 4;
  // Granules of 16 bytes (bf16: else 8): every one of a row starts on its own size, and no pair is cut by one.
  auto fits = [&](int E) {
    bool ok = a.d % E == 0 && (a.interleaved ? a.dims % E == 0 : a.dims / 2 % E == 0);
    for (int i = 0; i < a.n && ok; i++) {
      const NormItem& it = a.it[i];
      ok = ((reinterpret_cast<uintptr_t>(it.x) | reinterpret_cast<uintptr_t>(it.y) | reinterpret_cast<uintptr_t>(it.g)) % (E * size)) == 0 &&
           reinterpret_cast<uintptr_t>(it.w) % 16 == 0;
      for (long long v : {it.xs_b, it.xs_h, it.xs_r, it.ys_b, it.ys_h, it.ys_r, it.gs_b, it.gs_h, it.gs_r}) ok = ok && v % E == 0;
    }
    return ok;
  };
  a.granule = fits(16 / size) ? 16 / size : size == 2 && fits(4) ? 4 : 1;
  const int E = a.granule;
  double all = 0;                                  // rows x heads
  for (int i = 0; i < a.n; i++) all += (double)a.it[i].B * a.it[i].rows * a.it[i].heads;
  // Heads of a thread: four where there are many rows, one, which leaves no CU idle, elsewhere.  us forward, bf16, 32 + 8 heads, one / four: d = 128, in all
  // 16384 rows 5.5 / 7.3, 32768 6.8 / 8.2, 65536 10.7 / 12.2, 131072 16.4 / 16.1, 262144 30.6 / 28.0; d = 64, 32768 5.5 / 7.3, 131072 11.0 / 11.8, 262144 16.2 /
  // 15.7; so one would serve up to about 100 thousand rows, d = 128, and 200 thousand, d = 64, better, by up to 1.8 us.  The backward takes one,
  // with the next tile's on their way (four of them: 44 instead of 40).
  a.heads_each = !backward && all >= 32768 ? 4 : 1;
  long long blocks = 0;
  auto lay = [&](int tiles_each) {
    blocks = 0;
    for (int i = 0; i < a.n; i++) {
      NormItem& it = a.it[i];
      const int pairs = it.rotated ? a.dims / 2 : 0;
      const int rot = a.interleaved && E > 1 ? 2 * pairs / E : pairs / E, slots = rot + (a.d - 2 * pairs) / E;
      it.lanes_shift = 0;
      while ((1 << it.lanes_shift) * (E == 1 ? 2 : 1) < slots) it.lanes_shift++;
      // Rows and heads of a tile, whose product is given.  A row's work counts 2 a head that a thread takes, there or not, and the angle of a pair 1; in the
      // backward the next heads' tiles have the angles already, and of tiles that cost the same the ones with more rows are taken, which read longer
      // pieces.  us: 40 heads of 8192 rows, d = 128, bf16, forward, 4 rows x 32 heads 49.8, so (8 x 16) 42.4; backward of 40 heads, d = 64, 8 rows x
      // 8 and 4 heads 84, so (16 x 4 and 2) 69, of 32 heads, 16384 rows, d = 96, 92 and 76.
      const int groups = kNormThreads >> it.lanes_shift;
      double least = 0;
      it.rows_shift = 0;
      for (int shift = 0; (1 << shift) <= kNormRows && (groups >> shift) >= 1; shift++) {
        const int each = (groups >> shift) * a.heads_each;
        const double tiles = (it.heads + each - 1) / each, angles = (double)(1 << shift) * pairs / kNormThreads;
        const double cost = (tiles * 2 * a.heads_each + (backward ? angles : tiles * angles)) / (1 << shift);
        if (shift == 0 || cost < least * (backward ? 1.001 : 1.)) { least = cost; it.rows_shift = (short)shift; }
      }
      const int heads = (groups >> it.rows_shift) * a.heads_each;
      it.row_tiles = (int)(((long long)it.rows + (1 << it.rows_shift) - 1) >> it.rows_shift);
      it.head_tiles = (it.heads + heads - 1) / heads;
      it.first_block = (int)blocks;
      const double tiles = (double)it.B * it.row_tiles * it.head_tiles;
      if (tiles > 1 << 30 || blocks + tiles / tiles_each + 1 > 1 << 30) { blocks = -1; return; }
      blocks += ((long long)it.B * it.row_tiles * it.head_tiles + tiles_each - 1) / tiles_each;
    }
  };
  a.tiles_each = 1;
  lay(1);
  if (backward && blocks > kBackBlocks) {
    a.tiles_each = (int)((blocks + kBackBlocks - 1) / kBackBlocks);
    lay(a.tiles_each);
  }
  return blocks;
}

template <typename T, int E, bool INTER>
static void enqueue(const NormArgs& a, bool backward, long long blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(kNormThreads);
  if (backward) BURST_LAUNCH((norm_bwd_kernel<T, E, INTER>), grid, block, 0, s, a);
  else if (a.heads_each > 1) BURST_LAUNCH((norm_kernel<T, E, INTER, 4>), grid, block, 0, s, a);
  else BURST_LAUNCH((norm_kernel<T, E, INTER, 1>), grid, block, 0, s, a);
}
template <typename T, int E>
static void enqueue(const NormArgs& a, bool backward, long long blocks, hipStream_t s) {
  if (a.interleaved) enqueue<T, E, true>(a, backward, blocks, s);
  else enqueue<T, E, false>(a, backward, blocks, s);
}
static int launch(NormArgs& a, int dtype, bool backward, long long blocks, hipStream_t s) {
  constexpr long long kMost = 1 << 23;             // blocks of a launch: it can have 2^32 threads
  for (long long first = 0; first < blocks; first += kMost) {
    a.first = (int)first;
    const long long n = blocks - first < kMost ? blocks - first : kMost;
    if (dtype == BURST_BF16) {
      if (a.granule == 8) enqueue<bf16, 8>(a, backward, n, s);
      else if (a.granule == 4) enqueue<bf16, 4>(a, backward, n, s);
      else enqueue<bf16, 1>(a, backward, n, s);
    } else {
      if (a.granule == 4) enqueue<float, 4>(a, backward, n, s);
      else enqueue<float, 1>(a, backward, n, s);
    }
    const int e = launch_status();
    if (e != BURST_OK) return e;
  }
  return BURST_OK;
}
int launch_norm(NormArgs& a, int dtype, long long blocks, hipStream_t s) { return launch(a, dtype, false, blocks, s); }
int launch_norm_bwd(NormArgs& a, int dtype, long long blocks, hipStream_t s) { return launch(a, dtype, true, blocks, s); }
int launch_norm_sums(const NormSums& a, int weights, hipStream_t s) {
  const dim3 grid((unsigned)weights, (unsigned)((a.d + 31) / 32)), block(1024);
  BURST_LAUNCH(norm_sums_kernel, grid, block, 0, s, a);
  return launch_status();
}

}  // namespace burst
