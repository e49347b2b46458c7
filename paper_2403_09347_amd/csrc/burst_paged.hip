// Attention of new tokens over a paged cache (burst_paged_fwd): O = softmax(scale Q K^T) V over the keys that a token's
// position and window leave, K and V in pages, with the running maximum and sum of burst_local_fwd and nothing but
// O and lse stored.
//
// Two kinds of kernels, one of them a call.  paged_short_kernel: one wavefront and 16 rows (tokens x the heads of a group) at a time, every
// wavefront with a stream of K and V tiles of its own through LDS: single tokens, where reading the cache is the work (HBM).
// paged_chunk_kernel (bf16) and paged_chunk_f32_kernel, calls with longer sequences: 128 rows and four wavefronts that share the tiles, bound by
// the matrix and vector units.
// Either way the work is a sequence of units (32 or 64 keys of 16 or 128 rows, see burst_paged.h) that is cut into runs of equal length,
// as many as the chip holds at once, whatever the lengths of the sequences are: the arrays that say so are on the device, and a
// captured call is replayed with others.  Where a run ends inside an item, the item's partial results go to the workspace
// and paged_merge_kernel joins them, in their order: no atomics, the same bits every time.
#include "burst_paged_kernels.h"

namespace burst {

// Lanes' values of the four groups of 16 lanes, combined: every lane gets the result of the lanes equal to it modulo 16.
__device__ __forceinline__ float max_over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
__device__ __forceinline__ bool is_zero(float x) { return (__builtin_bit_cast(unsigned, x) << 1) == 0; }

// An item's row: its token and query head, if it has one.
struct ItemRow { bool there; int token, head; };
__device__ __forceinline__ ItemRow item_row(const PagedArgs& a, int of_heads, int block, int tokens, int r) {
  const int kvhead = of_heads / a.parts_each, part = of_heads - kvhead * a.parts_each;
  const int t = r / a.part_heads, j = part * a.part_heads + r - t * a.part_heads;
  ItemRow x;
  x.token = block * a.w.tokens + t;
  x.head = kvhead * a.group + j;
  x.there = t < a.w.tokens && x.token < tokens && j < a.group;
  return x;
}
__device__ __forceinline__ ItemRow item_row(const PagedArgs& a, const PagedSegment& g, int r) { return item_row(a, g.part, g.block, g.q.n, r); }
// The keys [lo, hi] that a token sees
struct KeyRange { int lo, hi; };
__device__ __forceinline__ KeyRange seen_keys(const PagedWork& w, const PagedSeq& q, int token) {
  const int pos = q.at + token;
  KeyRange k = {0, w.causal ? min(pos, q.len - 1) : q.len - 1};
  if (w.window > 0) k.lo = max(0, pos - w.window + 1);
  return k;
}

// A finished row (m in natural units, l, and its columns by `each`): the output and lse, or its partial result.
struct RowPlace {
  bool whole;
  float* part; float* ml;            // partial: columns; m and l
  size_t o;                          // element offset in O
  size_t lse;
};
__device__ __forceinline__ RowPlace row_place(const PagedArgs& a, const PagedSegment& g, int run, int rows_of_item, int r, const ItemRow& x) {
  RowPlace p;
  p.whole = g.whole();
  float* const base = a.part + (size_t)partial_slot(g, run) * rows_of_item * (a.d + 2);
  p.part = base + (size_t)r * a.d;
  p.ml = base + (size_t)rows_of_item * a.d + r;
  p.o = (size_t)(g.q.first + x.token) * a.o_row + (size_t)x.head * a.o_head;
  p.lse = (size_t)(g.q.first + x.token) * a.heads + x.head;
  return p;
}
__device__ __forceinline__ void store4(const PagedArgs& a, size_t at, const f32x4& v) {
  if (a.o_f32) {
    *reinterpret_cast<f32x4*>((float*)a.O + at) = v;
  } else {
    bf16x4 h;
#pragma unroll
    for (int k = 0; k < 4; k++) h[k] = (bf16)v[k];
    *reinterpret_cast<bf16x4*>((bf16*)a.O + at) = h;
  }
}
__device__ __forceinline__ void store1(const PagedArgs& a, size_t at, float v) {
  if (a.o_f32) ((float*)a.O)[at] = v;
  else ((bf16*)a.O)[at] = (bf16)v;
}
__device__ __forceinline__ float row_lse(float m, float l) { return is_zero(l) ? BURST_NEG_INF : m + __logf(l); }

// Rows whose accumulators came out infinite or NaN, by themselves with scalar products of the visible pairs only: a matrix product
// multiplies hidden pairs too (by a probability of 0, and 0 x inf is NaN).  One wavefront, one row at a time: 512 tokens over 8192 keys, 32 heads
// over 8, take 0.12 ms, 33 with an infinity that 8 x 512 rows see.  (Loads of 16 bytes and eight keys' at a time made that 21, and every
// call of the chunk kernel 1 % longer, which spilled more scalar registers.)
template <typename T>
__device__ __forceinline__ void row_again(const PagedArgs& a, const PagedSegment& g, int s_of, int run, int rows_of_item, int r, int lane) {
  const ItemRow x = item_row(a, g, r);
  if (!x.there) return;
  const int d = a.d, kvhead = g.part / a.parts_each;
  const T* const q = (const T*)a.Q + (size_t)(g.q.first + x.token) * a.q_row + (size_t)x.head * a.q_head;
  KeyRange k = seen_keys(a.w, g.q, x.token);
  k.lo = max(k.lo, g.from << a.w.unit_shift);
  k.hi = min(k.hi, (g.to << a.w.unit_shift) - 1);
  float m = BURST_NEG_INF, l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 1
  for (int k0 = k.lo; k0 <= k.hi; k0 += 64) {
    const int key = k0 + lane;
    int page = -1;
    if (key <= k.hi) page = checked_page(a.table[(long long)s_of * a.table_stride + (key >> a.page_shift)], a.pages);
    const bool seen = page >= 0;
    const long long row = (long long)page * a.p_page + (long long)kvhead * a.p_head + (long long)(key & ((1 << a.page_shift) - 1)) * a.p_row;
    float s = 0.f;
    if (seen) {
      const T* const kr = (const T*)a.K + row;
#pragma unroll 1
      for (int c = 0; c < d; c++) s = __builtin_fmaf((float)q[c], (float)kr[c], s);
      s = product(s, a.scale);
    } else {
      s = BURST_NEG_INF;
    }
    float mx = s;
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    const float to = fmaxf(m, mx), ref = to == BURST_NEG_INF ? 0.f : to, alpha = fast_exp2((m - ref) * kLog2e);
    const float p = seen ? fast_exp2((s - ref) * kLog2e) : 0.f;
    m = to;
    float sum = p;
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    l = l * alpha + sum;
    o0 *= alpha; o1 *= alpha;
    unsigned long long left = __builtin_amdgcn_ballot_w64(seen);
    const int row_lo = (int)row, row_hi = (int)(row >> 32);
#pragma unroll 1
    while (left != 0) {
      const int j = __builtin_ctzll(left);
      left &= left - 1;
      const float pj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), j));
      const long long at = (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane(row_hi, j) << 32) |
                                       (unsigned)__builtin_amdgcn_readlane(row_lo, j));
      const T* const vr = (const T*)a.V + at;
      if (lane < d) o0 = __builtin_fmaf(pj, (float)vr[lane], o0);
      if (lane + 64 < d) o1 = __builtin_fmaf(pj, (float)vr[lane + 64], o1);
    }
  }
  const RowPlace at = row_place(a, g, run, rows_of_item, r, x);
  const float inv = is_zero(l) ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const int c = lane + 64 * j;
    if (c >= d) continue;
    const float v = j ? o1 : o0;
    if (at.whole) store1(a, at.o + c, is_zero(l) ? 0.f : v * inv);
    else at.part[c] = v;
  }
  if (lane == 0) {
    if (at.whole) a.lse[at.lse] = row_lse(m, l);
    else { at.ml[0] = m; at.ml[rows_of_item] = l; }
  }
}

// Operands from LDS byte addresses (see lds_read_b128 and lds_read_tr).
__device__ __forceinline__ bf16x8 lds_b128(unsigned at) { return *(const bf16x8 __attribute__((address_space(3)))*)(size_t)at; }
__device__ __forceinline__ bf16x4 lds_tr(unsigned at) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(size_t)at));
}
// Keeps the compiler's scheduler from moving anything across.
#define BURST_FENCE() __builtin_amdgcn_sched_barrier(0)

// vmcnt(N), the other counters untouched; nothing moves across it
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// ------------------------------------------------------------------------------- short
// Groups of up to 16 heads: an item's part is its key/value head.
// S^T = K Q^T of 16 keys x 16 rows: lane (r = lane % 16, g = lane / 16) gets row r, keys 4g .. 4g + 3, which is also how the second
// product, O^T += V^T P^T, wants P.  The order of the summed columns is free, so a lane's operands are 16-byte pieces of a row of K or
// Q: granule 4 ks + g in step ks.  A stage is 16 keys, K and V, brought to LDS by DMA (rows beyond the sequence arrive as
// zeros) in a ring of stages that runs on across the items of the run; a wavefront waits for its own loads alone, there are no barriers.
// LDS rows of 8, 16 or 32 granules, permuted so that 16 rows of one granule column fall into different banks.
// Measured (32 query heads over 8, d = 128, us and the cache's bytes a second): 64 single tokens over 16 to 16384 keys each, 645 MB, 126 (5.1
// TB/s); one over 32768 keys, 134 MB, 37 (3.6 TB/s; 7 of them joining); 32 over 2000 keys, 32 heads of
// their own, 1.05 GB, 184 (5.7 TB/s).  A device copy reads and writes 5.0 TB/s.
template <int GR>
__device__ __forceinline__ int short_code(int row) { return GR == 8 ? (row >> 1) & 7 : row_code(row & 15); }

template <typename T, int D>
__global__ void __launch_bounds__(64, 1)
paged_short_kernel(PagedArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int ROWB = D * (int)sizeof(T), GR = ROWB / 16, TILE = 16 * ROWB;
  constexpr int NST = kShortLds / (2 * TILE);      // stages
  constexpr int RPL = 1024 / ROWB, NL = TILE / 1024, LOADS = 2 * NL;   // rows of a load; loads of K, of a stage
  constexpr int KS = GR / 4;                       // granule steps of a product over d
  constexpr int OB = D / 16;                       // 16-column blocks of O^T
  constexpr int NSEG = 16;                         // segments on their way: at most one a stage, and the one at work
  static_assert(NST >= 2 && NST < NSEG && (NST - 1) * LOADS < 64, "the ring fits LDS and the counter of loads");
  __shared__ __attribute__((aligned(16))) char smem[NST * 2 * TILE];
  __shared__ i32x4 segs[NSEG][3];
  const int lane = threadIdx.x, r = lane & 15, g = lane >> 4;
  int run;
  DeviceCursor fet;
  if (!start_run(a, blockIdx.x, lane, lane == 0, fet, run)) return;
  const unsigned lds0 = lds_addr(smem);
  const int d = a.d;
  const unsigned pitch = (unsigned)(a.p_row * sizeof(T)), row_bytes = (unsigned)(d * sizeof(T));
  const long long v_off = (const char*)a.V - (const char*)a.K;

  int goff[NL];
#pragma unroll
  for (int i = 0; i < NL; i++) {
    const int row = i * RPL + lane / GR, granule = (lane % GR) ^ short_code<GR>(row);
    goff[i] = granule * (16 / (int)sizeof(T)) < d ? row * (int)pitch + granule * 16 : (int)0x80000000u;
  }
  // The fetching side: stages [f_at, f_end) of fet.g are still to be asked for; the lanes hold the places of the 64 stages from f_base on.
  int f_at, f_end, f_base, seg_in = 0;
  int where_lo, where_hi;
  unsigned long long pages = 0;                    // those of the 64 that have a page
  auto look_up = [&]() __attribute__((always_inline)) {
    const PagedArgs& b = args_again<PagedArgs>();
    const int key = (f_at + lane) << 4, entry = table_entry(key, fet.g.q.len, b.page_shift);
    int page = -1;
    if (entry >= 0) page = checked_page(b.table[(long long)fet.s * b.table_stride + entry], b.pages);
    const long long at = (long long)max(page, 0) * b.p_page + (long long)fet.g.part * b.p_head +
                         (long long)(key & ((1 << b.page_shift) - 1)) * b.p_row;
    const long long where = (long long)(size_t)b.K + at * (long long)sizeof(T);
    where_lo = (int)where; where_hi = (int)(where >> 32);
    pages = __builtin_amdgcn_ballot_w64(page >= 0);
    f_base = f_at;
  };
  auto enter = [&]() __attribute__((always_inline)) {
    segment_tiles(args_again<PagedArgs>().w, fet.g, 4, f_at, f_end);
    if (lane == 0) {
      i32x4* const to = segs[seg_in % NSEG];
      to[0] = i32x4{fet.g.q.first, fet.g.q.n, fet.g.q.len, fet.g.part};
      to[1] = i32x4{fet.g.block, fet.g.from, fet.g.to, fet.s};
      to[2] = i32x4{f_at, f_end, fet.g.q.at, (fet.g.whole() ? 1 : 0) | (fet.g.from == fet.g.lo ? 2 : 0)};
    }
    seg_in++;
    look_up();
  };
  enter();
  unsigned gone = 0;                               // stages of the ring without a page
  int f_slot = 0, ahead = 0;                       // slot that is filled next; stages asked for and not yet used
  bool more = true;

  // addresses of the operands in a tile
  int kaddr[KS], vaddr[F32 ? GR / 16 : OB];
#pragma unroll
  for (int ks = 0; ks < KS; ks++) kaddr[ks] = r * ROWB + (((4 * ks + g) ^ short_code<GR>(r)) << 4);
  if constexpr (!F32) {                            // transposing reads: keys 4g .. 4g + 3, columns 16 ob .. 16 ob + 15
    const int row = 4 * g + (r >> 2);
#pragma unroll
    for (int ob = 0; ob < OB; ob++) vaddr[ob] = row * ROWB + (((2 * ob + ((r & 3) >> 1)) ^ short_code<GR>(row)) << 4) + (r & 1) * 8;
  }
  // The segment at work
  PagedSegment s = {};
  int seg_s = 0, seg_out = 0, st = 0, end = 0, slot = 0;
  ItemRow x = {};
  KeyRange see = {}, all = {};                     // keys of the lane's row; keys that every row sees
  i32x4 q[KS];
  f32x4 o[OB];
  float m = BURST_NEG_INF, l = 0.f;                // the row's reference (natural units); its sum over this lane's keys
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    while (ahead < NST && more) {                  // (one stage a turn once the ring is full)
      if (f_at == f_end) {
        if (!fet.next(args_again<PagedArgs>().w)) { more = false; break; }
        enter();
      } else if (f_at - f_base == 64) {
        look_up();
      }
      const int i = f_at - f_base;
      const bool ok = ((pages >> i) & 1) != 0;
      const int rows = ok ? min(16, fet.g.q.len - (f_at << 4)) : 0;
      const unsigned span = rows > 0 ? (unsigned)(rows - 1) * pitch + row_bytes : 0u;
      const long long at = (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane(where_hi, i) << 32) |
                                       (unsigned)__builtin_amdgcn_readlane(where_lo, i));
      const __amdgpu_buffer_rsrc_t krs = make_rsrc((const void*)at, span), vrs = make_rsrc((const void*)(at + v_off), span);
      const unsigned to = lds0 + (unsigned)f_slot * (2 * TILE);
#pragma unroll
      for (int k = 0; k < NL; k++) dma_b128_to_lds(krs, to + k * 1024u, goff[k]);
#pragma unroll
      for (int k = 0; k < NL; k++) dma_b128_to_lds(vrs, to + TILE + k * 1024u, goff[k]);
      gone = ok ? gone & ~(1u << f_slot) : gone | (1u << f_slot);
      f_slot = f_slot + 1 == NST ? 0 : f_slot + 1;
      ahead++;
      f_at++;
    }
    if (ahead == 0) break;
    if (st == end) {                               // the next segment
      const PagedArgs& b = args_again<PagedArgs>();
      const i32x4 *const from = segs[seg_out % NSEG], d0 = from[0], d1 = from[1], d2 = from[2];
      auto one = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
      seg_out++;
      s.q = PagedSeq{one(d0[0]), one(d0[1]), one(d0[2]), one(d2[2])};
      s.part = one(d0[3]); s.block = one(d1[0]); s.from = one(d1[1]); s.to = one(d1[2]);
      seg_s = one(d1[3]);
      st = one(d2[0]); end = one(d2[1]);
      s.lo = one(d2[3]) & 2 ? s.from : s.from - 1; // (as far as whole() and partial_slot() look at them)
      s.hi = one(d2[3]) & 1 ? s.to : s.to + 1;
      x = item_row(b, s, r);
      see = seen_keys(b.w, s.q, x.token);
      const T* const qr = (const T*)b.Q + (size_t)(s.q.first + (x.there ? x.token : 0)) * b.q_row + (size_t)(x.there ? x.head : 0) * b.q_head;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const int c = (4 * ks + g) * (16 / (int)sizeof(T));
        q[ks] = x.there && c < d ? *reinterpret_cast<const i32x4*>(qr + c) : i32x4{0, 0, 0, 0};
      }
      // (Waited for here, once a segment: the compiler, which does not know of the loads in flight, would wait for all of them
      // before the first product of every stage.)
#pragma unroll
      for (int ks = 0; ks < KS; ks++) asm volatile("" : "+v"(q[ks]));
#pragma unroll
      for (int b = 0; b < OB; b++) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      m = BURST_NEG_INF; l = 0.f;
      const int t0 = s.block * b.w.tokens, t1 = min(s.q.n, t0 + b.w.tokens) - 1;
      all = KeyRange{seen_keys(b.w, s.q, t1).lo, seen_keys(b.w, s.q, t0).hi};
    }
    if (ahead == NST) wait_loads<(NST - 1) * LOADS>();
    else wait_loads<0>();
    const char* const kl = smem + slot * (2 * TILE);
    const char* const vl = kl + TILE;
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      const i32x4 k = *reinterpret_cast<const i32x4*>(kl + kaddr[ks]);
      if constexpr (F32) {
        const f32x4 kf = __builtin_bit_cast(f32x4, k), qf = __builtin_bit_cast(f32x4, q[ks]);
#pragma unroll
        for (int j = 0; j < 4; j++) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j], qf[j], sc, 0, 0, 0);
      } else {
        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[ks]), sc, 0, 0, 0);
      }
    }
    const int key0 = st << 4;
    const bool none = ((gone >> slot) & 1) != 0;
#pragma unroll
    for (int j = 0; j < 4; j++) sc[j] = product(sc[j], a.scale);
    if (none || key0 < all.lo || key0 + 15 > all.hi) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int key = key0 + 4 * g + j;
        if (none || key < see.lo || key > see.hi) sc[j] = BURST_NEG_INF;
      }
    }
    const float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
    // A row's first reference, or one that has been exceeded by more than a factor of e^8 (l stays far from its range's end).
    if (__builtin_amdgcn_ballot_w64(mx > m + 8.f) != 0) {
      const float to = fmaxf(m, max_over_groups(mx)), alpha = fast_exp2((m - (to == BURST_NEG_INF ? 0.f : to)) * kLog2e);
      m = to;
      l *= alpha;
#pragma unroll
      for (int b = 0; b < OB; b++) o[b] *= alpha;
    }
    const float ref = m == BURST_NEG_INF ? 0.f : m;
    float p[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      p[j] = fast_exp2((sc[j] - ref) * kLog2e);
      l += p[j];
    }
    if constexpr (F32) {                           // block 4 half + c: columns 64 half + 4 (lane % 16) + c of V
#pragma unroll
      for (int j = 0; j < 4; j++)
#pragma unroll
        for (int half = 0; half < GR / 16; half++) {
          const int row = 4 * g + j;
          const f32x4 v = *reinterpret_cast<const f32x4*>(vl + row * ROWB + (((r + 16 * half) ^ short_code<GR>(row)) << 4));
#pragma unroll
          for (int c = 0; c < 4; c++) o[4 * half + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[c], p[j], o[4 * half + c], 0, 0, 0);
        }
    } else {                                       // P in two terms, 16 bits of it: the second products are not what bounds these calls
      bf16x4 p0, p1;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        p0[j] = (bf16)p[j];
        p1[j] = (bf16)(p[j] - (float)p0[j]);
      }
      s16x4 v[OB];
#pragma unroll
      for (int b = 0; b < OB; b++) v[b] = __builtin_bit_cast(s16x4, lds_read_tr(vl, vaddr[b]));
#pragma unroll
      for (int b = 0; b < OB; b++) o[b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[b], __builtin_bit_cast(s16x4, p1), o[b], 0, 0, 0);
#pragma unroll
      for (int b = 0; b < OB; b++) o[b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[b], __builtin_bit_cast(s16x4, p0), o[b], 0, 0, 0);
    }
    wait_lds();                                    // (the tile has been read: its slot is filled again)
    ahead--;
    slot = slot + 1 == NST ? 0 : slot + 1;
    if (++st < end) continue;

    const PagedArgs& b = args_again<PagedArgs>();
    l = sum_over_groups(l);
    unsigned most = larger_of(0, l);
#pragma unroll
    for (int k = 0; k < OB; k++)
#pragma unroll
      for (int j = 0; j < 4; j++) most = larger_of(most, o[k][j]);
    const unsigned long long bal = __builtin_amdgcn_ballot_w64(x.there && most >= kInfBits);
    unsigned redo = (unsigned)(bal | (bal >> 16) | (bal >> 32) | (bal >> 48)) & 0xffffu;
    if (x.there && !((redo >> r) & 1)) {
      const RowPlace at = row_place(b, s, run, kShortRows, r, x);
      const float inv = is_zero(l) ? 0.f : 1.f / l;
#pragma unroll
      for (int k = 0; k < OB; k++) {
        f32x4 v;
        int c;
        if constexpr (F32) {                       // row 4g + j of block 4 half + i holds column 64 half + 16 g + 4 j + i
          const int half = k >> 2, j = k & 3;
          c = 64 * half + 16 * g + 4 * j;
          v = f32x4{o[4 * half][j], o[4 * half + 1][j], o[4 * half + 2][j], o[4 * half + 3][j]};
        } else {
          c = 16 * k + 4 * g;
          v = o[k];
        }
        if (c >= d) continue;
        if (at.whole) store4(b, at.o + c, v * inv);
        else *reinterpret_cast<f32x4*>(at.part + c) = v;
      }
      if (g == 0) {
        if (at.whole) b.lse[at.lse] = row_lse(m, l);
        else { at.ml[0] = m; at.ml[kShortRows] = l; }
      }
    }
    for (; redo != 0; redo &= redo - 1) row_again<T>(b, s, seg_s, run, kShortRows, __builtin_ctz(redo), lane);
  }
}

// ------------------------------------------------------------------------------- chunk
// Four wavefronts of 32 rows each share K and V tiles, double-buffered in LDS (DMA, one barrier a tile).  Two workgroups a CU, so that one's
// vector work overlaps the other's matrix work.
// The fetching side, a tile of 1 << SHIFT keys ahead: tiles [f_at, f_end) of fet.g are still to be asked for.  A wavefront fetches a quarter of
// every tile, whose keys lie in one page; the lanes hold the places of the 64 groups of 16 keys from tile f_base on.
template <typename T, int D, int SHIFT>
struct TileFeed {
  static constexpr int ROWB = D * (int)sizeof(T), GR = ROWB / 16, TILE = ROWB << SHIFT;   // LDS bytes and granules of a row; bytes of a tile
  static constexpr int GROUPS = (1 << SHIFT) / 16, ROWS = (1 << SHIFT) / 4;               // of 16 keys in a tile; keys of a wavefront's quarter
  static constexpr int RPL = 1024 / ROWB, NL = ROWS / RPL;                                // rows of a load; loads
  static __device__ __forceinline__ int code(int row) { return short_code<GR>(row); }
  DeviceCursor fet;
  int w, lane;
  int f_first, f_at, f_end, f_base, where_lo, where_hi, goff[NL];
  unsigned long long pages;          // those of the 64 groups that have a page
  long long v_off;
  unsigned lds0, pitch, row_bytes;
  unsigned gone;                     // GROUPS bits a buffer: groups without a page
  bool more;                         // fet.g is the segment of the tile that was asked for last
  __device__ __forceinline__ int group() const { return w * ROWS / 16; }
  __device__ __forceinline__ int first_row() const { return w * ROWS % 16; }
  __device__ __forceinline__ bool start(const PagedArgs& a, int& run, const char* smem) {
    lane = threadIdx.x & 63;
    w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!start_run(a, blockIdx.x, lane, threadIdx.x == 0, fet, run)) return false;
    lds0 = lds_addr(smem) + (unsigned)(w * NL) * 1024u;
    pitch = (unsigned)(a.p_row * (int)sizeof(T)); row_bytes = (unsigned)(a.d * (int)sizeof(T));
    v_off = (const char*)a.V - (const char*)a.K;
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int row = i * RPL + lane / GR, granule = (lane % GR) ^ code(first_row() + row);
      goff[i] = granule * (16 / (int)sizeof(T)) < a.d ? row * (int)pitch + granule * 16 : (int)0x80000000u;
    }
    gone = 0;
    more = true;
    enter();
    fetch(0);
    return true;
  }
  __device__ __forceinline__ void look_up() {
    const PagedArgs& b = args_again<PagedArgs>();
    const int key = (f_at << SHIFT) + 16 * lane, entry = table_entry(key, fet.g.q.len, b.page_shift);
    int page = -1;
    if (entry >= 0) page = checked_page(b.table[(long long)fet.s * b.table_stride + entry], b.pages);
    const long long at = (long long)max(page, 0) * b.p_page + (long long)((unsigned)fet.g.part / (unsigned)b.parts_each) * b.p_head +
                         (long long)((key & ((1 << b.page_shift) - 1)) + first_row()) * b.p_row;
    const long long where = (long long)(size_t)b.K + at * (long long)sizeof(T);
    where_lo = (int)where; where_hi = (int)(where >> 32);
    pages = __builtin_amdgcn_ballot_w64(page >= 0);
    f_base = f_at;
  }
  __device__ __forceinline__ void enter() {
    segment_tiles(args_again<PagedArgs>().w, fet.g, SHIFT, f_at, f_end);
    f_first = f_at;
    look_up();
  }
  // asks for the next tile, if the run has one (`more`); K goes to buffer buf, V two tiles behind it
  __device__ __forceinline__ void fetch(int buf) {
    if (f_at == f_end) {
      if (!more || !fet.next(args_again<PagedArgs>().w)) { more = false; return; }
      enter();
    } else if (f_at - f_base == 64 / GROUPS) {
      look_up();
    }
    constexpr unsigned ALL = (1u << GROUPS) - 1;
    const int t = GROUPS * (f_at - f_base);
    const unsigned here = (unsigned)(pages >> t) & ALL;
    const int rows = (here >> group()) & 1 ? __builtin_amdgcn_readfirstlane(min(ROWS, fet.g.q.len - (f_at << SHIFT) - w * ROWS)) : 0;
    const unsigned span = rows > 0 ? (unsigned)(rows - 1) * pitch + row_bytes : 0u;
    const long long at = (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane(where_hi, t + group()) << 32) |
                                     (unsigned)__builtin_amdgcn_readlane(where_lo, t + group()));
    const __amdgpu_buffer_rsrc_t krs = make_rsrc((const void*)at, span), vrs = make_rsrc((const void*)(at + v_off), span);
    const unsigned to = lds0 + (unsigned)buf * TILE;
#pragma unroll
    for (int i = 0; i < NL; i++) {
      dma_b128_to_lds(krs, to + i * 1024u, goff[i]);
      dma_b128_to_lds(vrs, to + 2 * TILE + i * 1024u, goff[i]);
    }
    gone = (gone & ~(ALL << (GROUPS * buf))) | ((here ^ ALL) << (GROUPS * buf));
    f_at++;
  }
  __device__ __forceinline__ unsigned missing(int buf) const { return (gone >> (GROUPS * buf)) & ((1u << GROUPS) - 1); }
};

// bf16: tiles of 64 keys, operand orientation and LDS layout as in burst_plain_mfma.h: S^T = K Q^T with a row per lane, whose P is the operand
// of O^T += V^T P^T as it stands.
// Scores and references are in log2 units (one fma an exponent), as in the d = 64 and d = 128 kernels of the walks.
// Measured: 2048 tokens over 32768 keys, 32 heads over 8, d = 128, 1025 to 1115 us (0.95 to 1.04 PFLOP/s, cards differ; a large library product 1.14);
// 4096 tokens of 8192, d = 64, twice, 526 to 550 us (0.75 to 0.78).  At d = 64 a tile's products are 512 cycles of a wavefront and its vector instructions about
// 900, which two wavefronts a SIMD overlap in part.  (Four buffers instead of two at d = 64: 535 / 526 at that size, the others within 1 %.)
constexpr int kTile = 1 << kTileShift;             // keys
// C: columns that are computed, of the D that a row of LDS has.
// TERMS: bf16 terms that P goes into the second product in.  One (8 bits) at d = 64 and d = 128, as in the walks there, unless the caller asks for
// full_p; two (16 bits) otherwise.  O is then 2.35e-3 of its norm off 64 bits, or 1.66e-3, which is what rounding O to bf16 does alone, at
// any number of keys (both the errors and O go with the root of the sum of p^2).  us with one / two: 2048 tokens over 32768 keys, 32 heads over
// 8, d = 128, 1100 / 1470; 4096 of 8192, d = 64, twice, 544 / 697; 12 sequences of 1 to 512 over 600 to 8000 167 / 173; a window of 1024,
// d = 64, 36.3 / 41.2; 16 x 8 tokens over 8192 113.5 / 114.7; two prompts of 4096 of 8192, 32 heads over 8, at d = 32 433 / 508, d = 80 674 / 879, d = 96
// 698 / 915, d = 104 799 / 1061.
template <int D, int C, int TERMS>
__global__ void __launch_bounds__(256, 2)
paged_chunk_kernel(PagedArgs a) {
  typedef TileFeed<bf16, D, kTileShift> Feed;
  constexpr int ROWB = Feed::ROWB, TILE = Feed::TILE, KS = C / 16, DB = C / 32, AHEAD = 4;
  __shared__ __attribute__((aligned(16))) char smem[4 * TILE];   // K[2], V[2]
  int run;
  Feed f;
  if (!f.start(a, run, smem)) return;
  const int lane = f.lane, lr = lane & 31, h = lane >> 5, w = f.w, d = a.d;

  const unsigned base = lds_addr(smem);
  unsigned kaddr[KS], taddr[DB][2];                // of buffer 0
#pragma unroll
  for (int ks = 0; ks < KS; ks++) kaddr[ks] = base + lr * ROWB + (((2 * ks + h) ^ Feed::code(lr)) << 4);
#pragma unroll
  for (int db = 0; db < DB; db++)
#pragma unroll
    for (int sx = 0; sx < 2; sx++) {
      const int j16 = lane & 15, row = 8 * sx + 4 * h + (j16 >> 2), granule = db * 4 + 2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1);
      taddr[db][sx] = base + 2 * TILE + row * ROWB + ((granule ^ Feed::code(row)) << 4) + (j16 & 1) * 8;
    }
  const float c = a.scale * kLog2e;
  unsigned c1 = 0x0000bf80u, c2 = 0xbf800000u;     // (-1, 0) and (0, -1), in registers: x - bf16(x) is one dot product, exact
  asm("" : "+s"(c1), "+s"(c2));
  const bf16x2 minus_first = __builtin_bit_cast(bf16x2, c1), minus_second = __builtin_bit_cast(bf16x2, c2);
  int buf = 0;
#pragma unroll 1
  do {
    const PagedSegment s = f.fet.g;
    const int seg_s = f.fet.s, end = f.f_end;
    int at = f.f_first;
    const PagedArgs& b = args_again<PagedArgs>();
    const ItemRow x = item_row(b, s, 32 * w + lr);
    const KeyRange see = seen_keys(b.w, s.q, x.token);
    bf16x8 q[KS];
    {
      const bf16* const qr = (const bf16*)b.Q + (size_t)(s.q.first + (x.there ? x.token : 0)) * b.q_row + (size_t)(x.there ? x.head : 0) * b.q_head;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const int col = 16 * ks + 8 * h;
        const i32x4 v = x.there && col < d ? *reinterpret_cast<const i32x4*>(qr + col) : i32x4{0, 0, 0, 0};
        q[ks] = __builtin_bit_cast(bf16x8, v);
      }
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; db++)
#pragma unroll
      for (int r = 0; r < 16; r++) o[db][r] = 0.f;
    float m = BURST_NEG_INF, l = 0.f;              // reference (log2 units); the row's sum over this lane's keys
    // tokens of the wavefront's rows: what all of them see, and what any of them does
    const int most = min(b.w.tokens, s.q.n - s.block * b.w.tokens) - 1;
    const int t0 = s.block * b.w.tokens + 32 * w / b.part_heads, t1 = s.block * b.w.tokens + min((32 * w + 31) / b.part_heads, most);
    const bool rows_here = 32 * w / b.part_heads <= most;
    const KeyRange first = seen_keys(b.w, s.q, t0), last = seen_keys(b.w, s.q, t1);
#pragma unroll 1
    for (; at < end; at++, buf ^= 1) {
      __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0), lgkmcnt(0): the tile landed, reads of the one before are done
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const unsigned none = f.missing(buf);
      f.fetch(buf ^ 1);
      const int key0 = at << kTileShift;
      if (!rows_here || key0 > last.hi || key0 + kTile - 1 < first.lo) continue;   // none of the wavefront's rows sees the tile
      const unsigned tile = (unsigned)buf * TILE;
      f32x16 sc[2];
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int r = 0; r < 16; r++) sc[kb][r] = 0.f;
      // Operands are read AHEAD products before their own.  (Left alone the compiler reads each of them right before its product and
      // waits for it.)
      {
        bf16x8 k[2 * KS];
        auto read = [&](int i) __attribute__((always_inline)) { k[i] = lds_b128(kaddr[i >> 1] + tile + (i & 1) * 32 * ROWB); };
#pragma unroll
        for (int i = 0; i < AHEAD; i++) read(i);
        BURST_FENCE();
#pragma unroll
        for (int i = 0; i < 2 * KS; i++) {
          sc[i & 1] = mfma32(k[i], q[i >> 1], sc[i & 1]);
          if (i + AHEAD < 2 * KS) read(i + AHEAD);
          BURST_FENCE();
        }
      }
      if (none != 0 || key0 < last.lo || key0 + kTile - 1 > first.hi) {   // register r of block kb: key 32 kb + 8 (r / 4) + 4 h + r % 4
        const int lo = see.lo - key0 - 4 * h, hi = see.hi - key0 - 4 * h;
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
          for (int r = 0; r < 16; r++) {
            const int k = kb * 32 + 8 * (r >> 2) + (r & 3);
            if (k < lo || k > hi || ((none >> (2 * kb + (r >> 3))) & 1)) sc[kb][r] = BURST_NEG_INF;
          }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int r = 0; r < 16; r++) mx = fmaxf(mx, sc[kb][r]);
      mx *= c;
      if (__builtin_amdgcn_ballot_w64(mx > m + 8.f) != 0) {   // a row's first reference, or one exceeded by more than 2^8
        const float to = fmaxf(m, max_both_halves(mx)), alpha = fast_exp2(m - (to == BURST_NEG_INF ? 0.f : to));
        m = to;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
          for (int r = 0; r < 16; r++) o[db][r] *= alpha;
      }
      const float nref = m == BURST_NEG_INF ? 0.f : -m;
      // P of the next 16 keys is computed between the products of these, which add the smaller term first.
      bf16x8 p[4][TERMS], v[4 * DB];
      auto read = [&](int i) __attribute__((always_inline)) {
        const unsigned at = tile + (i / DB) * 16 * ROWB;
        v[i] = __builtin_shufflevector(lds_tr(taddr[i % DB][0] + at), lds_tr(taddr[i % DB][1] + at), 0, 1, 2, 3, 4, 5, 6, 7);
      };
      auto prob = [&](int kg, int t) __attribute__((always_inline)) {   // keys t and t + 1
        const float x = fast_exp2(__builtin_fmaf(sc[kg >> 1][8 * (kg & 1) + t], c, nref));
        const float y = fast_exp2(__builtin_fmaf(sc[kg >> 1][8 * (kg & 1) + t + 1], c, nref));
        l += x + y;                                // (unrounded: lse has 24 bits)
        bf16x2 pk;
        pk[0] = (bf16)x; pk[1] = (bf16)y;
        p[kg][0][t] = pk[0]; p[kg][0][t + 1] = pk[1];
        if constexpr (TERMS == 2) {
          p[kg][1][t] = (bf16)__builtin_amdgcn_fdot2_f32_bf16(pk, minus_first, x, false);
          p[kg][1][t + 1] = (bf16)__builtin_amdgcn_fdot2_f32_bf16(pk, minus_second, y, false);
        }
      };
#pragma unroll
      for (int i = 0; i < AHEAD; i++) read(i);
#pragma unroll
      for (int t = 0; t < 8; t += 2) prob(0, t);
      BURST_FENCE();
#pragma unroll
      for (int kg = 0; kg < 4; kg++)
#pragma unroll
        for (int term = TERMS - 1; term >= 0; term--)
#pragma unroll
          for (int db = 0; db < DB; db++) {
            const int i = kg * DB + db, at = (TERMS - 1 - term) * DB + db;
            o[db] = mfma32(v[i], p[kg][term], o[db]);
            if (term == 0 && i + AHEAD < 4 * DB) read(i + AHEAD);
            if (kg < 3)
#pragma unroll
              for (int t = 0; t < 4; t++)
                if (t * TERMS * DB / 4 == at) prob(kg + 1, 2 * t);
            BURST_FENCE();
          }
    }
    l = sum_both_halves(l);
    unsigned big = larger_of(0, l);
#pragma unroll
    for (int db = 0; db < DB; db++)
#pragma unroll
      for (int r = 0; r < 16; r++) big = larger_of(big, o[db][r]);
    const unsigned long long bal = __builtin_amdgcn_ballot_w64(x.there && big >= kInfBits);
    unsigned redo = (unsigned)(bal | (bal >> 32));
    if (x.there && !((redo >> lr) & 1)) {
      const RowPlace to = row_place(b, s, run, kChunkRows, 32 * w + lr, x);
      const float inv = is_zero(l) ? 0.f : 1.f / l;
#pragma unroll
      for (int db = 0; db < DB; db++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++) {
          const int col = db * 32 + 8 * q4 + 4 * h;
          if (col >= d) continue;
          const f32x4 v = {o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]};
          if (to.whole) store4(b, to.o + col, v * inv);
          else *reinterpret_cast<f32x4*>(to.part + col) = v;
        }
      if (h == 0) {
        const float mn = m * kLn2;
        if (to.whole) b.lse[to.lse] = row_lse(mn, l);
        else { to.ml[0] = mn; to.ml[kChunkRows] = l; }
      }
    }
    for (; redo != 0; redo &= redo - 1) row_again<bf16>(b, s, seg_s, run, kChunkRows, 32 * w + __builtin_ctz(redo), lane);
  } while (f.more);
}

// fp32: tiles of 32 keys, products as in the short kernel, two blocks of 16 rows a wavefront (each operand of K and V read from LDS serves
// both).  C: columns of the first product; the second one computes all D, whose blocks of 16 columns each hold every fourth column of 64.
// Bound by the fp32 matrix rate: 4096 tokens over themselves, causal, 8 heads, d = 128, 324 us (106 TFLOP/s; a large library product 153).
template <int D, int C>
__global__ void __launch_bounds__(256, 2)
paged_chunk_f32_kernel(PagedArgs a) {
  typedef TileFeed<float, D, kTileShiftF32> Feed;
  constexpr int ROWB = Feed::ROWB, TILE = Feed::TILE, GR = Feed::GR, KEYS = 1 << kTileShiftF32;
  constexpr int KS = C / 16, HV = GR / 16, OB = D / 16;   // granule steps of a product over d; 64-column parts; 16-column blocks of O^T
  __shared__ __attribute__((aligned(16))) char smem[4 * TILE];   // K[2], V[2]
  int run;
  Feed f;
  if (!f.start(a, run, smem)) return;
  const int lane = f.lane, r = lane & 15, g = lane >> 4, w = f.w, d = a.d;

  int kaddr[KS], vaddr[4][HV];                     // in a 16-key block of a tile
#pragma unroll
  for (int ks = 0; ks < KS; ks++) kaddr[ks] = r * ROWB + (((4 * ks + g) ^ Feed::code(r)) << 4);
#pragma unroll
  for (int j = 0; j < 4; j++)
#pragma unroll
    for (int half = 0; half < HV; half++) vaddr[j][half] = (4 * g + j) * ROWB + (((r + 16 * half) ^ Feed::code(4 * g + j)) << 4);
  int buf = 0;
#pragma unroll 1
  do {
    const PagedSegment s = f.fet.g;
    const int seg_s = f.fet.s, end = f.f_end;
    int at = f.f_first;
    const PagedArgs& b = args_again<PagedArgs>();
    ItemRow x[2];
    KeyRange see[2];
    f32x4 q[2][KS], o[2][OB];
    float m[2], l[2];                              // references (natural units); sums over this lane's keys
#pragma unroll
    for (int i = 0; i < 2; i++) {
      x[i] = item_row(b, s, 32 * w + 16 * i + r);
      see[i] = seen_keys(b.w, s.q, x[i].token);
      const float* const qr = (const float*)b.Q + (size_t)(s.q.first + (x[i].there ? x[i].token : 0)) * b.q_row + (size_t)(x[i].there ? x[i].head : 0) * b.q_head;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const int c = (4 * ks + g) * 4;
        q[i][ks] = x[i].there && c < d ? *reinterpret_cast<const f32x4*>(qr + c) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int k = 0; k < OB; k++) o[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[i] = BURST_NEG_INF; l[i] = 0.f;
    }
    const int most = min(b.w.tokens, s.q.n - s.block * b.w.tokens) - 1;
    const int t0 = s.block * b.w.tokens + 32 * w / b.part_heads, t1 = s.block * b.w.tokens + min((32 * w + 31) / b.part_heads, most);
    const bool rows_here = 32 * w / b.part_heads <= most;
    const KeyRange first = seen_keys(b.w, s.q, t0), last = seen_keys(b.w, s.q, t1);
#pragma unroll 1
    for (; at < end; at++, buf ^= 1) {
      __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0), lgkmcnt(0): the tile landed, reads of the one before are done
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const unsigned none = f.missing(buf);
      f.fetch(buf ^ 1);
      const int key0 = at * KEYS;
      if (!rows_here || key0 > last.hi || key0 + KEYS - 1 < first.lo) continue;
      const char* const kl = smem + buf * TILE;
      const char* const vl = smem + (2 + buf) * TILE;
      f32x4 sc[2][2];                              // [rows][keys]
#pragma unroll
      for (int i = 0; i < 2; i++) sc[i][0] = sc[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const f32x4 k0 = *reinterpret_cast<const f32x4*>(kl + kaddr[ks]), k1 = *reinterpret_cast<const f32x4*>(kl + 16 * ROWB + kaddr[ks]);
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int i = 0; i < 2; i++) {
            sc[i][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k0[j], q[i][ks][j], sc[i][0], 0, 0, 0);
            sc[i][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k1[j], q[i][ks][j], sc[i][1], 0, 0, 0);
          }
      }
      const bool masked = none != 0 || key0 < last.lo || key0 + KEYS - 1 > first.hi;
      bool raise = false;
      float mx[2];
#pragma unroll
      for (int i = 0; i < 2; i++) {
        mx[i] = BURST_NEG_INF;
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            float v = product(sc[i][kb][j], a.scale);
            const int key = key0 + 16 * kb + 4 * g + j;
            if (masked && (((none >> kb) & 1) != 0 || key < see[i].lo || key > see[i].hi)) v = BURST_NEG_INF;
            sc[i][kb][j] = v;
            mx[i] = fmaxf(mx[i], v);
          }
        raise |= mx[i] > m[i] + 8.f;
      }
      if (__builtin_amdgcn_ballot_w64(raise) != 0)  // see the short kernel
#pragma unroll
        for (int i = 0; i < 2; i++) {
          const float to = fmaxf(m[i], max_over_groups(mx[i])), alpha = fast_exp2((m[i] - (to == BURST_NEG_INF ? 0.f : to)) * kLog2e);
          m[i] = to;
          l[i] *= alpha;
#pragma unroll
          for (int k = 0; k < OB; k++) o[i][k] *= alpha;
        }
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const float ref = m[i] == BURST_NEG_INF ? 0.f : m[i];
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            sc[i][kb][j] = fast_exp2((sc[i][kb][j] - ref) * kLog2e);
            l[i] += sc[i][kb][j];
          }
      }
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int half = 0; half < HV; half++) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(vl + kb * 16 * ROWB + vaddr[j][half]);
#pragma unroll
            for (int c = 0; c < 4; c++)
#pragma unroll
              for (int i = 0; i < 2; i++) o[i][4 * half + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[c], sc[i][kb][j], o[i][4 * half + c], 0, 0, 0);
          }
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
      l[i] = sum_over_groups(l[i]);
      unsigned big = larger_of(0, l[i]);
#pragma unroll
      for (int k = 0; k < OB; k++)
#pragma unroll
        for (int j = 0; j < 4; j++) big = larger_of(big, o[i][k][j]);
      const unsigned long long bal = __builtin_amdgcn_ballot_w64(x[i].there && big >= kInfBits);
      unsigned redo = (unsigned)(bal | (bal >> 16) | (bal >> 32) | (bal >> 48)) & 0xffffu;
      if (x[i].there && !((redo >> r) & 1)) {
        const RowPlace to = row_place(b, s, run, kChunkRows, 32 * w + 16 * i + r, x[i]);
        const float inv = is_zero(l[i]) ? 0.f : 1.f / l[i];
#pragma unroll
        for (int half = 0; half < HV; half++)
#pragma unroll
          for (int j = 0; j < 4; j++) {            // row 4g + j of block 4 half + c holds column 64 half + 16 g + 4 j + c
            const int col = 64 * half + 16 * g + 4 * j;
            if (col >= d) continue;
            const f32x4 v = {o[i][4 * half][j], o[i][4 * half + 1][j], o[i][4 * half + 2][j], o[i][4 * half + 3][j]};
            if (to.whole) store4(b, to.o + col, v * inv);
            else *reinterpret_cast<f32x4*>(to.part + col) = v;
          }
        if (g == 0) {
          if (to.whole) b.lse[to.lse] = row_lse(m[i], l[i]);
          else { to.ml[0] = m[i]; to.ml[kChunkRows] = l[i]; }
        }
      }
      for (; redo != 0; redo &= redo - 1) row_again<float>(b, s, seg_s, run, kChunkRows, 32 * w + 16 * i + __builtin_ctz(redo), lane);
    }
  } while (f.more);
}

// ------------------------------------------------------------------------------- merge
// Joins the partial results of the items that more than one run has worked on: rows of the item that the start of a run is the first
// one to cut.  16 lanes take a row's columns of one part, eight each: all parts of a row one after the other where they are few, every fourth
// one with a wavefront on a row, or every 16th with a workgroup on a row.  (Bound by latency: 2048 tokens at the end of 4096, 512 items cut
// once, 65 thousand rows of two or three parts: 69 us with a wavefront a row, 21 so.)
struct Joined { float m, l; f32x4 o[2]; };
__device__ __forceinline__ void join_in(Joined& x, float m, float l, const f32x4 (&o)[2]) {
  const float top = fmaxf(x.m, m), ref = top == BURST_NEG_INF ? 0.f : top;
  const float f = fast_exp2((x.m - ref) * kLog2e), g = fast_exp2((m - ref) * kLog2e);
  x.m = top;
  x.l = (is_zero(f) ? 0.f : x.l * f) + (is_zero(g) ? 0.f : l * g);
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int k = 0; k < 4; k++) x.o[i][k] = (is_zero(f) ? 0.f : x.o[i][k] * f) + (is_zero(g) ? 0.f : o[i][k] * g);
}
__global__ void __launch_bounds__(256)
paged_merge_kernel(PagedArgs a, int rows_of_item) {
  __shared__ __attribute__((aligned(16))) float side[4][160];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = (lane & 15) * 4;
  const int run = blockIdx.x + 1, d = a.d;
  PagedJoin join = a.join[run];
  if (run >= a.join[0].n || join.n <= 0) return;
  join.n = min(join.n, a.runs - run + 1);          // (as they are; no access outside the workspace and the outputs if another call has written there)
  const bool few = rows_of_item <= kShortRows;
  const bool alone = join.n <= (few ? 8 : 32), together = join.n > (few ? 32 : 128);   // a lane group on a row; all wavefronts on a row
  const size_t slot = (size_t)rows_of_item * (d + 2);
  const float* const base = a.part + 2 * (size_t)(run - 1) * slot;
  const int step = alone ? 1 : together ? 16 : 4, begin = alone ? 0 : (together ? 4 * wave : 0) + (lane >> 4);
  const int rows = 16 / step;                      // of a workgroup at a time
  for (int r = blockIdx.y * rows + (alone ? 4 * wave + (lane >> 4) : together ? 0 : wave); r < rows_of_item; r += rows * gridDim.y) {
    const ItemRow x = item_row(a, join.part, join.block, join.count, r);
    if (!x.there || (unsigned)(join.first + x.token) >= (unsigned)a.w.rows || (unsigned)x.head >= (unsigned)a.heads) continue;   // (lanes that share a row alike)
    Joined sum = {BURST_NEG_INF, 0.f, {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}};
    for (int i0 = begin; i0 < join.n; i0 += 8 * step) {
      float m[8], l[8];
      f32x4 o[8][2];                                // (all of them asked for at once: every wait is for memory)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const int i = i0 + j * step;
        const float* const p = base + (2 * (size_t)i + (i == 0 ? 1 : 0)) * slot;
        m[j] = BURST_NEG_INF; l[j] = 0.f;
        o[j][0] = o[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (i >= join.n) continue;
        m[j] = p[(size_t)rows_of_item * d + r];
        l[j] = p[(size_t)rows_of_item * (d + 1) + r];
#pragma unroll
        for (int h = 0; h < 2; h++)
          if (c + 64 * h < d) o[j][h] = *reinterpret_cast<const f32x4*>(p + (size_t)r * d + c + 64 * h);
      }
#pragma unroll
      for (int j = 0; j < 8; j++) join_in(sum, m[j], l[j], o[j]);
    }
    for (int off = alone ? 64 : 16; off < 64; off <<= 1) {   // the lane groups
      f32x4 o[2];
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int e = 0; e < 4; e++) o[h][e] = __shfl_xor(sum.o[h][e], off);
      join_in(sum, __shfl_xor(sum.m, off), __shfl_xor(sum.l, off), o);
    }
    if (together) {
      __syncthreads();
      if (lane < 16) {
        *reinterpret_cast<f32x4*>(&side[wave][c]) = sum.o[0];
        *reinterpret_cast<f32x4*>(&side[wave][c + 64]) = sum.o[1];
        if (lane == 0) { side[wave][128] = sum.m; side[wave][129] = sum.l; }
      }
      __syncthreads();
      if (wave != 0) continue;
      for (int w = 1; w < 4; w++) {
        const f32x4 o[2] = {*reinterpret_cast<const f32x4*>(&side[w][c]), *reinterpret_cast<const f32x4*>(&side[w][c + 64])};
        join_in(sum, side[w][128], side[w][129], o);
      }
    }
    if (!alone && lane >= 16) continue;
    const size_t row = (size_t)(join.first + x.token), at = row * a.o_row + (size_t)x.head * a.o_head;
    const float inv = is_zero(sum.l) ? 0.f : 1.f / sum.l;
#pragma unroll
    for (int h = 0; h < 2; h++)
      if (c + 64 * h < d) store4(a, at + c + 64 * h, is_zero(sum.l) ? f32x4{0.f, 0.f, 0.f, 0.f} : sum.o[h] * inv);
    if (c == 0) a.lse[row * a.heads + x.head] = row_lse(sum.m, sum.l);
  }
}

// ------------------------------------------------------------------------------- launches
int launch_paged_short(const PagedArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)a.runs), block(64);
  if (dtype == BURST_BF16) {
    if (a.d <= 64) BURST_LAUNCH((paged_short_kernel<bf16, 64>), grid, block, 0, s, a);
    else BURST_LAUNCH((paged_short_kernel<bf16, 128>), grid, block, 0, s, a);
  } else {
    if (a.d <= 64) BURST_LAUNCH((paged_short_kernel<float, 64>), grid, block, 0, s, a);
    else BURST_LAUNCH((paged_short_kernel<float, 128>), grid, block, 0, s, a);
  }
  return launch_status();
}
int launch_paged_chunk(const PagedArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)a.runs), block(256);
  if (dtype == BURST_BF16) {
    const bool one = !a.full_p && (a.d == 64 || a.d == 128);
    if (a.d <= 32) BURST_LAUNCH((paged_chunk_kernel<64, 32, 2>), grid, block, 0, s, a);
    else if (a.d <= 64 && one) BURST_LAUNCH((paged_chunk_kernel<64, 64, 1>), grid, block, 0, s, a);
    else if (a.d <= 64) BURST_LAUNCH((paged_chunk_kernel<64, 64, 2>), grid, block, 0, s, a);
    else if (a.d <= 96) BURST_LAUNCH((paged_chunk_kernel<128, 96, 2>), grid, block, 0, s, a);
    else if (one) BURST_LAUNCH((paged_chunk_kernel<128, 128, 1>), grid, block, 0, s, a);
    else BURST_LAUNCH((paged_chunk_kernel<128, 128, 2>), grid, block, 0, s, a);
  } else {
    if (a.d <= 64) BURST_LAUNCH((paged_chunk_f32_kernel<64, 64>), grid, block, 0, s, a);
    else if (a.d <= 96) BURST_LAUNCH((paged_chunk_f32_kernel<128, 96>), grid, block, 0, s, a);
    else BURST_LAUNCH((paged_chunk_f32_kernel<128, 128>), grid, block, 0, s, a);
  }
  return launch_status();
}
int launch_paged_merge(const PagedArgs& a, int rows_of_item, hipStream_t s) {
  if (a.runs < 2) return BURST_OK;
  BURST_LAUNCH(paged_merge_kernel, dim3((unsigned)a.runs - 1, rows_of_item <= kShortRows ? 4 : 16), dim3(256), 0, s, a, rows_of_item);
  return launch_status();
}

}  // namespace burst
