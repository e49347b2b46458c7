/*
 * burst.h -- C ABI of the MI355X (gfx950) local-attention library.
 *
 * One device's share of a sequence-parallel attention ring (paper Sec. 2.2-2.4):
 * a resident query slice Q_i is attended against key/value chunks (K_j, V_j) that
 * arrive one at a time.  Each chunk's partial result is folded into a running
 * state (O_acc, m, l) by online softmax (paper Alg. 1); burst_finalize turns the
 * state into the output O_i and its log-sum-exp lse_i; the backward (paper Alg. 2)
 * recomputes the attention probabilities of a block pair from lse_i.
 *
 * Conventions common to every entry point
 *   - All data pointers are DEVICE pointers owned by the caller.  The library
 *     never frees caller memory and never synchronises the stream; every call
 *     only enqueues kernels on `stream` (a hipStream_t passed as void*, NULL =
 *     the default stream).  Pointers must be 16-byte aligned.
 *   - Tensors are indexed [B, H, rows, d] with d contiguous; per-row vectors
 *     (m, l, lse, D) are [B, H, rows].  fp32 tensors are always dense in that
 *     order; the tensors of type `dtype` are too unless burst_params.q_strides /
 *     kv_strides say otherwise.  K, V, dK, dV may have fewer heads than Q
 *     (burst_params.kv_heads; not in the paper).
 *   - Q, K, V, O, dO have element type `dtype` (bf16 or fp32).  The running
 *     state, lse, D and all gradients are fp32 (burst_walk_bwd with half_grads writes
 *     gradients of type `dtype`).
 *   - Scores are S = scale * Q K^T (Eq. 1 has scale = 1/sqrt(d); Alg. 1/2 omit
 *     it, here it is always applied).  scale must be finite and > 0.
 *   - Masking (not in the paper): with causal != 0 the key at global position
 *     k_off + c is visible to the query at global position q_off + r iff
 *     k_off + c <= q_off + r.  With window = w > 0 (paper Sec. 2.6: similarities
 *     a sparse pattern does not need are skipped) the key is visible only if
 *     k_off + c > q_off + r - w: a sliding window, the query itself and its w - 1
 *     predecessors when combined with causal; w = 0 means no window.  Key tiles and
 *     whole chunks outside the window are skipped, not computed and masked.
 *     With block_mask != NULL (block-sparse patterns, Sec. 2.6) a key must in addition
 *     lie in a block whose mask byte is nonzero; the three conditions are ANDed.  Key
 *     tiles no row of a workgroup can see are skipped.  The mask is read while the
 *     kernels run: keep it unchanged until they have finished.
 *     A row that sees no key keeps its state.
 *   - Return value: 0 on success, a negative burst_status otherwise.  On error
 *     nothing is enqueued and no output is written (entry points that enqueue
 *     several kernels check every kernel's limits before the first launch; only
 *     a launch failure reported by the HIP runtime itself, BURST_ERR_LAUNCH, can
 *     leave earlier kernels of the same call enqueued).
 *   - Thread safety: entry points may be called from several host threads.  The first
 *     call of a kernel family on a device sets that family's shared-memory function
 *     attributes (once per device, whichever thread comes first); that call cannot be
 *     recorded into a HIP graph, so run each entry point once eagerly on a device
 *     before capturing it.
 *   - Supported shapes: B, H >= 1; Nq, Nc >= 0 (0 = nothing to do); 1 <= d <= 128.
 *     Any Nq, Nc (ragged tails) are accepted.  bf16 with d a multiple of 8 runs on the
 *     bf16 matrix instructions, everything else (and slices, chunks or strides beyond
 *     32-bit byte offsets) on the fp32 one.  Probabilities and dS enter the second
 *     products rounded to bf16 at d = 64 and d = 128, with all their 24 bits otherwise
 *     (d = 128 as well: dK and dV of grouped heads with Nq no multiple of 64).
 *   - Infinities and NaN: at d = 64 and d = 128 (bf16) a hidden pair may be multiplied as
 *     zero, so that an infinite or NaN value can make NaN of rows (keys) that share a
 *     tile with one that sees it.  The other calls keep to the visible pairs.
 */
#ifndef BURST_H
#define BURST_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum burst_dtype { BURST_BF16 = 0, BURST_F32 = 1 };

enum burst_status {
  BURST_OK = 0,
  BURST_ERR_NULL = -1,      /* a required pointer is NULL */
  BURST_ERR_ALIGN = -2,     /* a pointer is not 16-byte aligned */
  BURST_ERR_SHAPE = -3,     /* unsupported or inconsistent sizes, bad scale */
  BURST_ERR_DTYPE = -4,     /* unknown dtype */
  BURST_ERR_ARCH = -5,      /* current device is not gfx950 */
  BURST_ERR_LAUNCH = -6,    /* the HIP runtime reported a launch error */
  BURST_ERR_ALLOC = -7,     /* internal scratch allocation failed */
  BURST_ERR_TOO_LARGE = -8  /* burst_local_bwd_static: B*H*Nq > BURST_STATIC_MAX_ROWS */
};

typedef struct burst_params {
  int32_t B;        /* batch */
  int32_t H;        /* heads (the paper's Z) */
  int32_t Nq;       /* rows of the resident query slice (the paper's N/G) */
  int32_t Nc;       /* rows of this key/value chunk */
  int32_t d;        /* head dimension */
  int32_t dtype;    /* burst_dtype of Q, K, V, O, dO */
  int32_t causal;   /* 0 = every key visible, 1 = mask by global position */
  float   scale;    /* softmax scale, normally 1/sqrt(d) */
  int64_t q_off;    /* global position of query row 0 */
  int64_t k_off;    /* global position of row 0 of this chunk */
  int64_t window;   /* 0 = none; w > 0: keys at positions <= query position - w are hidden */
  const uint8_t* block_mask; /* NULL = none; else DEVICE pointer to a row-major byte matrix
                              * [ceil(Nq / block)][ceil(Nc / block)] for THIS query slice x chunk
                              * pair (one for all heads, or one per (batch, head), see
                              * block_mask_stride): entry (i, j) = 0 hides
                              * keys j*block .. of the chunk from query rows i*block .. of the slice */
  int32_t block;    /* edge of a mask block in rows = keys; a positive multiple of 64 when
                     * block_mask != NULL, ignored otherwise */
  int32_t kv_heads; /* 0 or H: K, V, dK, dV have H heads.  Otherwise (grouped-query attention) they
                     * have kv_heads heads, [B, kv_heads, Nc, d]; H must be a multiple of kv_heads and
                     * query head h uses key/value head h / (H / kv_heads); dK, dV sum over the group */
  int64_t block_mask_stride; /* bytes from one (batch, query head)'s flag matrix to the next, B*H
                     * matrices in all; 0 = one matrix shared by every batch entry and head */
  int64_t q_strides[3];  /* element strides {batch, head, row} of Q, dO and O (input and output);
                     * all zero = contiguous [B, H, Nq, d].  The last dimension is always contiguous.
                     * E.g. {Nq*H*d, d, H*d} addresses sequence-major [B, Nq, H, d] tensors (the
                     * layout of Sec. 2.2's backward messages) without a copy.  Row stride >= d, each
                     * stride a multiple of 16 bytes, none negative. */
  int64_t kv_strides[3]; /* the same for K_chunk and V_chunk ({batch, head, row}; kv_heads heads) */
} burst_params;

/* Alg. 1, initialisation: O_acc = 0, l = 0, m = -inf.
 * O_acc [B,H,Nq,d] fp32, m and l [B,H,Nq] fp32 (all written). */
int burst_state_init(float* O_acc, float* m, float* l, const burst_params* p, void* stream);

/* Alg. 1, body of the loop for one chunk, computed tile by tile (Sec. 2.4):
 * S = scale Q K_chunk^T (masked), per-row max / exp / sum, P V_chunk, and the
 * online-softmax merge into the state (m_new = max, rescale of l and O_acc).
 * Q [B,H,Nq,d], K_chunk and V_chunk [B,H,Nc,d] (read only); O_acc, m, l are
 * read and updated in place.  The state is any triple for which
 * m + log l and O_acc / l are the true log-sum-exp and output of the keys seen
 * so far; m is in natural-log units of the scaled scores and only a reference
 * point (it need not be the exact running maximum).  No S or P is ever stored. */
int burst_local_fwd(const void* Q, const void* K_chunk, const void* V_chunk,
                    float* O_acc, float* m, float* l, const burst_params* p, void* stream);

/* Alg. 1, last two steps: O = diag(l)^-1 O_acc (written as `dtype`),
 * lse = m + log l (fp32).  Rows with l = 0 give O = 0, lse = -inf. */
int burst_finalize(const float* O_acc, const float* m, const float* l,
                   void* O_out, float* lse, const burst_params* p, void* stream);

/* Alg. 1, the merge step on its own: state a <- merge(state a, state b), for
 * combining two partial walks over disjoint key sets (tree / multi-device
 * combine).  a is updated in place, b is read only. */
int burst_merge_state(float* O_a, float* m_a, float* l_a,
                      const float* O_b, const float* m_b, const float* l_b,
                      const burst_params* p, void* stream);

/* Alg. 2, pre-step: D = rowsum(dO o O).  O and dO [B,H,Nq,d] of `dtype`,
 * D [B,H,Nq] fp32 (written). */
int burst_bwd_prepare(const void* O, const void* dO, float* D, const burst_params* p, void* stream);

/* Alg. 2, one block pair (query slice x one chunk): recompute
 * S = scale Q K_chunk^T and P = exp(S - lse); dV += P^T dO; dP = dO V^T;
 * dS = P o (dP - D); dK += scale dS^T Q; dQ += scale dS K.
 * D may be NULL: it is then computed from O and dO into a scratch buffer that
 * the library owns, one per (device, stream), allocated with hipMalloc on the first
 * such call (and again when a later call needs a larger one: the old block is kept,
 * never freed, since enqueued kernels may still read it) and kept until process
 * exit.  Such a call therefore may allocate (never under stream capture: pass D
 * there), but it never frees or synchronises.  Calls with D == NULL are serialised
 * by a library lock from the buffer lookup to the last enqueue; consecutive calls
 * on one stream reuse the buffer in stream order.  With a non-NULL D nothing is
 * allocated or locked, O is not read and may be NULL.
 * dQ [B,H,Nq,d], dK_chunk and dV_chunk [B,H,Nc,d], all fp32.
 * accumulate_dq / accumulate_dkv: 1 = add to what the buffer holds (the caller
 * zero-fills before the first block pair), 0 = the buffer is overwritten with
 * this block pair's contribution.  Every output row is owned by one wavefront
 * (no atomics), so results are bitwise reproducible from run to run. */
int burst_local_bwd(const void* Q, const void* K_chunk, const void* V_chunk,
                    const void* O, const void* dO, const float* lse, const float* D,
                    float* dQ, float* dK_chunk, float* dV_chunk,
                    int accumulate_dq, int accumulate_dkv,
                    const burst_params* p, void* stream);

/* For callers that cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, conventions and results as
 * burst_local_bwd with D == NULL (D = rowsum(dO o O) is computed by the call), except that D lives
 * in a static device array inside the library (BURST_STATIC_MAX_ROWS floats = 8 MiB per GPU, held
 * until the process ends) instead of an allocated buffer: this entry point calls no hipMalloc, no
 * hipFree and no allocating library routine, ever.  Its first call on a device looks up that
 * device's address of the array and sets the kernels' function attributes: run it once eagerly
 * on a device before capturing it.
 * Limit: B*H*Nq <= BURST_STATIC_MAX_ROWS, else BURST_ERR_TOO_LARGE (nothing enqueued).
 * All calls on one GPU share the array, which keeps the last call's D: nothing in it has to start
 * at zero (each call rewrites the B*H*Nq entries it reads), but two calls whose kernels can overlap
 * on one GPU (different streams without an event between them) race on it.  Calls on one stream,
 * from any number of host threads, are safe. */
#define BURST_STATIC_MAX_ROWS (2 * 1024 * 1024)
int burst_local_bwd_static(const void* Q, const void* K_chunk, const void* V_chunk,
                           const void* O, const void* dO, const float* lse,
                           float* dQ, float* dK_chunk, float* dV_chunk,
                           int accumulate_dq, int accumulate_dkv,
                           const burst_params* p, void* stream);

/* Size in bytes of the D buffer a burst_local_bwd call with these parameters and D == NULL needs
 * (B*H*Nq*4; the library's own buffer may be larger).  It is the only device memory the library
 * ever holds for a call: every other entry point, and burst_local_bwd with D given, is handed all
 * its buffers (the tiled steps keep S and P in registers, Sec. 2.4, and need no workspace).  A
 * caller that wants no library allocation allocates this many bytes, calls burst_bwd_prepare and
 * passes D.  Returns 0 for an invalid parameter block. */
size_t burst_workspace_bytes(const burst_params* p);

/* The two halves of burst_local_bwd on their own, for callers that need only one side
 * (Alg. 2 with the query side travelling needs dQ_j from every device but dK_i, dV_i only
 * locally) or that time them separately.  Same arguments and conventions as above; D must
 * be given.  burst_local_bwd(D != NULL) is exactly _dq followed by _dkv. */
int burst_local_bwd_dq(const void* Q, const void* K_chunk, const void* V_chunk,
                       const void* dO, const float* lse, const float* D,
                       float* dQ, int accumulate_dq, const burst_params* p, void* stream);
int burst_local_bwd_dkv(const void* Q, const void* K_chunk, const void* V_chunk,
                        const void* dO, const float* lse, const float* D,
                        float* dK_chunk, float* dV_chunk, int accumulate_dkv,
                        const burst_params* p, void* stream);

/* A whole walk in one call, for chunks that are already resident (or have arrived together): the
 * kernels go from one chunk to the next with the state in registers and the next tile in flight,
 * instead of storing and reloading it between launches. */
typedef struct burst_chunk {
  const void* K; const void* V;      /* [B, kv_heads, Nc, d] of `dtype` */
  void* dK; void* dV;                /* burst_walk_bwd: the same shapes, dense; ignored by burst_walk_fwd */
  const uint8_t* block_mask;         /* as in burst_params, for this chunk (edge: burst_params.block) */
  int64_t block_mask_stride;
  int64_t k_off;                     /* global position of row 0 */
  int64_t kv_strides[3];             /* as in burst_params; all zero = contiguous */
  int32_t Nc;                        /* rows, >= 0 */
  int32_t reserved;                  /* 0 */
} burst_chunk;
/* burst_state_init, burst_local_fwd for each of the n_chunks chunks in order, burst_finalize: the same
 * O, lse and final state.  `p` gives everything but Nc, k_off, block_mask, block_mask_stride and
 * kv_strides, which are taken from the chunks.  workspace: device memory of at least
 * burst_walk_workspace_bytes(..., BURST_WALK_FORWARD) bytes, 16-byte aligned, contents undefined before and after, or NULL;
 * with it a walk that would leave much of the chip idle (few rows; fp32 also up to 1024 blocks of 32 rows above 64 columns) is
 * spread over it by splitting the keys into ranges whose partial states are merged at the end, and the workgroups of such a
 * walk may halve every tile between two groups of wavefronts (the sums then come in another order than chunk by chunk).
 * O_acc, m, l may all be NULL: the state is then not kept (workspace: burst_walk_workspace_bytes(..., BURST_WALK_NO_STATE)),
 * and a walk of one chunk may have two groups, or the other d = 128 kernels, with and without a workspace.
 * Which of these a call has depends on its sizes alone, the number of heads among them: a call repeated gives the same bits, a
 * head in a call of other sizes the same values up to rounding. */
int burst_walk_fwd(const void* Q, const burst_chunk* chunks, int n_chunks, float* O_acc, float* m, float* l,
                   void* O_out, float* lse, void* workspace, size_t workspace_bytes,
                   const burst_params* p, void* stream);
/* burst_bwd_prepare (when O is given; D is then written, else read), then burst_local_bwd for each
 * chunk in order, with the dK and dV of the chunk.  accumulate_dq = 0: dQ is overwritten with the
 * contribution of all chunks; accumulate_dkv applies to every chunk's dK and dV.  dQ and the chunks' dK,
 * dV are fp32 or, with half_grads, of `dtype` (each value is the fp32 sum rounded once); half_grads
 * excludes both accumulate flags, and needs the workspace that burst_walk_workspace_bytes(...,
 * BURST_WALK_HALF_GRADS) asks for (BURST_ERR_SHAPE if a part of it that it cannot do without is missing).
 * With the workspace few or unequal walks over query tiles (grouped heads, few keys, causal masks) are also cut
 * into parts whose partial dK, dV are added at the end; key ranges, groups and the order of sums as in burst_walk_fwd
 * (half_grads in the place of the state that is not kept). */
int burst_walk_bwd(const void* Q, const burst_chunk* chunks, int n_chunks, const void* O, const void* dO,
                   const float* lse, float* D, void* dQ, int accumulate_dq, int accumulate_dkv, int half_grads,
                   void* workspace, size_t workspace_bytes, const burst_params* p, void* stream);
/* Bytes of workspace that either of the two can use (or, under these flags, needs) for these arguments;
 * 0: none.  Host logic, no device call. */
size_t burst_walk_workspace_bytes(const burst_chunk* chunks, int n_chunks, const burst_params* p, int flags);
/* How burst_walk_bwd lays out its first dK/dV launch for these arguments and fp32 gradients: 0 = a workgroup per block of
 * keys, 1 = the walks over query tiles cut into parts (with the workspace), 2 = one workgroup per CU that takes several
 * blocks in turn; a negative burst_status for invalid arguments.  (With half_grads a walk of one chunk for which this is 1 may
 * have a workgroup per 64 keys instead, not cut.)  Host logic, no device call. */
int burst_walk_dkv_form(const burst_chunk* chunks, int n_chunks, const burst_params* p, int with_workspace);
#define BURST_WALK_HALF_GRADS 1   /* for burst_walk_bwd with half_grads */
#define BURST_WALK_NO_STATE 2     /* for burst_walk_fwd without O_acc, m, l */
#define BURST_WALK_FORWARD 4      /* for burst_walk_fwd alone: not what only burst_walk_bwd uses */

/* Alg. 1, body of the loop for one chunk exactly as printed, WITHOUT the tiling of
 * Sec. 2.4 (the "w/o LAO" variant of the paper's ablation, Tables 2-3): the whole
 * S_ij = scale Q K_chunk^T and P_ij = exp(S_ij - m_ij) of the block pair are stored in
 * `workspace` between the steps, then O_ij = P_ij V_chunk is merged into the state.
 * Same arguments, masking and resulting state as burst_local_fwd (up to rounding).
 * workspace: device memory, 256-byte aligned, at least
 * burst_materialized_workspace_bytes(p) bytes (B H Nq Nc (4 + element size) plus the
 * chunk's row statistics); owned by the caller, contents undefined afterwards except
 * that it starts with S_ij as fp32 [B,H,Nq,ceil8(Nc)] (raw scaled scores, unmasked),
 * followed at the next 256-byte boundary by P_ij in `dtype` with the same pitch
 * (masked entries and the padding columns are 0).  Returns BURST_ERR_SHAPE if
 * workspace_bytes is too small.  burst_materialized_workspace_bytes returns 0 for
 * invalid parameters. */
size_t burst_materialized_workspace_bytes(const burst_params* p);
int burst_local_fwd_materialized(const void* Q, const void* K_chunk, const void* V_chunk,
                                 float* O_acc, float* m, float* l,
                                 void* workspace, size_t workspace_bytes,
                                 const burst_params* p, void* stream);

/* Alg. 2, one block pair, in the same untiled form (the backward of the "w/o LAO" variant): the
 * seven steps of the loop body one after the other, S_ij, P_ij, dP_ij and dS_ij of the whole
 * block pair stored in `workspace` between them.  Same arguments, masking and results as
 * burst_local_bwd with D given (up to rounding).  workspace: device memory, 256-byte aligned,
 * at least burst_materialized_bwd_workspace_bytes(p) bytes (B H Nq Nc (4 + 2 element sizes));
 * afterwards it starts with dP_ij as fp32 [B,H,Nq,ceil8(Nc)], followed at the next 256-byte
 * boundaries by P_ij and dS_ij in `dtype` with the same pitch (hidden entries and padding 0;
 * dS_ij without the factor scale). */
size_t burst_materialized_bwd_workspace_bytes(const burst_params* p);
int burst_local_bwd_materialized(const void* Q, const void* K_chunk, const void* V_chunk,
                                 const void* dO, const float* lse, const float* D,
                                 float* dQ, float* dK_chunk, float* dV_chunk,
                                 int accumulate_dq, int accumulate_dkv,
                                 void* workspace, size_t workspace_bytes,
                                 const burst_params* p, void* stream);

/* Positions beside the attention, and a cache of keys and values in pages (not in the paper: the rotation that models apply to Q and
 * K before the walks above, with the positions that a ring's slices have; and what serves the sequence afterwards, token by
 * token).  The arrays of numbers that these calls read on the device (starts, lengths, table, positions, offsets) are aligned to
 * their element type, and no value in them leads to an access outside the tensors. */

/* Rotation of pairs of columns by an angle of 2 pi x position x turns[pair]: a pair (a, b) becomes
 * (a cos - b sin, b cos + a sin) x amplitude.  The angle is computed in 64 bits from the position, cos and sin to 24 bits. */
typedef struct burst_rotary {
  const double* turns;  /* DEVICE [dims / 2]: turns per position of every pair */
  int32_t dims;         /* rotated columns, even, 2 .. d; the columns from dims on are copied */
  int32_t interleaved;  /* 0: columns i and i + dims / 2 are a pair; 1: columns 2 i and 2 i + 1 */
  float   amplitude;    /* finite, normally 1 */
  int32_t inverse;      /* 1: by the negative angle, which takes the gradient of the output to that of the input */
} burst_rotary;
/* One tensor [B, heads, rows, d] and its rotated copy. */
typedef struct burst_rows {
  const void* x; void* y;            /* y: written, every row in a place of its own; x itself (then with the same strides) or memory that x does not share */
  const int64_t* positions;          /* DEVICE: row n of batch entry b is at offset + positions[b * positions_stride + n]; NULL: offset + n */
  int64_t positions_stride, offset;
  int64_t x_strides[3], y_strides[3];/* element strides {batch, head, row}; all zero = contiguous */
  int32_t B, heads, rows;            /* 0 .. 2^31 - 256 */
  int32_t reserved;                  /* 0 */
} burst_rows;
/* Rotates n tensors (queries and the chunks' keys of a walk) of head dimension d, 2 <= d <= 128, and type `dtype`.  Rows may start anywhere
 * (elements aligned to their own size); rows and column pairs on 16-byte boundaries are read and written 16 bytes at a time. */
int burst_rotate(const burst_rows* tensors, int n, const burst_rotary* r, int d, int dtype, void* stream);

/* Rows normalised by their root mean square, weighted and rotated, in one pass (models that normalise every head's queries and keys before the
 * rotation): with r = (mean of x^2 over the d columns + eps)^(-1/2), y is the rotation (see burst_rotate) of x r w.  All of it in 32 bits (angles in
 * 64), rounded once; sums of squares beyond 32 bits' range count as infinite. */
typedef struct burst_norm_rows {
  burst_rows rows;                   /* x and y.  burst_norm_rotate_bwd: x is the gradient of the result and y that of what it was made of, NULL: not wanted */
  const void* from;                  /* burst_norm_rotate_bwd: what the forward call read */
  int64_t from_strides[3];           /* as in burst_rows */
  int32_t weight;                    /* which of the weights; -1: none (1 for every column) */
  int32_t reserved;                  /* 0 */
} burst_norm_rows;
typedef struct burst_norm_weight {
  const void* w;                     /* DEVICE [d], elements aligned to their own size */
  void* dw;                          /* burst_norm_rotate_bwd: written, [d] of the type of w; NULL: not wanted */
  int32_t f32;                       /* w and dw are fp32 whatever the dtype */
  int32_t reserved;                  /* 0 */
} burst_norm_weight;
/* n tensors with `weights` weights, each of one tensor or of several; r = NULL: not rotated.  eps >= 2^-126.  y is x itself (then with the same strides)
 * or memory that x does not share. */
int burst_norm_rotate(const burst_norm_rows* tensors, int n, const burst_norm_weight* w, int weights, float eps, const burst_rotary* r, int d,
                      int dtype, void* stream);
/* Gradients of all of them, those of a weight summed over every row of all its tensors (in fp32, in an order that follows from the sizes, strides and alignments
 * of the call; rounded once).  r as in the forward call (r->inverse = 0).  workspace: burst_norm_workspace_bytes of the same arguments, 16-byte aligned; none is needed where no
 * weight's gradient is wanted. */
int burst_norm_rotate_bwd(const burst_norm_rows* tensors, int n, const burst_norm_weight* w, int weights, float eps, const burst_rotary* r, int d,
                          int dtype, void* workspace, size_t workspace_bytes, void* stream);
/* Follows from the sizes, strides and alignments of the tensors and from which gradients are wanted; 0 for invalid arguments.  Host logic, no device call. */
size_t burst_norm_workspace_bytes(const burst_norm_rows* tensors, int n, const burst_norm_weight* w, int weights, float eps, const burst_rotary* r, int d,
                                  int dtype);

/* The new tokens of several sequences and the pages of their caches.  New tokens lie packed, sequence after sequence:
 * sequence s has rows starts[s] .. starts[s + 1] - 1 of the token tensors, which are indexed [row, head, d].  lengths[s] counts
 * the tokens of the sequence, the new ones among them: new token t of n is at position lengths[s] - n + t, and position p
 * is row p % page of page table[s * table_stride + p / page].  Lengths are cut to 0 .. 2^30 and starts to 0 .. rows; a
 * page that is not in 0 .. pages - 1 holds no keys, and neither does a position behind the table's row (from width * page on): new tokens there are
 * not kept, and see the keys that are.  Starts do not decrease: where they do, burst_paged_fwd writes nothing, and which tokens
 * burst_cache_append takes for whose is not defined.  The arrays are not to
 * change while a call that reads them runs. */
typedef struct burst_paged_params {
  int32_t sequences, rows;           /* >= 0, < 2^30; rows: of the token tensors, those behind the last sequence among them */
  int32_t H, kv_heads, d, dtype;     /* H a multiple of kv_heads; d a multiple of 8 (bf16) or 4 (fp32), at most 128 */
  int32_t pages, page, width;        /* pages; rows of a page: a power of two, 16 or more; pages of a table row; width * page < 2^30 */
  int32_t max_new;                   /* most new tokens of any sequence as far as the caller knows it, 0 = not known: chooses the kernel only */
  int32_t causal;                    /* burst_paged_fwd: 0 = every key of the sequence is visible, 1 = those up to the token's position */
  int32_t out_f32;                   /* burst_paged_fwd: 1 = O is fp32 whatever the dtype */
  float   scale;                     /* burst_paged_fwd: as in burst_params */
  int32_t full_p;                    /* burst_paged_fwd, bf16: 1 = probabilities with 16 bits at every d (see there) */
  int64_t window;                    /* burst_paged_fwd: as in burst_params */
  const int32_t* starts; const int32_t* lengths; const int32_t* table;   /* DEVICE [sequences + 1], [sequences], [sequences][width] */
  int64_t table_stride;              /* entries from one sequence's pages to the next's; 0 = width */
  int64_t page_strides[3];           /* elements {page, head, row} of K_pages and V_pages; all zero = dense [pages, kv_heads, page, d] */
  int64_t q_strides[2], kv_strides[2], o_strides[2];   /* elements {row, head} of Q; of K and V (new tokens); of O or Q_out; both zero = dense.
                                      * Strides in multiples of 16 bytes (burst_cache_append: any), none negative, none 0 between rows that are written */
} burst_paged_params;
/* Writes the new tokens' keys and values (K, V [rows, kv_heads, d]) to their places in K_pages and V_pages, the keys rotated by their
 * positions + offsets[s] (int64 DEVICE [sequences], NULL: 0; what the ring keeps before this device's share).  r = NULL: nothing is rotated.
 * Q, if not NULL: the queries [rows, H, d] are rotated likewise to Q_out.  Tokens at positions below 0, behind the table or in pages that are none are left
 * out (their queries are rotated if they have a position), rows of Q_out behind the last sequence left as they were.  One launch.
 * Pages that share a place, by equal table entries of two sequences say, must not both get a new token there. */
int burst_cache_append(const void* K, const void* V, void* K_pages, void* V_pages, const void* Q, void* Q_out,
                       const int64_t* offsets, const burst_rotary* r, const burst_paged_params* p, void* stream);
/* burst_cache_append with more to say about the rows. */
typedef struct burst_store {
  const void* q_weight; const void* k_weight;   /* DEVICE [d]: Q, K are normalised first (see burst_norm_rotate); NULL: not */
  int32_t q_weight_f32, k_weight_f32;           /* these weights are fp32 whatever the dtype */
  float   eps;                                  /* of the norms, >= 2^-126 if there are any */
  int32_t reserved;                             /* 0 */
  const int64_t* slots;                         /* DEVICE [rows]: row i's key and value go to row slots[i] % page of page slots[i] / page, instead of by the
                                                 * table; negative, or in a page that is none: left out.  No two rows go to one place */
  const int64_t* positions;                     /* DEVICE [rows]: positions of the rotation, instead of the place in the sequence; negative: the row is left out */
  const int64_t* offsets;                       /* as burst_cache_append's; NULL if there are positions */
} burst_store;
/* With both slots and positions nothing else is read of the batch (starts, lengths and table may be NULL); with one of them, rows that belong to no sequence
 * are left out. */
int burst_cache_store(const void* K, const void* V, void* K_pages, void* V_pages, const void* Q, void* Q_out,
                      const burst_store* how, const burst_rotary* r, const burst_paged_params* p, void* stream);
/* Attention of the new tokens over their sequences' pages: O [rows, H, d] of `dtype` (fp32 with out_f32) and lse [rows, H] fp32,
 * dense.  Tokens that see no key get O = 0 and lse = -inf; rows behind the last sequence are left as they were.  (O as fp32, lse, 1) is
 * a state that burst_merge_state takes: sequences whose cache is spread over a ring are put together so.
 * Hidden keys have no effect whatever they hold.  The order of the sums depends on the sizes, lengths and max_new of the call, all sequences'
 * among them; a call repeated gives the same bits.  bf16 probabilities enter the second product with 16 bits (two bf16 terms); at d = 64 and
 * d = 128 the kernel of longer chunks rounds them to bf16 once, as burst_local_fwd does there, unless full_p is set.
 * workspace: burst_paged_workspace_bytes(p) bytes of device memory, 16-byte aligned, contents undefined before and after; two
 * calls that may run at the same time need one each. */
int burst_paged_fwd(const void* Q, const void* K_pages, const void* V_pages, void* O, float* lse, void* workspace,
                    size_t workspace_bytes, const burst_paged_params* p, void* stream);
/* Does not depend on what the arrays on the device hold; 0 for invalid parameters.  Host logic, no device call. */
size_t burst_paged_workspace_bytes(const burst_paged_params* p);
/* The same for drafted tokens, a tree of them a sequence (causal != 0).  tree: DEVICE [rows][words], row i's mask at tree + i * tree_stride (0 = words): new
 * token t of a sequence sees all keys before the sequence's new tokens, and new token j if bit j % 64 of word j / 64 of its row is set (itself among
 * them; bits from the number of new tokens on mean nothing).  With a window w, the keys before the new tokens at positions up to b + depth - w are hidden, where b is the
 * position of the first new token and depth + 1 the number of bits; the mask alone says which new tokens are seen.  Sequences with more than 64 * words new
 * tokens are chunks of prompts, as in burst_paged_fwd.  The masks are not to change while the call runs.  Workspace as burst_paged_fwd's. */
int burst_paged_tree_fwd(const void* Q, const void* K_pages, const void* V_pages, void* O, float* lse, const int64_t* tree, int words, int64_t tree_stride,
                         void* workspace, size_t workspace_bytes, const burst_paged_params* p, void* stream);

/* The books of such a cache, kept on the device: what a step's calls read, from the lengths of its sequences.
 * Sequences are served in their order, those that do not fit are passed over: their new tokens have to fit into the token tensors behind those of the sequences served before,
 * all of their tokens into a row of the table, and the pages that they still lack have to be on the stack.  Entries of a served sequence's row that new
 * tokens lie in and that hold no page (nothing in 0 .. pages - 1) get the pages from the top of the stack, in their order; what is there is kept, so that the same call again
 * changes nothing.  Sequences that have ended give the pages of their row back first, in order, and have -1 in all of it. */
typedef struct burst_plan {
  int32_t sequences, rows;           /* 0 .. 4096; 0 .. 2^20 - 1, of the token tensors */
  int32_t pages, page, width;        /* as in burst_paged_params */
  int32_t words, most;               /* of the masks; columns of parents */
  int32_t window;                    /* masks name the last so many tokens of a branch, the token itself among them: what a window of the attention leaves of it (0: all of it).  A
                                      * token so deep sees no key before the new ones either, which that number of bits tells burst_paged_tree_fwd as well */
  const int32_t* added;              /* DEVICE [sequences]: new tokens; negative: the sequence has ended */
  const int32_t* lengths;            /* DEVICE [sequences]: tokens that are in the cache (cut to 0 .. 2^30) */
  int32_t* table; int64_t table_stride;   /* DEVICE [sequences][width], read and written; stride as in burst_paged_params */
  int32_t* free_pages; int32_t* free_count;   /* DEVICE [pages], [1]: the stack of pages that are free, its top at free_count - 1 (cut to 0 .. pages); read and written */
  const int32_t* parents; int64_t parents_stride;   /* DEVICE [sequences][most] (stride: 0 = most): the new token that each new token hangs on, one before it; negative, another, or not among
                                      * the columns: none.  NULL: no trees (with most = 0 any other address has them) */
  int32_t* starts; int32_t* totals;  /* written, DEVICE [sequences + 1], [sequences]: starts and lengths for the paged calls (a sequence that was passed over has no new tokens) */
  int64_t* slots; int64_t* positions;   /* written, DEVICE [rows]: see burst_store; -1 behind the last sequence.  Positions of trees: tokens before the new ones + depth */
  int64_t* tree;                     /* written if there are parents, DEVICE [rows][words]: see burst_paged_tree_fwd; 0 for chunks of more than 64 * words tokens, whose parents are
                                      * not looked at */
} burst_plan;
/* The arrays that are written lie apart from one another and from those that are read. */
int burst_cache_plan(const burst_plan* p, void* stream);
/* Keeps some of the new tokens of every sequence, in all layers' pages: with b = lengths[s] - the number of new tokens, the row at position b + kept[s * kept_stride + j] goes to
 * position b + j, for j < counts[s] (cut to 0 .. most and to the new tokens), and lengths_out[s] is b + counts[s].  The numbers in kept (kept_stride: 0 = most) increase within a
 * sequence; where they do not, or are none of a new token, it is not defined which row is where (it is some new token's, or what was there).  Rows whose place is in no
 * page stay.  pools: HOST array of n different tensors of pages, keys' and values', that lie as page_strides say.  lengths_out is none of the arrays that are read.  sequences: at most 65535. */
int burst_cache_keep(void* const* pools, int n, const int32_t* kept, int64_t kept_stride, int most, const int32_t* counts, int32_t* lengths_out,
                     const burst_paged_params* p, void* stream);

/* For tests and tuning (no counterpart in the paper): which of the two kernel families serves
 * bf16, d = 128 calls.  0 = chosen per call (the default): forward and dQ from how well the call's
 * workgroups fill the chip and from the flags' block edge, dK/dV always hand-scheduled, with 64
 * instead of 128 keys per workgroup for 64-wide block flags; 1 = always the hand-scheduled kernels
 * (256 query rows, 128 keys per workgroup); 2 = always the plainly written ones (128 rows, 64 keys
 * per workgroup).  Process-wide; results of the two
 * families agree within the tolerance, not bitwise.  Returns BURST_ERR_SHAPE for another value. */
int burst_set_kernel_family(int family);
/* Which family would serve burst_local_fwd / the dQ half of burst_local_bwd for these parameters
 * under the current setting: 1 or 2 as above, 0 = neither (another head dimension or type, or a
 * shape only the generic kernels take); a negative burst_status for an invalid block.  Walks of several chunks
 * choose likewise for each of them; a causal walk of one chunk without a state (with half_grads) may take family 2 where
 * this is 1.  Host logic only, no device call. */
int burst_kernel_family_for(const burst_params* p);

/* Timing helper for harnesses that cannot create HIP events themselves:
 * records/queries events on the same stream the kernels are launched on.
 * burst_event_create returns an opaque handle (NULL on failure). */
void* burst_event_create(void);
int   burst_event_record(void* event, void* stream);
int   burst_event_elapsed_ms(void* start, void* stop, float* ms); /* waits for `stop` */
void  burst_event_destroy(void* event);

/* Micro-benchmarks for the measurement harness (no counterpart in the paper): the rates the
 * attention kernels are compared with, measured with the instruction forms they use.
 * burst_probe_mfma: 256 workgroups of 4 * wavefronts_per_simd (1 or 2) wavefronts; each wavefront
 * issues iters * 16 v_mfma_f32_32x32x16_bf16 (32768 FLOP each) and nothing else.  a_from_lds: 0 =
 * both operands stay in registers, 1 = the A operand of every MFMA is read fresh from LDS (128-bit
 * reads), 2 = of every second MFMA.  operands: 64 KiB of bf16 values on the device (their contents
 * set how many bits toggle, and with that the clock the chip sustains); sink: 256 * 512 floats,
 * written.  The caller times the launch.
 * burst_probe_atomic_dq: the memory traffic of a backward that would compute a block pair once,
 * keys stationary, and get its dQ partial sums out of the workgroups: heads * key_blocks workgroups
 * (heads a multiple of 8), each adding one [64][128] tile per 64 query rows into dQ [heads][Nq][128]
 * (Nq a multiple of 64).  mode 1: fp32 atomic adds; mode 0: plain stores in the same pattern; mode 2:
 * plain load-add-store in the same pattern (racing: timing only).  No arithmetic: a lower bound on
 * what such a kernel would take. */
int burst_probe_mfma(int a_from_lds, int wavefronts_per_simd, const void* operands, float* sink, int iters,
                     void* stream);
int burst_probe_atomic_dq(float* dQ, int heads, int Nq, int key_blocks, int mode, void* stream);

const char* burst_strerror(int status);
int         burst_version(void);

#ifdef __cplusplus
}
#endif
#endif /* BURST_H */
