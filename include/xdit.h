/*
 * xdit.h -- C ABI of the MI355X (gfx950) DiT attention hot path of xDiT
 * (arXiv 2411.01738): the PipeFusion patch step, the sequence-parallel chunk
 * step and the log-sum-exp merge of chunk partials, as one GPU executes them;
 * and what surrounds the attention in a layer: rotary positions, norms of
 * queries and keys, and the gradients of these and of the chunk step.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Pointers: every tensor pointer is a DEVICE pointer, owned by the caller, at
 *   least 16-byte aligned, to dense row-major storage.  The library allocates
 *   nothing and keeps no state except a per-thread stream and error message,
 *   the GEMM plans of xdit_stage_step (hipBLASLt's own memory) and the static
 *   scratch array of xdit_chunk_attn_split_noalloc.  Exceptions:
 *   xdit_lse_merge's `outs` / `lses` are HOST arrays holding `n` device
 *   pointers; dims, scaling, strides and xdit_qk of rotation and norms are
 *   host data too; rotation and norms take strided tensors; norm weights,
 *   their gradients and the LSE of the gradients need their type's alignment.
 * Layouts (the paper fixes none; this is the layout a QKV projection emits):
 *   activations  [B, N, H, d]  sequence-major, d contiguous (q, k, v, out,
 *                              fresh_k, fresh_v, merge partials)
 *   K/V buffer   [2, B, N, H, d]  plane 0 = K, plane 1 = V
 *   LSE          [B, H, Nq]    float32, natural log of sum_j exp(s_j) where
 *                              s_j = (q . k_j) / sqrt(d)
 * dtype: XDIT_BF16 or XDIT_F32, the element type of every activation tensor
 *   of a call (LSE is always float32).  bf16 calls compute QK^T and PV on the
 *   matrix cores with float32 accumulation and round the output to nearest
 *   even; f32 calls use float32 products throughout.
 * head_dim: 64, 72 or 128.
 * Softmax scale: always 1/sqrt(head_dim).  Attention is full (no mask).
 * Streams: every call is asynchronous on the stream set by xdit_set_stream
 *   for the calling thread (NULL = the default stream).  Device faults surface
 *   at the caller's next synchronisation.
 * Errors: 0 on success, a negative xdit_status otherwise.  Every argument is
 *   checked before anything is launched, so a rejected call has no side
 *   effects (the K/V buffer is untouched); xdit_last_error() then describes
 *   the problem.  NaN / Inf inputs are not checked and propagate.
 * A pointer may be NULL only where the tensor it stands for has no elements.
 * Tuning (environment, read at every call; results stay within the same
 *   tolerance, only the work decomposition changes): XDIT_ATTN_KERNEL = o2 |
 *   w32 | pp | w64 selects the bf16 attention decomposition, XDIT_ATTN_TILE =
 *   wide | narrow | quad | oct | six | strip the workgroup shape of unsplit
 *   launches (narrow, six: head_dim <= 72; oct: 72, 128), and
 *   XDIT_PARTITION = none | balanced the partition of *_split calls made with
 *   splits <= 0.  Unset, the library chooses.
 */
#ifndef XDIT_H
#define XDIT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { XDIT_BF16 = 0, XDIT_F32 = 1, XDIT_I64 = 2 }; /* XDIT_I64: positions only */

/* Norms of xdit_qk_norm_rope. */
enum { XDIT_NORM_NONE = 0, XDIT_NORM_RMS = 1, XDIT_NORM_LAYER = 2 };

/* Which elements of a head rotate together: neighbours (2i, 2i + 1), or
 * (i, i + rot_dim / 2). */
enum { XDIT_PAIRS_INTERLEAVED = 0, XDIT_PAIRS_HALF = 1 };

/* Scaling of a rotary table's frequencies (xdit_rope_table). */
enum { XDIT_ROPE_NONE = 0, XDIT_ROPE_LINEAR = 1, XDIT_ROPE_NTK = 2, XDIT_ROPE_RAMP = 3 };

/* Gradients of xdit_chunk_attn_bwd that are float32 sums to add to. */
enum { XDIT_ACCUM_DQ = 1, XDIT_ACCUM_DKV = 2 };

/* Upper bound on the axes of one rotary table. */
#define XDIT_MAX_AXES 4

/* Upper bound on the number of partials one xdit_lse_merge call accepts. */
#define XDIT_MAX_PARTIALS 64

/* Upper bound on the fresh row ranges of one xdit_patch_attn_ranges call. */
#define XDIT_MAX_RANGES 2

/* Upper bound on the key splits of one *_split call. */
#define XDIT_MAX_SPLITS 16

typedef enum {
    XDIT_OK = 0,
    XDIT_ERR_NULL = -1,        /* a required pointer is NULL                  */
    XDIT_ERR_DTYPE = -2,       /* unknown dtype                               */
    XDIT_ERR_SHAPE = -3,       /* negative or oversized dimension             */
    XDIT_ERR_RANGE = -4,       /* patch slice outside the buffer; bad n       */
    XDIT_ERR_LAYOUT = -5,      /* pointer not 16-byte aligned                 */
    XDIT_ERR_ALIAS = -6,       /* an output overlaps an input it must not     */
    XDIT_ERR_UNSUPPORTED = -7, /* head_dim not in {64, 72, 128}               */
    XDIT_ERR_HIP = -8          /* the HIP runtime refused a launch            */
} xdit_status;

/*
 * PipeFusion patch step (Section 4.1.2; buffer contents per Section 4.1.4).
 *
 * One layer's full-sequence K/V buffer holds, for every row, either fresh K/V
 * of the current diffusion step or stale K/V left by the previous step.  The
 * patch step first overwrites rows [patch_off, patch_off + patch_len) of both
 * planes with this patch's fresh K/V, then computes attention of the patch's
 * queries over all seq_len rows of the updated buffer, so the fresh slice is
 * seen by this call's own attention and by every later call.  Within one
 * diffusion step, calling this for patches 0..M-1 in order leaves patches
 * <= p fresh when patch p runs.
 *
 *   q        [B, patch_len, H, d]   queries of the patch's rows
 *   kv_buf   [2, B, seq_len, H, d]  the layer's K/V buffer; MUTATED in place:
 *                                   afterwards rows [off, off+len) equal
 *                                   fresh_k / fresh_v bit for bit and every
 *                                   other row is unchanged
 *   fresh_k, fresh_v [B, patch_len, H, d]
 *   out      [B, patch_len, H, d]   attention output
 * Requires 0 <= patch_off, 0 <= patch_len, patch_off + patch_len <= seq_len.
 * patch_len = 0 is a no-op.  out must not overlap any input; q, fresh_k and
 * fresh_v must not overlap kv_buf (the buffer is written while they are read).
 */
int xdit_patch_attn(const void* q, void* kv_buf, int64_t patch_off, int64_t patch_len,
                    const void* fresh_k, const void* fresh_v, void* out,
                    int64_t batch, int64_t seq_len, int64_t heads, int64_t head_dim,
                    int32_t dtype);

/*
 * The patch step in its general form (Sections 4.1.2 and 4.1.4): the fresh
 * K/V rows cover up to XDIT_MAX_RANGES disjoint row ranges of the buffer and
 * the queries are rows of their own.  Two uses come from the paper:
 *   - in-context conditioning (Section 4.1.2): the text tokens travel with
 *     patch 0, so that micro-step refreshes the patch's image rows and the
 *     text rows, and its queries are the rows of both;
 *   - hybrid parallelism (Section 4.1.4): a PipeFusion stage stores the K/V
 *     gathered over its sequence-parallel group while its queries are only
 *     the local shard, so every rank's buffer stays identical.
 * First rows [range_off[r], range_off[r] + range_len[r]) of both planes are
 * overwritten with the fresh rows (range 0's rows first, then range 1's),
 * then out = attention(q, updated K, updated V) and, if lse is not NULL, its
 * log-sum-exp.  xdit_patch_attn is the case of one range with q_len equal to
 * its length and no LSE.
 *
 *   q          [B, q_len, H, d]
 *   kv_buf     [2, B, seq_len, H, d]  MUTATED as above
 *   n_ranges   0 .. XDIT_MAX_RANGES; range_off / range_len are HOST arrays of
 *              n_ranges entries, each range inside [0, seq_len), pairwise
 *              disjoint (empty ranges allowed)
 *   fresh_k, fresh_v [B, F, H, d], F = sum of range_len
 *   out        [B, q_len, H, d]
 *   lse        [B, H, q_len] float32, or NULL
 * q_len = 0 performs only the update; F = 0 is plain attention over the
 * buffer.  out and lse must not overlap any input or each other; q and the
 * fresh rows must not overlap kv_buf.
 */
int xdit_patch_attn_ranges(const void* q, int64_t q_len, void* kv_buf, int32_t n_ranges,
                           const int64_t* range_off, const int64_t* range_len, const void* fresh_k,
                           const void* fresh_v, void* out, float* lse, int64_t batch,
                           int64_t seq_len, int64_t heads, int64_t head_dim, int32_t dtype);

/*
 * Sequence-parallel chunk step (Section 4.1.1: SP-Ring computes attention as
 * a parallel FlashAttention over K/V sub-blocks exchanged peer to peer).
 * Attention of q over one K/V chunk, returning the normalised partial output
 * and its log-sum-exp, which xdit_lse_merge combines across chunks.  With the
 * whole sequence as the chunk this is plain full attention.
 *
 *   q    [B, q_len, H, d]
 *   k, v [B, kv_len, H, d]
 *   out  [B, q_len, H, d]
 *   lse  [B, H, q_len] float32, or NULL to skip it
 * kv_len = 0 gives out = 0 and lse = -inf.  q_len = 0 is a no-op.
 * out and lse must not overlap q, k or v (or each other).
 */
int xdit_chunk_attn(const void* q, const void* k, const void* v, void* out, float* lse,
                    int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                    int64_t head_dim, int32_t dtype);

/*
 * Ring step with the merge fused in (Section 4.1.1: SP-Ring accumulates the
 * partial attention of each K/V sub-block it receives).  Attention of q over
 * one K/V chunk is merged into the running output and log-sum-exp of the
 * chunks before it:
 *   L = ln(e^{lse} + e^{lse_c}),  out = e^{lse - L} * out + e^{lse_c - L} * o_c
 * with (o_c, lse_c) this chunk's attention; out and lse are read, then
 * overwritten with the merged state.  A running lse of -inf marks an empty
 * state: its out is ignored (it may hold anything, NaN included), so a ring
 * starts from lse = -inf or from xdit_chunk_attn's result.  After every chunk
 * of the sequence, out and lse equal attention over the whole sequence.
 * Arguments and requirements as for xdit_chunk_attn, except that lse is
 * required.  The running out is stored in the I/O dtype after every step.
 */
int xdit_chunk_attn_accum(const void* q, const void* k, const void* v, void* out, float* lse,
                          int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                          int64_t head_dim, int32_t dtype);

/*
 * Log-sum-exp merge of n chunk partials into attention over the union of the
 * chunks (Section 4.1.1: the sharded computation gives the serial result):
 *   M = max_r lse_r,  L = M + ln sum_r exp(lse_r - M),
 *   out = sum_r exp(lse_r - L) * outs[r]      (float32 arithmetic)
 * A partial with lse = -inf (an empty chunk) has weight 0; if all are -inf,
 * out = 0 and L = -inf.
 *
 *   outs    HOST array of n device pointers, each [B, q_len, H, d] (dtype)
 *   lses    HOST array of n device pointers, each [B, H, q_len] float32
 *   n       1 <= n <= XDIT_MAX_PARTIALS
 *   out     [B, q_len, H, d]; may be exactly outs[r] (in-place), must not
 *           otherwise overlap a partial
 *   lse_out [B, H, q_len] float32 merged L, or NULL; must not overlap lses
 */
int xdit_lse_merge(const void* const* outs, const float* const* lses, int32_t n, void* out,
                   float* lse_out, int64_t batch, int64_t q_len, int64_t heads,
                   int64_t head_dim, int32_t dtype);

/*
 * Key-split forms of xdit_chunk_attn and xdit_patch_attn_ranges, for launches
 * whose query tiles (128 rows each, per batch and head) leave CUs of the 256
 * idle: too few query tiles, or a last round of workgroups that is nearly
 * empty.  The K/V sweep of a query tile is cut into consecutive parts that
 * run as separate workgroups; each part writes its partial output and
 * log-sum-exp (float32) into the workspace, and a fix-up launch combines the
 * parts of each cut sweep by the log-sum-exp merge of Section 4.1.1 (the
 * same arithmetic as xdit_lse_merge) into out and lse.  The results equal
 * the unsplit call's up to float32 rounding of the merge.
 *
 *   splits     1 .. XDIT_MAX_SPLITS, or <= 0 to let the library choose
 *              splits > 1: every sweep is cut into `splits` even parts;
 *              1: the unsplit call;
 *              <= 0: the library's choice from a time model of the launch:
 *              no cut, every sweep cut into s even parts (few query tiles),
 *              or the query tiles of the full rounds of workgroups swept
 *              whole and each of the r left over cut into min(16, 256 / r)
 *              parts (a nearly empty last round); a cut is taken only when
 *              the model saves at least 10 %
 *   workspace  device memory of at least xdit_split_workspace_bytes(...)
 *              bytes for the same sizes and splits, 256-byte aligned, not
 *              overlapping any argument; unused (may be NULL) when no cut
 *              happens.  Its contents on entry do not matter.
 * xdit_split_workspace_bytes returns 0 when the sizes lead to no cut, -1 for
 * sizes or splits the calls reject.  float32 calls, and calls whose sweeps
 * hold one K/V tile or less (128 keys at d <= 72, 64 at d = 128), run
 * unsplit.  Other arguments as for the unsplit calls.  The sweep and the
 * fix-up are two launches on the calling thread's stream.
 * xdit_chunk_attn_accum_split is the same for the ring step
 * xdit_chunk_attn_accum: the fix-up merges each cut sweep's result into the
 * running (out, lse) as the unsplit call does.
 */
int64_t xdit_split_workspace_bytes(int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                                   int64_t head_dim, int32_t dtype, int32_t splits);
int xdit_chunk_attn_split(const void* q, const void* k, const void* v, void* out, float* lse,
                          int32_t splits, void* workspace, int64_t workspace_bytes, int64_t batch,
                          int64_t q_len, int64_t kv_len, int64_t heads, int64_t head_dim,
                          int32_t dtype);
int xdit_chunk_attn_accum_split(const void* q, const void* k, const void* v, void* out, float* lse,
                                int32_t splits, void* workspace, int64_t workspace_bytes,
                                int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                                int64_t head_dim, int32_t dtype);
int xdit_patch_attn_split(const void* q, int64_t q_len, void* kv_buf, int32_t n_ranges,
                          const int64_t* range_off, const int64_t* range_len, const void* fresh_k,
                          const void* fresh_v, void* out, float* lse, int32_t splits,
                          void* workspace, int64_t workspace_bytes, int64_t batch, int64_t seq_len,
                          int64_t heads, int64_t head_dim, int32_t dtype);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * operation as xdit_chunk_attn_split, with the partial slots of cut sweeps
 * kept in a fixed device array inside the library instead of a caller
 * workspace.  Arguments and results as for xdit_chunk_attn_split without
 * the workspace.
 *   Limit: the partition's slots (xdit_split_workspace_bytes for the same
 *   sizes and splits) must fit in xdit_noalloc_scratch_bytes() bytes
 *   (16 MiB: the Flux 2048px share, 4224 queries over a 4224-key chunk with
 *   24 heads of 128, needs 15.9 MB); larger partitions are rejected with
 *   XDIT_ERR_RANGE before anything is launched.
 *   The array is one per GPU, allocated when the library is loaded onto it
 *   and held until the process ends; its device address is looked up on the
 *   first call on each device.  Every call on a GPU uses that GPU's array:
 *   calls that overlap on one GPU (other streams, other threads) race on it
 *   and must be ordered by the caller.  No call allocates or frees memory.
 */
int xdit_chunk_attn_split_noalloc(const void* q, const void* k, const void* v, void* out, float* lse,
                                  int32_t splits, int64_t batch, int64_t q_len, int64_t kv_len,
                                  int64_t heads, int64_t head_dim, int32_t dtype);
int64_t xdit_noalloc_scratch_bytes(void);

/*
 * The update half of the patch step on its own (Section 4.1.2): copy the
 * fresh K/V rows into rows [patch_off, patch_off + patch_len) of kv_buf,
 * bit for bit, leaving every other row unchanged.  xdit_patch_attn performs
 * the same update itself; this entry point serves callers that fill the
 * buffer without attending (e.g. storing K/V received by SP, Section 4.1.4).
 * Arguments and requirements as for xdit_patch_attn.
 */
int xdit_kv_update(void* kv_buf, int64_t patch_off, int64_t patch_len, const void* fresh_k,
                   const void* fresh_v, int64_t batch, int64_t seq_len, int64_t heads,
                   int64_t head_dim, int32_t dtype);

/*
 * One PipeFusion stage micro-step at one attention layer (Section 4.1.2: a
 * device runs each patch through its stage's layers; Section 3: QKV
 * projections come before self-attention, whose output is projected back):
 *
 *   q = x wq,  k = x wk,  v = x wv      (projections of the patch's rows)
 *   the patch step of xdit_patch_attn with fresh K/V = (k, v), output o
 *   y = o wo
 *
 *   x          [B, patch_len, C]        the patch's hidden states, C = hidden
 *   wq, wk, wv [C, H*d]                 row-major, so q[b, i] = x[b, i] wq
 *   wo         [H*d, C]
 *   kv_buf     [2, B, seq_len, H, d]    MUTATED as by xdit_patch_attn: rows
 *                                       [patch_off, patch_off + patch_len)
 *                                       take k and v bit for bit
 *   q, k, v, o [B, patch_len, H, d]     caller-owned intermediates, written
 *   y          [B, patch_len, C]        output
 * bf16 only (XDIT_ERR_UNSUPPORTED otherwise); the GEMMs (hipBLASLt) and the
 * attention accumulate in float32 and round each result to bf16.  No
 * biases, norms or gates.  No output may overlap another buffer or any
 * input; other requirements as for xdit_patch_attn; 1 <= hidden <= 65536.
 * The library allocates nothing itself; hipBLASLt keeps one handle per
 * device and per-shape plans from the first call on (its own host and
 * device memory).  The first call of each shape times hipBLASLt's candidate
 * algorithms on its own operands and synchronises the calling stream (so it
 * must not run under graph capture); later calls only launch.
 * XDIT_ERR_HIP if hipBLASLt refuses a GEMM.  Five launches on the calling
 * thread's stream.
 */
int xdit_stage_step(const void* x, const void* wq, const void* wk, const void* wv, const void* wo,
                    void* kv_buf, int64_t patch_off, int64_t patch_len, void* q, void* k, void* v,
                    void* o, void* y, int64_t batch, int64_t seq_len, int64_t heads,
                    int64_t head_dim, int64_t hidden, int32_t dtype);

/*
 * Gradients of chunk attention.  With s_ij = (q_i . k_j) / sqrt(d):
 *   P_ij = exp(s_ij - lse_i),  D_i = dout_i . out_i - dlse_i
 *   dv_j = sum_i P_ij dout_i
 *   dk_j = sum_i P_ij (dout_i . v_j - D_i) q_i / sqrt(d)
 *   dq_i = sum_j P_ij (dout_i . v_j - D_i) k_j / sqrt(d)
 * out and lse are what xdit_chunk_attn gave for these chunk's keys, dlse the
 * gradient of that lse: the chunk's partial is then merged further.  Or out
 * and lse are those of all chunks of a sequence (merged, or a ring's running
 * state) with dout their gradient: the call then gives this chunk's dk and dv
 * and its part of dq, and the parts of all chunks add up (XDIT_ACCUM_DQ).
 *   q, out, dout [B, q_len, H, d];  k, v [B, kv_len, H, d]
 *   lse, dlse    [B, H, q_len] float32; dlse may be NULL (zeros)
 *   dq           [B, q_len, H, d], dk, dv [B, kv_len, H, d], written; with
 *                XDIT_ACCUM_DQ dq, with XDIT_ACCUM_DKV dk and dv, is a float32
 *                tensor that the gradient is added to (dk and dv travel with
 *                their chunk through the ring)
 *   workspace    xdit_chunk_attn_bwd_workspace_bytes(...) bytes, 256-byte
 *                aligned, overlapping nothing; its contents on entry do not
 *                matter.  Calls that overlap in time need one each.
 * A row whose lse is -inf (it met no key) has no part in any gradient.  Its out
 * and dlse may hold anything; its q and dout are multiplied by zeros, so they
 * must be finite, and their products with k and v too.  kv_len = 0 gives dq = 0,
 * q_len = 0 gives dk = dv = 0.  Sums are float32 and their order is fixed: the
 * same call gives the same bits.  bf16 calls round P and the scores' gradient to
 * bf16 as operands of the matrix cores.  No output overlaps another tensor.
 */
int64_t xdit_chunk_attn_bwd_workspace_bytes(int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads,
                                            int64_t head_dim, int32_t dtype);
int xdit_chunk_attn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                        const void* dout, const float* dlse, void* dq, void* dk, void* dv, int32_t accum,
                        void* workspace, int64_t workspace_bytes, int64_t batch, int64_t q_len,
                        int64_t kv_len, int64_t heads, int64_t head_dim, int32_t dtype);

/*
 * The table of a rotary position embedding: of every row, the cosines and
 * sines of its pairs' angles.  A row has a position on each of n_axes axes
 * (text, height and width of an image, time of a video); axis a turns
 * dims[a] / 2 pairs, the axes' pairs one after another:
 *   angle = position * w,  w = theta^(-2 i / dims[a]),  i = 0 .. dims[a]/2 - 1
 * Angles are formed and reduced in 64 bits: an angle of size a is off by at most
 * 4 a * 2^-52 (on the slope of a ramp about three times that) before the table is
 * rounded to float32.
 *   pos      [n, n_axes]  int64 (XDIT_I64) or float32 (XDIT_F32: fractional
 *                         positions of a grid that is stretched or cropped)
 *   dims     HOST array of n_axes even positive numbers, at most 256 in all
 *   scaling  HOST, or NULL for none:
 *     XDIT_ROPE_LINEAR  w / factor
 *     XDIT_ROPE_NTK     theta * factor^(dims[a] / (dims[a] - 2)) in theta's
 *                       place (every dims[a] > 2): the fastest pair keeps its
 *                       frequency, the slowest is divided by factor
 *     XDIT_ROPE_RAMP    by the turns that a pair makes over the original
 *                       length, t = orig_len * w / (2 pi): w where t >= fast,
 *                       w / factor where t <= slow, linear in t between
 *                       (fast > slow)
 *     magnitude         times every cosine and sine, whatever the kind
 *   cos, sin [n, sum(dims) / 2] float32
 * n = 0 is a no-op.  cos and sin must not overlap each other or pos.
 */
typedef struct {
    int32_t kind; /* XDIT_ROPE_* */
    double factor, orig_len, fast, slow, magnitude;
} xdit_rope_scaling;
int xdit_rope_table(const void* pos, int32_t pos_dtype, int64_t n, int32_t n_axes, const int32_t* dims,
                    double theta, const xdit_rope_scaling* scaling, float* cos, float* sin);

/*
 * Rotation of heads by position: pair (x0, x1) number i of the first rot_dim
 * elements of each head becomes (x0 c - x1 s, x1 c + x0 s) with c, s of the
 * row's column i; the other elements are copied.  transpose != 0 turns back
 * by the same angles: the gradient of the rotation (table magnitudes apply
 * again, as the gradient has them).
 *   x, y     [batch, tokens, heads, head_dim]; y may be exactly x (the same
 *            pointer and strides), must not overlap it otherwise
 *   strides  HOST array of 2 x 3: the batch, token and head strides of x and
 *            y in elements (multiples of 16 bytes; the elements of a head are
 *            contiguous), or NULL for dense tensors
 *   cos, sin [tokens, rot_dim / 2] float32, or with table_per_batch != 0
 *            [batch, tokens, rot_dim / 2]; dense, as xdit_rope_table writes them
 *   rot_dim  a multiple of 8, at most head_dim
 *   layout   XDIT_PAIRS_*
 * Products and sums are float32, rounded once.
 */
int xdit_rope(const void* x, const float* cos, const float* sin, void* y, const int64_t* strides,
              int64_t batch, int64_t tokens, int64_t heads, int64_t head_dim, int64_t rot_dim,
              int32_t table_per_batch, int32_t layout, int32_t transpose, int32_t dtype);

/*
 * What a layer does to its queries and keys between their projection and the
 * attention: each head is normalised over its head_dim elements and rotated.
 *   RMS    n = x / sqrt(mean(x^2) + eps)
 *   LAYER  n = (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps)
 *   NONE   out = rotation(x), no weights; rot_dim > 0
 *   out = rotation(n * w + b)
 * Queries and keys have weights and biases of their own.  Statistics and
 * products are float32, rounded once.
 */
typedef struct {
    int64_t batch, tokens, q_heads, k_heads, head_dim; /* k_heads = 0: no keys */
    int32_t dtype;           /* of queries, keys and their gradients */
    int32_t norm;            /* XDIT_NORM_* */
    double eps;
    const void *wq, *wk;     /* [head_dim], or NULL for ones */
    const void *bq, *bk;     /* [head_dim], or NULL for zeros; LAYER only */
    int32_t weight_dtype;    /* of the four: XDIT_BF16 or XDIT_F32 */
    int32_t layout;          /* XDIT_PAIRS_* */
    int64_t rot_dim;         /* 0: no rotation (cos and sin NULL) */
    const float *cos, *sin;  /* as for xdit_rope */
    int32_t table_per_batch;
    const int64_t* strides;  /* HOST: batch, token and head strides in elements
                                of each tensor of the call, in the order of its
                                arguments, or NULL for dense tensors */
} xdit_qk;

/*
 *   q, q_out [batch, tokens, q_heads, head_dim]
 *   k, k_out [batch, tokens, k_heads, head_dim]
 * q_out may be exactly q, and k_out exactly k (the same pointer and strides);
 * otherwise outputs overlap nothing.  Interleaved views of one buffer (a fused
 * projection's) count by their elements, where these keep to different parts of
 * some stride.  strides: 4 x 3 (q, k, q_out, k_out).
 */
int xdit_qk_norm_rope(const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out);

/*
 * Gradients of xdit_qk_norm_rope, from its inputs q and k (not kept
 * normalised) and the gradients of its outputs.
 *   dq_out, dk_out  gradients of q_out and k_out
 *   dq, dk          of q and k; dq may be exactly dq_out or q, dk exactly
 *                   dk_out or k, otherwise they overlap nothing
 *   dwq, dwk, dbq, dbk  [head_dim] float32 gradients of weights and biases,
 *                   summed over batch, tokens and heads in float32 in a fixed
 *                   order; NULL where not wanted (dbq, dbk: LAYER only)
 *   workspace       xdit_qk_norm_rope_bwd_workspace_bytes(...) bytes, 16-byte
 *                   aligned, overlapping nothing; unused (may be NULL) when no
 *                   weight or bias gradient is wanted
 * strides: 6 x 3 (q, k, dq_out, dk_out, dq, dk).  With no rows the weights'
 * and biases' gradients are zero.
 */
int64_t xdit_qk_norm_rope_bwd_workspace_bytes(int64_t batch, int64_t tokens, int64_t q_heads, int64_t k_heads,
                                              int64_t head_dim, int32_t dtype);
int xdit_qk_norm_rope_bwd(const xdit_qk* p, const void* q, const void* k, const void* dq_out,
                          const void* dk_out, void* dq, void* dk, float* dwq, float* dwk, float* dbq,
                          float* dbk, void* workspace, int64_t workspace_bytes);

/*
 * xdit_stage_step with the queries and keys normalised and rotated between
 * their projection and the attention:
 *   q = x wq,  k = x wk,  v = x wv
 *   q, k = xdit_qk_norm_rope(qk, q, k), in place
 *   the patch step with fresh K/V = (k, v), output o
 *   y = o wo
 * qk describes the patch's rows: batch, tokens = patch_len, q_heads = k_heads
 * = heads, head_dim and dtype as in the call, dense tensors (strides NULL); its
 * table holds the patch's rows (row patch_off on of the sequence's).  q and k
 * hold the normalised and rotated rows afterwards, as the buffer does.  Other
 * arguments and requirements as for xdit_stage_step; no output may overlap the
 * weights or the table.  Six launches.
 */
int xdit_stage_step_qk(const xdit_qk* qk, const void* x, const void* wq, const void* wk, const void* wv,
                       const void* wo, void* kv_buf, int64_t patch_off, int64_t patch_len, void* q,
                       void* k, void* v, void* o, void* y, int64_t batch, int64_t seq_len,
                       int64_t heads, int64_t head_dim, int64_t hidden, int32_t dtype);

/* Stream for the calling thread's later launches (a hipStream_t; NULL = the
 * default stream).  Always returns XDIT_OK. */
int xdit_set_stream(void* stream);
void* xdit_get_stream(void);

/* Message describing the calling thread's most recent failure ("" if none).
 * Valid until that thread's next call into the library. */
const char* xdit_last_error(void);

/* Library version string. */
const char* xdit_version(void);

#ifdef __cplusplus
}
#endif

#endif /* XDIT_H */
