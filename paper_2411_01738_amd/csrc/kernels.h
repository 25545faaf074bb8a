// Internal interface between the C-ABI layer (xdit_api.cpp) and the HIP
// kernels.  Shapes have been validated before any of these is called.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xdit {

// One attention launch: chunk attention (fresh_k == nullptr) or a fused
// PipeFusion patch step: K/V rows in the fresh ranges [off0, off0+len0) and
// [off1, off1+len1) come from fresh_k/fresh_v (rows 0..len0-1, then
// len0..len0+len1-1) and are written back into the buffer planes wk/wv.
struct AttnParams {
    const void* q;        // [B, Nq, H, D]
    const void* k;        // [B, Nk, H, D]  (patch: K plane of the buffer)
    const void* v;        // [B, Nk, H, D]  (patch: V plane of the buffer)
    const void* fresh_k;  // [B, len0 + len1, H, D] or nullptr
    const void* fresh_v;
    void* wk;             // patch write-back target planes (== k / v) or nullptr
    void* wv;
    void* out;            // [B, Nq, H, D]
    float* lse;           // [B, H, Nq] or nullptr
    int B, H, Nq, Nk, D;
    int off0, len0;       // first fresh range
    int off1, len1;       // second fresh range (len1 == 0: none); disjoint from the first
    int accum;            // merge into the running (out, lse) instead of overwriting them
    // Work partition (bf16 only; 128-row query tiles).  parts = 0: one
    // workgroup per query tile.  parts > 0: `whole` workgroups (a multiple
    // of 8) sweep the first `whole` query tiles whole, and the (query tile,
    // K/V tile) units of the others are cut into `parts` contiguous ranges,
    // one workgroup each; partials of cut sweeps go to `part`
    // (kPartSlotRows * (D + 1) floats per slot; slots 0..parts-1, and
    // parts..2*parts-1 when ranges may cross query tiles) and a fix-up
    // launch merges them.
    int64_t whole, parts;
    float* part;
};

struct MergeParams {
    const void* const* outs;  // host array of n device pointers
    const float* const* lses; // host array of n device pointers
    int n;
    void* out;
    float* lse_out;           // or nullptr
    int B, Nq, H, D;
};

// Copy fresh rows [fbase, fbase+len) of fresh_k/fresh_v [B, frows, H, D]
// into rows [off, off+len) of both buffer planes.
struct UpdateParams {
    void* kv_buf;             // [2, B, N, H, D]
    const void* fresh_k;      // [B, frows, H, D]
    const void* fresh_v;
    int B, N, H, D, off, len;
    int frows, fbase;
    int esize;                // bytes per element
};

// Rows of one head, [B, N, H, D] with the strides (in elements) of any order.
struct HeadView {
    const void* p;
    int64_t sb, st, sh;  // batch, token, head
};

// Queries (side 0) and keys (side 1) normalised per head and rotated, or the
// gradients of that.  A side with no heads is absent.
struct NormRopeSide {
    HeadView x, g, y;    // input; gradient of the output (backward); output, or the input's gradient
    const void* w;       // [D] weight and bias, or nullptr
    const void* b;
    float* dw;           // [D] gradients of weight and bias, or nullptr
    float* db;
    int heads;
};

struct NormRopeParams {
    NormRopeSide side[2];
    const float* cos;    // [N, rot / 2] (table_batch = 0) or [B, N, rot / 2]
    const float* sin;
    int64_t table_batch; // elements between the tables of two batches
    int B, N, D, rot;
    int bf16, weight_bf16;
    int norm;            // XDIT_NORM_*
    int half;            // pairs (i, i + rot / 2) instead of (2i, 2i + 1)
    int transpose;       // rotate by the negative angles (no norm)
    float eps;
    float* part;         // backward: workspace of norm_rope_bwd_partials
};

struct RopeTableParams {
    const void* pos;     // [n, axes], int64 or float32
    int pos_i64;
    int axes;
    int dims[4];         // rotated dims of each axis, even
    double theta, factor, orig_len, fast, slow, magnitude;
    int scaling;         // XDIT_ROPE_*
    float* cos;          // [n, sum(dims) / 2]
    float* sin;
    int64_t n;
};

// Gradients of one chunk's attention (O and LSE possibly of more chunks).
struct AttnBwdParams {
    const void *q, *k, *v;       // [B, Nq or Nk, H, D]
    const void *out, *dout;      // [B, Nq, H, D]
    const float *lse, *dlse;     // [B, H, Nq]; dlse or nullptr
    void *dq, *dk, *dv;
    int B, H, Nq, Nk, D, bf16;
    int accum_q, accum_kv;       // dq; dk and dv: float32 sums to add to
    int q_splits, kv_splits;     // parts that a sweep is cut into, summed by launch_bwd_join
    float* rows;                 // workspace: [B * H][2][Nq], filled by launch_bwd_rows
    float *q_part, *kv_part;     // workspace of cut sweeps: [splits][B, N, H, D], dk's and then dv's
};

constexpr int kMaxPartials = 64;
constexpr int kPartSlotRows = 128;  // query rows of a partitioned launch's tile
constexpr int kMaxSweepParts = 17;  // most partition ranges one sweep may meet

hipError_t launch_attn_bf16(const AttnParams& p, hipStream_t s);
// Time of an unpartitioned bf16 launch of more 128-row query tiles than CUs,
// for the partition's model (pick_parts in xdit_api.cpp) and in its units;
// six_sweep: one round of 192-row tiles.  Quad and oct cost 1.9 times what
// pick_shape's model says (2.1-2.2 us and 2.4 us per unit of that at d = 64
// and 72, the partition's units 1.13 and 1.3 us); 192-row tiles at d = 64
// take 5 % more per round when there are several.
double unsplit_cost(int D, int64_t bh, int64_t Nq, int64_t Nk, double six_sweep);
// The second launch of a partitioned bf16 attention (128-row query tiles,
// sweeps of T K/V tiles): merges the partials of the cut sweeps into out
// and lse.
hipError_t launch_attn_fixup(const AttnParams& p, int q_tiles, int T, hipStream_t s);
// bf16 attention with 64 query rows per wave and one wave per SIMD (head
// dim 128); hipErrorNotSupported for shapes it does not take.
hipError_t launch_attn_w64(const AttnParams& p, hipStream_t s);
hipError_t launch_attn_f32(const AttnParams& p, hipStream_t s);
hipError_t launch_merge_bf16(const MergeParams& p, hipStream_t s);
hipError_t launch_merge_f32(const MergeParams& p, hipStream_t s);
hipError_t launch_kv_update(const UpdateParams& p, hipStream_t s);
hipError_t launch_norm_rope(const NormRopeParams& p, hipStream_t s);
// The gradients of the norm and rotation: dx per head (side[].y), and the
// weights' and biases' gradients by way of p.part
// (norm_rope_bwd_partials floats).
hipError_t launch_norm_rope_bwd(const NormRopeParams& p, hipStream_t s);
int64_t norm_rope_bwd_partials(int64_t rows, int heads0, int heads1, int D, bool bf16);
// Into how many parts the sweeps of a gradient call are cut, and the resident
// rows of a workgroup.
struct BwdSplits {
    int q, kv, rows;
};
BwdSplits bwd_splits(int64_t bh, int64_t Nq, int64_t Nk, int D, bool bf16);
hipError_t launch_bwd_rows(const AttnBwdParams& p, hipStream_t s);
// both sweeps: dq, dk and dv, or the partials of the cut ones
hipError_t launch_attn_bwd_bf16(const AttnBwdParams& p, hipStream_t s);
hipError_t launch_attn_bwd_f32(const AttnBwdParams& p, hipStream_t s);
// the sums of the cut sweeps' partials (nothing to do where none is cut)
hipError_t launch_bwd_join(const AttnBwdParams& p, hipStream_t s);
hipError_t launch_rope_table(const RopeTableParams& p, hipStream_t s);

}  // namespace xdit
