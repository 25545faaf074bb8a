// What a layer does to its queries and keys between their projection and the
// attention: a norm over each head's D values and the rotation of pairs of
// them by the token's position, in one pass, and the gradients of both; the
// rotation alone; and the table of the angles' cosines and sines.
//
// Per head x of D values, with weight w and bias b (or none):
//   rms    n = x r,             r = 1 / sqrt(mean(x^2) + eps)
//   layer  n = (x - mean(x)) r, r = 1 / sqrt(mean((x - mean(x))^2) + eps)
//   y = R (n w + b), R rotating pair i of the first `rot` dims by angle i:
//   y0 = x0 c - x1 s, y1 = x1 c + x0 s, pairs (2i, 2i + 1) or (i, i + rot/2).
// Backward, with g the gradient of y and h = R^T g (the same rotation with -s):
//   db = sum h, dw = sum h n over all rows,
//   dx = r (h w - n mean(h w n) [- mean(h w) for the layer norm]).
// All of it in float32, rounded once at the store.
//
// What bounds it: memory.  Each head is read and written once; the tables are
// read once per token and batch of heads.  bf16, where a large copy reaches 5.1
// TB/s: RMS norms and rotation of 4224 tokens, 24 + 24 heads of 128, 22.6 us (4.7
// TB/s; a copy of as much 21); layer norms and rotation of 17550 tokens, 48 + 48
// heads of 64, 78 us (5.5 TB/s), their gradients 127 us (5.1 TB/s), the rotation of
// one such tensor 42 us (5.1 TB/s).  float32: 41, 162, 267 and 83 us.
//
// Work: a lane holds 2 V values of a head, both elements of each of its
// pairs, so the rotation needs no other lane: the runs at V p and D / 2 + V p for
// neighbouring pairs (in one run they took 7 % more at D = 128), at V p and
// rot / 2 + V p for pairs half a rotation apart.  D / (2 V) lanes hold a head and
// share its sums; a wave holds 64 / that many heads (7 at D = 72, one lane idle)
// and loads the angles of a token once for up to kBatch heads of a lane; where it
// takes further tokens, these are of the same heads, so that weights stay in
// registers.  Weights come in wide loads: element by element they took 8 % of a
// long forward pass.
#include "kernels.h"

#include <math.h>

namespace xdit {
namespace {

#include "attn_common.h"

constexpr int kWaves = 4;   // waves per workgroup, a token each at a time
constexpr int kBatch = 4;   // heads of a lane per token, their loads issued together
// Pairs of neighbours: the runs of V from V p on of both halves of the head, so
// that a load or store of a head's lanes is one piece; at d = 72, whose V is 4, one
// run of 2 V (the pieces would be of 8 bytes).
template <int D>
constexpr bool kSplit = D != 72;
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct NrSide {
    const char* x;
    const char* g;
    char* y;
    int64_t xb, xt, xh, gb, gt, gh, yb, yt, yh;  // byte strides
    const void* w;
    const void* b;
    int heads;
    int grads;  // bit 0: weight, bit 1: bias
};

struct NrArgs {
    NrSide side[2];
    int nb0;  // batches of heads of side 0 (blockIdx.y below it)
    const float* cos;
    const float* sin;
    int64_t table_batch;
    uint32_t rows, N;
    int rot, half, weight_bf16;
    float sgn, eps;
    float* part;       // partials of side 0: weight's, then bias's; then side 1's
    int64_t part1;     // first partial (in floats) of side 1
};

__device__ __forceinline__ float bf16f(uint32_t lo16) { return __uint_as_float(lo16 << 16); }

// A run of V values of type T as it lies in memory, and to float32
template <typename T, int V>
struct Run;
template <>
struct Run<uint16_t, 8> {
    typedef u32x4 Raw;
};
template <>
struct Run<uint16_t, 4> {
    typedef u32x2 Raw;
};
template <>
struct Run<float, 4> {
    typedef f32x4 Raw;
};
template <typename T, int V>
__device__ __forceinline__ void unpack(const typename Run<T, V>::Raw& r, float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = r[e];
    } else {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            f[2 * e] = bf16f(r[e] & 0xffffu);
            f[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
        }
    }
}
// float32 values rounded to nearest even and stored
template <typename T, int V>
__device__ __forceinline__ void store_run(char* p, const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *(f32x4*)(p + 4 * i) = f32x4{f[i], f[i + 1], f[i + 2], f[i + 3]};
    } else if constexpr (V == 8) {
        *(u32x4*)p = u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                           pack_bf16x2(f[6], f[7])};
    } else {
        *(u32x2*)p = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
    }
}
// V weights from element e on, of either type (in wide loads where they are
// aligned so); `fill` where there are none
template <int V>
__device__ __forceinline__ void load_weights(const void* w, int is_bf16, int e, float fill, float* f) {
    const char* p = (const char*)w + (is_bf16 ? 2 : 4) * e;
    if (w == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = fill;
    } else if (((uintptr_t)w & 15) == 0) {
        if (is_bf16) {
            unpack<uint16_t, V>(*(const typename Run<uint16_t, V>::Raw*)p, f);
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 4) unpack<float, 4>(*(const f32x4*)(p + 4 * i), f + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = is_bf16 ? bf16f(((const uint16_t*)p)[i]) : ((const float*)p)[i];
    }
}

// Sum over the L lanes of a head, the same bits in each of them.
template <int L>
__device__ __forceinline__ float head_sum(float v, int lane, int p) {
    if constexpr (L == 9) {  // by threes
        const int t = lane - p % 3;
        v = __shfl(v, t) + __shfl(v, t + 1) + __shfl(v, t + 2);
        const int h = lane - p;
        return __shfl(v, h) + __shfl(v, h + 3) + __shfl(v, h + 6);
    } else {
#pragma unroll
        for (int o = 1; o < L; o *= 2) v += __shfl_xor(v, o);
        return v;
    }
}

// A lane's pairs i below t1 (i < V / 2) or t2 (the others) rotated by (c, s):
// pairs of neighbours, or of the runs a and b = a + V.  The others stay as they
// are, whatever stands beside them.
template <int V>
__device__ __forceinline__ void rotate(float* x, const float* c, const float* s, int t1, int t2, bool half) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float a = half ? x[i] : x[2 * i], b = half ? x[V + i] : x[2 * i + 1];
        const bool on = i < (i < V / 2 ? t1 : t2);
        const float ya = on ? a * c[i] - b * s[i] : a, yb = on ? b * c[i] + a * s[i] : b;
        if (half) {
            x[i] = ya;
            x[V + i] = yb;
        } else {
            x[2 * i] = ya;
            x[2 * i + 1] = yb;
        }
    }
}

template <typename T, int D, int V, int NORM, bool BWD, bool HALF>
__global__ __launch_bounds__(64 * kWaves) void norm_rope_kernel(NrArgs a) {
    constexpr int L = D / (2 * V), G = 64 / L, ES = sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int p = lane % L, grp = lane / L;
    const bool second = (int)blockIdx.y >= a.nb0;
    const NrSide& sd = a.side[second];
    const int head0 = ((int)blockIdx.y - (second ? a.nb0 : 0)) * kBatch * G + grp;
    const int rp = a.rot / 2;

    // this lane's two runs of V elements; its pair i is that of number p1 + i (i <
    // V / 2) or p2 + i, and turns if i is below t1 or t2 (steps of V / 2 pairs)
    constexpr bool SPLIT = !HALF && kSplit<D>;
    const int col = V * p;
    int oa = SPLIT ? col : 2 * col, ob = SPLIT ? D / 2 + col : oa + V;
    if (HALF) {
        if (col < rp) oa = col, ob = rp + col;
        else oa = a.rot + 2 * (col - rp), ob = oa + V;
    }
    const int p1 = SPLIT ? col / 2 : col, p2 = SPLIT ? D / 4 + col / 2 - V / 2 : col;
    const int t1 = rp - p1, t2 = rp - p2;
    float w[2 * V], bias[2 * V];
    if constexpr (NORM != 0) {
        load_weights<V>(sd.w, a.weight_bf16, oa, 1.f, w);
        load_weights<V>(sd.w, a.weight_bf16, ob, 1.f, w + V);
        if constexpr (!BWD) {
            load_weights<V>(sd.b, a.weight_bf16, oa, 0.f, bias);
            load_weights<V>(sd.b, a.weight_bf16, ob, 0.f, bias + V);
        }
    }
    float dw[2 * V], db[2 * V];
    if constexpr (BWD)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) dw[i] = db[i] = 0.f;

    for (uint32_t row = blockIdx.x * kWaves + wave; row < a.rows; row += gridDim.x * kWaves) {
        const uint32_t b = row / a.N, n = row - b * a.N;
        // the loads of a token's angles and of a lane's heads together, as they lie in memory
        f32x4 cv[V / 4], sv[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            cv[i] = sv[i] = f32x4{};
            const int64_t at = b * a.table_batch + (int64_t)n * rp + 4 * i;
            if constexpr (SPLIT && V == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (2 * h < (h == 0 ? t1 : t2)) {
                        const f32x2 cc = *(const f32x2*)(a.cos + at + (h == 0 ? p1 : p2) + 2 * h);
                        const f32x2 ss = *(const f32x2*)(a.sin + at + (h == 0 ? p1 : p2) + 2 * h);
                        cv[i][2 * h] = cc[0], cv[i][2 * h + 1] = cc[1];
                        sv[i][2 * h] = ss[0], sv[i][2 * h + 1] = ss[1];
                    }
            } else if (4 * i < (4 * i < V / 2 ? t1 : t2)) {
                cv[i] = *(const f32x4*)(a.cos + at + (4 * i < V / 2 ? p1 : p2));
                sv[i] = *(const f32x4*)(a.sin + at + (4 * i < V / 2 ? p1 : p2));
            }
        }
        typedef typename Run<T, V>::Raw Raw;
        Raw x[kBatch][2], g[BWD ? kBatch : 1][2];
        const char* px = sd.x + b * sd.xb + n * sd.xt;
        const char* pg = BWD ? sd.g + b * sd.gb + n * sd.gt : nullptr;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int h = head0 + u * G;
            x[u][0] = x[u][1] = Raw{};
            if constexpr (BWD) g[u][0] = g[u][1] = Raw{};
            if (grp < G && h < sd.heads) {
                x[u][0] = *(const Raw*)(px + h * sd.xh + ES * oa);
                x[u][1] = *(const Raw*)(px + h * sd.xh + ES * ob);
                if constexpr (BWD) {
                    g[u][0] = *(const Raw*)(pg + h * sd.gh + ES * oa);
                    g[u][1] = *(const Raw*)(pg + h * sd.gh + ES * ob);
                }
            }
        }
        float c[V], s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = cv[i / 4][i % 4], s[i] = sv[i / 4][i % 4] * a.sgn;
        char* py = sd.y + b * sd.yb + n * sd.yt;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int h = head0 + u * G;
            const bool live = grp < G && h < sd.heads;
            if (head0 - grp + u * G >= sd.heads) break;  // no head of the wave is left
            float v[2 * V];
            unpack<T, V>(x[u][0], v);
            unpack<T, V>(x[u][1], v + V);
            if constexpr (NORM == 2) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) m += v[i];
                m = head_sum<L>(m, lane, p) * (1.f / D);
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) v[i] -= m;
            }
            if constexpr (NORM != 0) {
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) q = __builtin_fmaf(v[i], v[i], q);
                q = head_sum<L>(q, lane, p);
                // lanes without a head hold zeros: no quotient of theirs reaches a sum
                const float r = live ? rsqrtf(q * (1.f / D) + a.eps) : 0.f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) v[i] *= r;
                if constexpr (!BWD) {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) v[i] = __builtin_fmaf(v[i], w[i], bias[i]);
                } else {
                    float gv[2 * V];
                    unpack<T, V>(g[u][0], gv);
                    unpack<T, V>(g[u][1], gv + V);
                    rotate<V>(gv, c, s, t1, t2, HALF);
                    float m1 = 0.f, m2 = 0.f;
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        dw[i] = __builtin_fmaf(gv[i], v[i], dw[i]);
                        if constexpr (NORM == 2) db[i] += gv[i];
                        gv[i] *= w[i];
                        m1 = __builtin_fmaf(gv[i], v[i], m1);
                        if constexpr (NORM == 2) m2 += gv[i];
                    }
                    m1 = head_sum<L>(m1, lane, p) * (1.f / D);
                    if constexpr (NORM == 2) m2 = head_sum<L>(m2, lane, p) * (1.f / D);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) v[i] = r * (gv[i] - __builtin_fmaf(v[i], m1, m2));
                }
            }
            if constexpr (!BWD) rotate<V>(v, c, s, t1, t2, HALF);
            if (live) {
                store_run<T, V>(py + h * sd.yh + ES * oa, v);
                store_run<T, V>(py + h * sd.yh + ES * ob, v + V);
            }
        }
    }

    // the workgroup's sums of the weights' gradients, heads and waves in order
    if constexpr (BWD) {
        __shared__ float red[64 * kWaves * 2 * V];
        const int64_t slots = (int64_t)gridDim.x * (second ? gridDim.y - a.nb0 : a.nb0);
        const int64_t slot = (int64_t)(blockIdx.y - (second ? a.nb0 : 0)) * gridDim.x + blockIdx.x;
#pragma unroll
        for (int k = 0; k < (NORM == 2 ? 2 : 1); ++k) {
            if (!(sd.grads & (1 << k))) continue;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) red[threadIdx.x * 2 * V + i] = k == 0 ? dw[i] : db[i];
            __syncthreads();
            if (threadIdx.x < D) {
                const int tp = threadIdx.x / (2 * V), ti = threadIdx.x % (2 * V);
                float sum = 0.f;
                for (int j = 0; j < kWaves * G; ++j)
                    sum += red[((j / G) * 64 + (j % G) * L + tp) * 2 * V + ti];
                int e = SPLIT ? V * tp + ti + (ti < V ? 0 : D / 2 - V) : 2 * V * tp + ti;
                if (HALF) {
                    const int tc = V * tp;
                    if (tc < rp) e = (ti < V ? tc : rp + tc - V) + ti;
                    else e = a.rot + 2 * (tc - rp) + ti;
                }
                a.part[(second ? a.part1 : 0) + (k * slots + slot) * D + e] = sum;
            }
        }
    }
}

// Sums of the partials in a fixed order: a workgroup takes 16 columns, a thread
// four of them in every 64th partial, then lanes and waves are joined.
// blockIdx.y: weight and bias of side 0, then of side 1.
struct NrSumArgs {
    const float* part[4];
    float* out[4];
    int slots[4];
    int D;
};
constexpr int kSumCols = 16, kSumThreads = 256;

__global__ __launch_bounds__(kSumThreads) void norm_rope_sum_kernel(NrSumArgs a) {
    __shared__ f32x4 red[kSumThreads / 64][4];
    const int q = blockIdx.y;
    if (a.out[q] == nullptr) return;
    const int tx = threadIdx.x & 3, e = blockIdx.x * kSumCols + 4 * tx;
    f32x4 sum = {};
    if (e < a.D) {
        const float* p = a.part[q] + e;
#pragma unroll 4
        for (int j = threadIdx.x >> 2; j < a.slots[q]; j += kSumThreads / 4) sum += *(const f32x4*)(p + (int64_t)j * a.D);
    }
#pragma unroll
    for (int o = 4; o < 64; o *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], o);
    if ((threadIdx.x & 63) < 4) red[threadIdx.x >> 6][tx] = sum;
    __syncthreads();
    if (threadIdx.x < 4 && e < a.D) {
        for (int w = 1; w < kSumThreads / 64; ++w) sum += red[w][tx];
#pragma unroll
        for (int i = 0; i < 4; ++i) a.out[q][e + i] = sum[i];
    }
}

struct NrGrid {
    int nb0, nb1;
    unsigned gx;
};

// Workgroups along the tokens, a token per wave at a time: forward as many as
// there are (up to 2^31 threads: a launch holds fewer than 2^32); backward, where
// each sums its weights' gradients, at most 512 in all with as many tokens for
// each.  So many run at once where a run is 8 values (184 to 206 registers, two
// waves per SIMD); of the forms whose runs are 4 values (114 to 156) 768 or 1024
// would.  Measured, us, at 512 / 1024 / 2048 workgroups: gradients of 4224 tokens,
// 24 + 24 heads of 128 37.8 / 38.9 / 40.5, with 72 dims of the half layout rotated
// (runs of 4) 46.7 / 40.6 / 39.7; 2 x 4096, 16 + 16 of 72 30.7 / 28.5 / 30.4;
// 17550, 48 + 48 of 64, layer norm 128 / 129 / 136; float32: the first 70.2 / 69.4 /
// 68.4, the last 267 / 266 / 262.  At 1024 / 2048 / a workgroup per 4 tokens: norms
// of the first 22.8 / 24.5 / 22.9, of 2 x 4096 16.5 / 17.8 / 17.9, of 17550 89 / 87 /
// 78; rotation of 17550, 48 heads of 64 48 / 45 / 41.
NrGrid nr_grid(int64_t rows, int heads0, int heads1, int G, bool bwd) {
    NrGrid r;
    r.nb0 = (heads0 + kBatch * G - 1) / (kBatch * G);
    r.nb1 = (heads1 + kBatch * G - 1) / (kBatch * G);
    const int64_t need = (rows + kWaves - 1) / kWaves, nb = r.nb0 + r.nb1 > 0 ? r.nb0 + r.nb1 : 1;
    const int64_t all = bwd ? 512 : 1 << 23, most = all / nb > 1 ? all / nb : 1;
    const int64_t each = (need + most - 1) / most;
    r.gx = (unsigned)(each > 0 ? (need + each - 1) / each : 0);
    return r;
}

// values of a run: 16 bytes where a head's lanes divide it so, 4 values otherwise
int run_of(int D, bool bf16, int rot, int half) {
    return bf16 && D % 16 == 0 && (!half || rot % 16 == 0) ? 8 : 4;
}

template <typename T, int D, int V>
hipError_t launch_form(const NrArgs& a, dim3 grid, int norm, int half, bool bwd, hipStream_t s) {
    const dim3 block(64 * kWaves);
#define XDIT_NR(N, W, F) hipLaunchKernelGGL((norm_rope_kernel<T, D, V, N, W, F>), grid, block, 0, s, a)
    if (bwd) {
        if (norm == 1) {
            if (half) XDIT_NR(1, true, true);
            else XDIT_NR(1, true, false);
        } else {
            if (half) XDIT_NR(2, true, true);
            else XDIT_NR(2, true, false);
        }
    } else if (norm == 0) {
        if (half) XDIT_NR(0, false, true);
        else XDIT_NR(0, false, false);
    } else if (norm == 1) {
        if (half) XDIT_NR(1, false, true);
        else XDIT_NR(1, false, false);
    } else {
        if (half) XDIT_NR(2, false, true);
        else XDIT_NR(2, false, false);
    }
#undef XDIT_NR
    return hipGetLastError();
}

hipError_t launch_any(const NormRopeParams& p, bool bwd, hipStream_t s) {
    const int V = run_of(p.D, p.bf16, p.rot, p.half);
    const int64_t es = p.bf16 ? 2 : 4;
    const int64_t rows = (int64_t)p.B * p.N;
    const NrGrid g = nr_grid(rows, p.side[0].heads, p.side[1].heads, 64 / (p.D / (2 * V)), bwd);
    const dim3 grid(g.gx, (unsigned)(g.nb0 + g.nb1));
    NrArgs a{};
    for (int i = 0; i < 2; ++i) {
        const NormRopeSide& f = p.side[i];
        NrSide& t = a.side[i];
        t.x = (const char*)f.x.p, t.xb = es * f.x.sb, t.xt = es * f.x.st, t.xh = es * f.x.sh;
        t.g = (const char*)f.g.p, t.gb = es * f.g.sb, t.gt = es * f.g.st, t.gh = es * f.g.sh;
        t.y = (char*)f.y.p, t.yb = es * f.y.sb, t.yt = es * f.y.st, t.yh = es * f.y.sh;
        t.w = f.w, t.b = f.b, t.heads = f.heads;
        t.grads = (f.dw ? 1 : 0) | (f.db ? 2 : 0);
    }
    a.nb0 = g.nb0;
    a.cos = p.cos, a.sin = p.sin, a.table_batch = p.table_batch;
    a.rows = (uint32_t)rows, a.N = (uint32_t)(p.N > 0 ? p.N : 1);
    a.rot = p.cos ? p.rot : 0, a.half = p.half, a.weight_bf16 = p.weight_bf16;
    a.sgn = bwd || p.transpose ? -1.f : 1.f;
    a.eps = p.eps;
    a.part = p.part;
    a.part1 = (int64_t)2 * g.nb0 * g.gx * p.D;
    const int half = p.half && a.rot > 0;
    if (grid.x > 0 && grid.y > 0) {
        hipError_t e = hipErrorInvalidValue;
        if (p.bf16) {
            if (p.D == 64) e = V == 8 ? launch_form<uint16_t, 64, 8>(a, grid, p.norm, half, bwd, s)
                                      : launch_form<uint16_t, 64, 4>(a, grid, p.norm, half, bwd, s);
            else if (p.D == 72) e = launch_form<uint16_t, 72, 4>(a, grid, p.norm, half, bwd, s);
            else if (p.D == 128) e = V == 8 ? launch_form<uint16_t, 128, 8>(a, grid, p.norm, half, bwd, s)
                                            : launch_form<uint16_t, 128, 4>(a, grid, p.norm, half, bwd, s);
        } else {
            if (p.D == 64) e = launch_form<float, 64, 4>(a, grid, p.norm, half, bwd, s);
            else if (p.D == 72) e = launch_form<float, 72, 4>(a, grid, p.norm, half, bwd, s);
            else if (p.D == 128) e = launch_form<float, 128, 4>(a, grid, p.norm, half, bwd, s);
        }
        if (e != hipSuccess) return e;
    }
    if (!bwd) return hipSuccess;
    NrSumArgs r{};
    r.D = p.D;
    bool any = false;
    for (int i = 0; i < 2; ++i) {
        const int nb = i == 0 ? g.nb0 : g.nb1;
        float* out[2] = {p.side[i].dw, p.side[i].db};
        for (int k = 0; k < 2; ++k) {
            r.out[2 * i + k] = out[k];
            r.slots[2 * i + k] = (int)(nb * g.gx);
            r.part[2 * i + k] = a.part + (i ? a.part1 : 0) + (int64_t)k * nb * g.gx * p.D;
            any = any || out[k] != nullptr;
        }
    }
    if (!any) return hipSuccess;
    hipLaunchKernelGGL(norm_rope_sum_kernel, dim3((p.D + kSumCols - 1) / kSumCols, 4), dim3(kSumThreads), 0, s, r);
    return hipGetLastError();
}

// cos and sin of a quarter turn times f, |f| <= 1/2, by their Taylor series at
// x = f pi/2 (|x| <= pi/4: the first terms left out are 2e-14 and 4e-13; the
// table is float32), then the quarter turns before it.
__device__ __forceinline__ void quarter_sincos(double f, int quarters, double* sn, double* cs) {
    const double x = f * 1.5707963267948966, z = x * x;
    double s = 1. / 6227020800.;
    s = fma(s, z, -1. / 39916800.);
    s = fma(s, z, 1. / 362880.);
    s = fma(s, z, -1. / 5040.);
    s = fma(s, z, 1. / 120.);
    s = fma(s, z, -1. / 6.);
    s = fma(s * z, x, x);
    double c = 1. / 479001600.;
    c = fma(c, z, -1. / 3628800.);
    c = fma(c, z, 1. / 40320.);
    c = fma(c, z, -1. / 720.);
    c = fma(c, z, 1. / 24.);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.);
    const double a = quarters & 1 ? c : s, b = quarters & 1 ? s : c;
    *sn = quarters & 2 ? -a : a;
    *cs = (quarters + 1) & 2 ? -b : b;
}

// A thread's columns are fixed: their frequencies once, a column per thread of
// the workgroup, in quarter turns and 64 bits (an angle of 10^6 in float32 is off
// by 0.06), then per row the products with the position, their whole quarter turns
// taken off exactly.  Bound by stores and 64-bit arithmetic, 25 operations an
// angle, and by the start of one round of workgroups: 131072 x 64 angles take 18 to
// 20 us (68 MB at 3.4 to 3.7 TB/s; one column a thread 26; the library's sincospi
// took 27), 2^20 x 64 124 us (4.4 TB/s; 191), 32768 x 64 8.2 (9.8).  The highest term
// of each series, and the product with a magnitude of 1, are more than a float32
// table needs.
//
// Frequencies are 2^(i rate): the rounding of an exponent of size e would be
// one of e ln 2 / 2 steps in the frequency (up to 7 measured at dims of 72, theta
// 10^4), so the rate comes in two parts, and what the product of its first part
// and i rounds away goes into the result to first order.
struct TableAxes {
    double rate[4], rest[4];  // of each axis: log2 of a pair's frequency over that of the pair before, scaling included
};

template <int V, int R>  // V columns of a thread, R rows whose positions load together
__global__ __launch_bounds__(256) void rope_table_kernel(RopeTableParams a, TableAxes ax, int cols, int rows_per_block) {
    typedef float out_t __attribute__((ext_vector_type(V)));
    __shared__ double freq[128];
    const int col = threadIdx.x % (cols / V) * V, sub = threadIdx.x / (cols / V);
    int axis[V];
#pragma unroll
    for (int v = 0, k = 0, end = a.dims[0] / 2; v < V; ++v) {
        while (k + 1 < a.axes && col + v >= end) end += a.dims[++k] / 2;
        axis[v] = k;
    }
    const int64_t step = (int64_t)gridDim.x * rows_per_block;
    int64_t n0 = (int64_t)blockIdx.x * rows_per_block + sub;
    double pos[R][V];
    auto load = [&] {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t n = n0 + r * step < a.n ? n0 + r * step : 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t at = n * a.axes + axis[v];
                if (v > 0 && axis[v] == axis[v - 1]) pos[r][v] = pos[r][v - 1];
                else pos[r][v] = a.pos_i64 ? (double)((const int64_t*)a.pos)[at] : (double)((const float*)a.pos)[at];
            }
        }
    };
    load();
    if ((int)threadIdx.x < cols) {
        int i = threadIdx.x, k = 0;
        while (k + 1 < a.axes && i >= a.dims[k] / 2) i -= a.dims[k++] / 2;
        const double e = i * ax.rate[k];
        double w = exp2(e);
        w = fma(w, 0.6931471805599453 * fma((double)i, ax.rest[k], fma((double)i, ax.rate[k], -e)), w);
        if (a.scaling == 1) w /= a.factor;
        if (a.scaling == 3) {
            const double turns = a.orig_len * w * 0.15915494309189535;  // 1 / (2 pi)
            const double share = fmin(1.0, fmax(0.0, (turns - a.slow) / (a.fast - a.slow)));
            w = w * (share + (1.0 - share) / a.factor);
        }
        freq[threadIdx.x] = w * 0.6366197723675814;  // 2 / pi
    }
    __syncthreads();
    if (sub >= rows_per_block || n0 >= a.n) return;
    double w[V];
#pragma unroll
    for (int v = 0; v < V; ++v) w[v] = freq[col + v];
    float *pc = a.cos + n0 * cols + col, *ps = a.sin + n0 * cols + col;
    for (;;) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (n0 + r * step >= a.n) break;
            out_t c, s;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                double t = pos[r][v] * w[v];
                if (fabs(t) >= 0x1p50) t = fma(-4.0, rint(0.25 * t), t);  // whole turns off, so that the sum below is exact
                const double m = t + 0x1.8p52;  // the whole quarter turns, in the sum's low bits
                double sn, cs;
                quarter_sincos(t - (m - 0x1.8p52), (int)__builtin_bit_cast(uint64_t, m), &sn, &cs);
                c[v] = (float)(cs * a.magnitude);
                s[v] = (float)(sn * a.magnitude);
            }
            *(out_t*)pc = c;
            *(out_t*)ps = s;
            pc += step * cols;
            ps += step * cols;
        }
        n0 += R * step;
        if (n0 >= a.n) break;
        load();
    }
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeParams& p, hipStream_t s) { return launch_any(p, false, s); }
hipError_t launch_norm_rope_bwd(const NormRopeParams& p, hipStream_t s) { return launch_any(p, true, s); }

int64_t norm_rope_bwd_partials(int64_t rows, int heads0, int heads1, int D, bool bf16) {
    // either width of a run may be the one that the call's rotation needs
    int64_t most = 0;
    for (int V : {4, 8}) {
        if (V == 8 && run_of(D, bf16, 0, 0) != 8) continue;
        const NrGrid g = nr_grid(rows, heads0, heads1, 64 / (D / (2 * V)), true);
        const int64_t n = (int64_t)2 * (g.nb0 + g.nb1) * g.gx * D;
        if (n > most) most = n;
    }
    return most;
}

hipError_t launch_rope_table(const RopeTableParams& p, hipStream_t s) {
    int cols = 0;
    for (int i = 0; i < p.axes; ++i) cols += p.dims[i] / 2;
    if (p.n == 0) return hipSuccess;
    TableAxes ax{};
    for (int i = 0; i < p.axes; ++i) {
        const long double dim = p.dims[i];
        const long double rate = -2 * (log2l(p.theta) + (p.scaling == 2 ? dim / (dim - 2) * log2l(p.factor) : 0)) / dim;
        ax.rate[i] = (double)rate;
        ax.rest[i] = (double)(rate - ax.rate[i]);
    }
    const bool wide = cols % 4 == 0;  // stores of 16 bytes
    const int rpb = 256 / (wide ? cols / 4 : cols), rows = rpb * (wide ? 1 : 4);
    const int64_t need = (p.n + rows - 1) / rows;
    const dim3 grid((unsigned)(need < 2048 ? need : 2048));
    hipLaunchKernelGGL((wide ? rope_table_kernel<4, 1> : rope_table_kernel<1, 4>), grid, dim3(256), 0, s, p, ax, cols, rpb);
    return hipGetLastError();
}

}  // namespace xdit
