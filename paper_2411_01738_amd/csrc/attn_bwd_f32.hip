// Gradients of float32 attention: the formulas and sweeps of attn_bwd.hip with
// float32 products throughout, on v_mfma_f32_16x16x4_f32.
//
// What bounds it: the float32 matrix rate.  2 x 16 heads of 72, 1024 x 1024: 293
// us, 115 TFLOP/s over its seven products (128 with the padding of 72 to 80)
// where a large product reaches 150.
//
// One workgroup = 64 resident rows, 4 waves of 16; tiles of 32 streamed rows
// come straight into LDS, two stages.  X = T1 R1^T and Y = T2 R2^T take dims
// 16-byte chunk by chunk, lane group g chunk 4j + g, so one read feeds four
// products; in A^T += T^T W the accumulator registers of P and dS are the
// operand as they stand (register i: rows 4g + i), and T is read by columns, 4
// bytes a lane.  d = 72: the fifth 16-byte step and the fifth block of 16 dims
// are half padding.  Blocks of 32 resident rows (v_mfma_f32_32x32x2_f32) held
// d = 128's operands and sums in 290 registers, half of which moved between the
// two register files in every tile.
#include "kernels.h"

#include <math.h>

#include <type_traits>

namespace xdit {
namespace {

#include "attn_common.h"

struct BwdF32Args {
    const float* r1;
    const float* r2;
    const float* t1;
    const float* t2;
    const float* rows;  // per (batch, head): [2][Nq] -l sqrt(d), -D
    float* o1;
    float* o2;
    float* part;
    int64_t part_elems;
    int B, H, Nr, Nt, r_tiles, splits;
    int accum;
    float c2, scale;
};

constexpr int kRows = 64, kTile = 32;

// LDS: two stages of both tiles, then of the rows' scalars
template <int D>
constexpr int lds_bytes() {
    return 4 * kTile * 4 * D + 2 * 8 * kTile;
}

template <int D, bool KV>
__device__ __forceinline__ void sweep(const BwdF32Args& a, unsigned char* lds, int logical) {
    constexpr int CH = D / 4, ROWB = 4 * D, STAGE = kTile * ROWB, DBLK = (D + 15) / 16, KQ = (CH + 3) / 4;
    constexpr int DMA = STAGE / 1024, DMA_PER_WAVE = (DMA + 3) / 4;
    constexpr int ROWBASE = 4 * STAGE;
    static_assert(STAGE % 1024 == 0, "tiles are whole 64-lane loads");
    // 16-byte chunk c of row r sits in slot c ^ swz(r): sixteen rows' equal
    // chunks, and four rows' 64 bytes, lie in distinct banks
    auto swz = [](int r) { return D == 72 ? (r >> 3) & 1 : r & 15; };

    const int tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int sp = logical % a.splits, pair = logical / a.splits;
    const int rt = pair % a.r_tiles, bh = pair / a.r_tiles;
    const int hh = bh % a.H, b = bh / a.H;
    const uint32_t rowb = (uint32_t)a.H * D * 4, headb = (uint32_t)hh * D * 4;
    const int64_t rs = (int64_t)a.H * D, headoff = (int64_t)hh * D;
    const int all_tiles = (a.Nt + kTile - 1) / kTile;
    const int tb = (int)((int64_t)all_tiles * sp / a.splits);
    const int ntiles = (int)((int64_t)all_tiles * (sp + 1) / a.splits) - tb;
    auto rows_rsrc = [&](const float* base, int64_t n, int row0) -> Rsrc {
        return rsrc(base + ((int64_t)b * n + row0) * rs + headoff, n > row0 ? (uint32_t)(n - row0) * rowb - headb : 0u);
    };

    // resident operands: chunk 4j + g of row c (zeros past d and past the end)
    const int row = rt * kRows + wave * 16 + c;
    f32x4 r1[KQ], r2[KQ];
    {
        const Rsrc q1 = rows_rsrc(a.r1, a.Nr, rt * kRows), q2 = rows_rsrc(a.r2, a.Nr, rt * kRows);
#pragma unroll
        for (int j = 0; j < KQ; ++j) {
            const uint32_t off = 4 * j + g < CH ? (uint32_t)(wave * 16 + c) * rowb + 16 * (4 * j + g) : kOOB;
            r1[j] = __builtin_bit_cast(f32x4, bload(q1, off));
            r2[j] = __builtin_bit_cast(f32x4, bload(q2, off));
        }
    }
    float nl = 0.f, nd = 0.f;
    if constexpr (!KV) {
        const float* rows = a.rows + (int64_t)bh * 2 * a.Nr;
        if (row < a.Nr) {
            nl = rows[row];
            nd = rows[a.Nr + row];
        }
    }
    uint32_t dma_off[DMA_PER_WAVE];
#pragma unroll
    for (int n = 0; n < DMA_PER_WAVE; ++n) {
        const int p = 64 * (wave + 4 * n) + lane, r = p / CH;
        dma_off[n] = (uint32_t)r * rowb + 16 * ((p % CH) ^ swz(r));
    }
    auto load_tile = [&](int t, int s) {
        const int lo = (tb + t) * kTile;
        const Rsrc q1 = rows_rsrc(a.t1, a.Nt, lo), q2 = rows_rsrc(a.t2, a.Nt, lo);
#pragma unroll
        for (int n = 0; n < DMA_PER_WAVE; ++n) {
            const int ins = wave + 4 * n;
            if (DMA % 4 == 0 || ins < DMA) {
                dma16(q1, lds + 2 * s * STAGE + 1024 * ins, dma_off[n]);
                dma16(q2, lds + (2 * s + 1) * STAGE + 1024 * ins, dma_off[n]);
            }
        }
        if constexpr (KV) {
            if (wave == 3) {  // 32 values of -l sqrt(d), then 32 of -D
                const Rsrc qr = rsrc(a.rows + (int64_t)bh * 2 * a.Nt, (uint32_t)a.Nt * 8);
                const int j = lo + (lane & 31);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(qr, (lds_void*)(lds + ROWBASE + 8 * kTile * s), 4,
                                                         j < a.Nt ? 4u * (uint32_t)(j + (lane < 32 ? 0 : a.Nt)) : kOOB, 0, 0, 0);
            }
        }
    };

    f32x4 acc1[KV ? DBLK : 1], acc2[DBLK];
#pragma unroll
    for (int db = 0; db < DBLK; ++db) {
        if constexpr (KV) acc1[db] = f32x4{};
        acc2[db] = f32x4{};
    }
    // LDS addresses in stage 0 (T1's tile; T2's follows it).  Operand chunk 4j + g
    // of row c: swizzled rows start at multiples of 256 bytes, so chunks 4j and
    // dims 16db away have 64j (64db) exclusive-ored in; those of d = 72 add it.
    const uint32_t lds_u32 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    constexpr bool XOR = D != 72;
    uint32_t op0 = lds_u32 + c * ROWB + 16 * (g ^ swz(c));
    // (d = 72: past d, a chunk that is not there meets zeros of the resident
    // operand: any finite values do)
    const uint32_t pad = CH % 4 != 0 && 4 * (KQ - 1) + g >= CH ? 64 * (KQ - 1) : 0;
    uint32_t col0[4];  // columns c of rows 4g + i
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * g + i;
        col0[i] = lds_u32 + r * ROWB + 16 * ((c >> 2) ^ swz(r)) + 4 * (c & 3);
    }
    // A^T += T^T W: lane c is dim 16db + c of rows 4g + i of the block at off (a
    // lane past d reads on into the next row; its result is not stored)
    auto gather = [&](auto off_c, const uint32_t (&col)[4], const float (&w)[4], f32x4* acc) {
        constexpr int OFF = decltype(off_c)::value;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            static_for<0, DBLK>([&](auto db_c) {
                constexpr int db = decltype(db_c)::value;
                const float x = lds_ld<float>(XOR ? (col[i] ^ (64 * db)) + OFF : col[i] + (OFF + 64 * db));
                acc[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, w[i], acc[db], 0, 0, 0);
            });
    };

    const bool idle = rt * kRows + wave * 16 >= a.Nr;  // all of the wave's rows lie past the end
    if (ntiles > 0) load_tile(0, 0);
    for (int t = 0; t < ntiles; ++t) {
        const int s = t & 1;
        // tile t has landed in every wave, and every wave is done with tile t - 1
        wait_vmem<0>();
        __syncthreads();
        if (t + 1 < ntiles) load_tile(t + 1, s ^ 1);
        if (idle) continue;
        uint32_t op = op0 + 2 * s * STAGE, col[4];
        asm volatile("" : "+v"(op));  // opaque: what derives from it is not kept in registers
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            col[i] = col0[i] + 2 * s * STAGE;
            asm volatile("" : "+v"(col[i]));
        }
        f32x4 x[2] = {}, y[2] = {};
        static_for<0, KQ>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value;
            const uint32_t at = XOR ? op ^ (64 * j) : j == KQ - 1 ? op + 64 * j - pad : op + 64 * j;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 u1 = lds_ld<f32x4>(at + 16 * k * ROWB), u2 = lds_ld<f32x4>(at + 16 * k * ROWB + STAGE);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(u1[e], r1[j][e], x[k], 0, 0, 0);
                    y[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(u2[e], r2[j][e], y[k], 0, 0, 0);
                }
            }
        });
        static_for<0, 2>([&](auto k_c) {
            constexpr int k = decltype(k_c)::value;
            f32x4 l = {nl, nl, nl, nl}, dd = {nd, nd, nd, nd};
            if constexpr (KV) {
                const f32x4* q = (const f32x4*)(lds + ROWBASE + 8 * kTile * s + 64 * k + 16 * g);
                l = q[0];
                dd = q[8];
            }
            float p[4], z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[k][i], a.c2, l[i] * a.c2));
                // streamed keys past the end have no probability
                if (!KV && (tb + t) * kTile + 16 * k + 4 * g + i >= a.Nt) p[i] = 0.f;
                z[i] = p[i] * (y[k][i] + dd[i]);
            }
            if constexpr (KV) gather(std::integral_constant<int, STAGE + 16 * k * ROWB>{}, col, p, acc1);
            gather(std::integral_constant<int, 16 * k * ROWB>{}, col, z, acc2);
        });
    }

    if (row >= a.Nr) return;
    const int64_t at0 = ((int64_t)b * a.Nr + row) * rs + headoff;
    auto result = [&](float* dst, int64_t part0, const f32x4* acc, float f) {
#pragma unroll
        for (int db = 0; db < DBLK; ++db) {
            const int dim = 16 * db + 4 * g;
            if (D % 16 != 0 && dim >= D) continue;
            const f32x4 v = acc[db] * f;
            if (a.splits > 1) {
                *(f32x4*)(a.part + part0 + (int64_t)sp * a.part_elems + at0 + dim) = v;
            } else {
                f32x4* o = (f32x4*)(dst + at0 + dim);
                *o = a.accum ? *o + v : v;
            }
        }
    };
    result(a.o2, 0, acc2, a.scale);
    if constexpr (KV) result(a.o1, a.splits * a.part_elems, acc1, 1.f);
}

// Both sweeps in one launch, the longer workgroups first, as in attn_bwd.hip.
template <int D>
__global__ __launch_bounds__(256, 2) void attn_bwd_f32_kernel(BwdF32Args kv, BwdF32Args q, int n_first, int kv_first) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[lds_bytes<D>()];
    const int first = (int)blockIdx.x < n_first;
    const int id = first ? blockIdx.x : blockIdx.x - n_first, n = first ? n_first : gridDim.x - n_first;
    if (first == kv_first) sweep<D, true>(kv, lds, xcd_remap(id, n));
    else sweep<D, false>(q, lds, xcd_remap(id, n));
}

BwdF32Args sweep_args(const AttnBwdParams& p, bool kv) {
    BwdF32Args a{};
    a.r1 = (const float*)(kv ? p.k : p.q);
    a.r2 = (const float*)(kv ? p.v : p.dout);
    a.t1 = (const float*)(kv ? p.q : p.k);
    a.t2 = (const float*)(kv ? p.dout : p.v);
    a.rows = p.rows;
    a.o1 = (float*)p.dv;
    a.o2 = (float*)(kv ? p.dk : p.dq);
    a.B = p.B, a.H = p.H;
    a.Nr = kv ? p.Nk : p.Nq, a.Nt = kv ? p.Nq : p.Nk;
    a.r_tiles = (a.Nr + kRows - 1) / kRows;
    a.splits = kv ? p.kv_splits : p.q_splits;
    a.accum = kv ? p.accum_kv : p.accum_q;
    a.part = kv ? p.kv_part : p.q_part;
    a.part_elems = (int64_t)p.B * a.Nr * p.H * p.D;
    a.scale = 1.f / sqrtf((float)p.D);
    a.c2 = a.scale * 1.4426950408889634f;
    return a;
}

template <int D>
hipError_t launch_sweeps(const BwdF32Args& kv, const BwdF32Args& q, hipStream_t s) {
    const int64_t n_kv = (int64_t)kv.B * kv.H * kv.r_tiles * kv.splits;
    const int64_t n_q = (int64_t)q.B * q.H * q.r_tiles * q.splits;
    if (n_kv + n_q == 0) return hipSuccess;
    const int kv_first = 4 * (int64_t)kv.Nt * q.splits >= 3 * (int64_t)q.Nt * kv.splits;
    hipLaunchKernelGGL(attn_bwd_f32_kernel<D>, dim3((unsigned)(n_kv + n_q)), dim3(256), 0, s, kv, q,
                       (int)(kv_first ? n_kv : n_q), kv_first);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_bwd_f32(const AttnBwdParams& p, hipStream_t s) {
    const BwdF32Args kv = sweep_args(p, true), q = sweep_args(p, false);
    if (p.D == 64) return launch_sweeps<64>(kv, q, s);
    if (p.D == 72) return launch_sweeps<72>(kv, q, s);
    return launch_sweeps<128>(kv, q, s);
}

}  // namespace xdit
