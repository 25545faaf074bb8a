// Gradients of bf16 attention (chunk attention with O and LSE, possibly merged
// with other chunks) on the gfx950 matrix cores.
//
// Per (batch, head), with s_ij = (q_i . k_j) / sqrt(d), the LSE l_i and output
// o_i of the row (over all chunks), and the gradients g_i of o_i, e_i of l_i:
//   P_ij  = exp(s_ij - l_i)
//   D_i   = g_i . o_i - e_i
//   dS_ij = P_ij (g_i . v_j - D_i)
//   dV_j  = sum_i P_ij g_i
//   dK_j  = sum_i dS_ij q_i / sqrt(d),  dQ_i = sum_j dS_ij k_j / sqrt(d)
// The probabilities are computed again from the scores; nothing of size
// queries x keys is stored.  P and dS are rounded to bf16 because they are
// operands of bf16 products (half a step, 2^-8 relative, each; the sums are
// float32).  The roundings of a sum's terms are independent: the root mean square
// error of a result is 0.0024 relative where its own rounding gives 0.0017
// (measured).  float32 products, which would keep them, run at a ninth of the rate.
//
// What bounds it: the matrix cores (24 heads of 128, 4224 x 4224: 683 us, 1120
// TFLOP/s over the seven products, where a large product of random values
// reaches 1372).  One sweep gives dK and dV (four products
// of queries x keys x d), another dQ (three), seven in place of the five that
// are needed: a single sweep would have to add its part of the other side's
// gradient to memory for every tile, by atomics whose order changes the result
// or through partials larger than the inputs.
//
// Work decomposition: one workgroup = kRows resident rows (keys of dK/dV,
// queries of dQ) of one (batch, head), 4 waves of 32 rows each, whose two
// operands stay in registers; the other side's two tensors stream through LDS
// in tiles (memory straight into LDS, four stages, one barrier per tile):
//   resident x streamed:  dK/dV: K, V x Q, G     dQ: Q, G x K, V
//   X = T1 R1^T (scores), Y = T2 R2^T (g . v): a lane holds 16 streamed rows
//   of one resident row;
//   P and dS in these registers are at once the operands of the products that
//   sum over streamed rows, A1^T += T2^T P and A2^T += T1^T dS, whose other
//   operand is read from the same tiles by the transposing LDS read.
// Layout of a tile in LDS, order of rows in a block (krow) and the padding of
// d = 72 are those of attn_bf16.hip.  For dK/dV the rows' -l_i sqrt(d) and
// -D_i come along with the tiles and are what X and Y start from; for dQ they
// belong to the lane.
#include "kernels.h"

#include <math.h>

#include <type_traits>

namespace xdit {
namespace {

#include "attn_common.h"

struct BwdArgs {
    const uint16_t* r1;   // resident operands, [B, Nr, H, D]
    const uint16_t* r2;
    const uint16_t* t1;   // streamed ones, [B, Nt, H, D]
    const uint16_t* t2;
    const float* rows;    // per (batch, head): [2][Nq] -l sqrt(d), -D
    void* o1;             // dV (KV only)
    void* o2;             // dK or dQ
    float* part;          // splits > 1: float32 partials [splits][B, Nr, H, D] of o2, then of o1
    int64_t part_elems;   // B * Nr * H * D
    int B, H, Nr, Nt, r_tiles, splits;
    int accum;            // o1, o2 are float32 sums to add to
    float c2, scale;      // softmax scale * log2(e), softmax scale
};

constexpr int kRows = 128;

template <int D, bool KV>
struct BCfg {
    static constexpr int NW = 4, THREADS = 64 * NW;
    static constexpr int NB = D > 96 ? 1 : 2;           // 32-row blocks of a tile
    static constexpr int BN = 32 * NB;                  // streamed rows per tile
    static constexpr int CH = D / 8, ROWB = 16 * CH;    // 16-byte chunks and bytes of a row
    static constexpr int KSTEPS = (D + 15) / 16;
    static constexpr int DBLK = D / 32;
    static constexpr bool TAIL = D % 32 != 0;           // d = 72: dims 64..71 on the 16x16x32 instruction
    static constexpr bool PERM = CH != 8;
    static constexpr int E_ROWS = PERM ? 2 : 8;         // rows between the two half k-steps of a transposing read
    __device__ static constexpr int swz(int r) {
        if constexpr (CH == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        else if constexpr (CH == 16) return r & 15;
        else return 0;
    }
    static constexpr bool SWIZZLED = CH == 8 || CH == 16;
    static constexpr int REGION = BN * ROWB;            // one tile of one tensor
    static constexpr int NST = 4;
    static constexpr int T2BASE = NST * REGION;         // T1's regions, then T2's
    static constexpr int ROWBASE = 2 * NST * REGION;    // then the rows' scalars (KV)
    static constexpr int ROWREGION = KV ? 8 * BN : 0;
    static constexpr int LDS_BYTES = ROWBASE + NST * ROWREGION;
    static constexpr int DMA_PER_TILE = REGION / 1024;
    static constexpr int DMA_PER_WAVE = (DMA_PER_TILE + NW - 1) / NW;
    static_assert(REGION % 1024 == 0 && LDS_BYTES <= kLdsBytes / 2, "two workgroups per CU");
};

// Workgroup `logical` of the dK/dV sweep (KV) or the dQ sweep.
template <int D, bool KV>
__device__ __forceinline__ void sweep(const BwdArgs& a, unsigned char* lds, int logical) {
    using C = BCfg<D, KV>;
    constexpr int NST = C::NST, NB = C::NB, BN = C::BN, KSTEPS = C::KSTEPS, DBLK = C::DBLK, NW = C::NW;

    const int tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, hf = lane >> 5;
    const int sp = logical % a.splits, pair = logical / a.splits;
    const int rt = pair % a.r_tiles, bh = pair / a.r_tiles;
    const int hh = bh % a.H, b = bh / a.H;
    const uint32_t rowb = (uint32_t)a.H * D * 2, headb = (uint32_t)hh * D * 2;
    const int64_t rs = (int64_t)a.H * D, headoff = (int64_t)hh * D;
    const uint32_t lds_u32 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;

    // this workgroup's tiles of the sweep
    const int all_tiles = (a.Nt + BN - 1) / BN;
    const int tb = (int)((int64_t)all_tiles * sp / a.splits);
    const int ntiles = (int)((int64_t)all_tiles * (sp + 1) / a.splits) - tb;

    auto rows_rsrc = [&](const uint16_t* base, int64_t n, int row0) -> Rsrc {
        return rsrc(base + ((int64_t)b * n + row0) * rs + headoff, n > row0 ? (uint32_t)(n - row0) * rowb - headb : 0u);
    };

    // resident operands: row `row` of this wave, chunk 2kk + hf; chunks past d
    // and rows past the end read as zero
    const int row = rt * kRows + wave * 32 + c;
    bf16x8 r1[KSTEPS], r2[KSTEPS];
    {
        const Rsrc q1 = rows_rsrc(a.r1, a.Nr, rt * kRows), q2 = rows_rsrc(a.r2, a.Nr, rt * kRows);
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) {
            const uint32_t off = 2 * kk + hf < C::CH ? (uint32_t)(wave * 32 + c) * rowb + 32 * kk + 16 * hf : kOOB;
            r1[kk] = __builtin_bit_cast(bf16x8, bload(q1, off));
            r2[kk] = __builtin_bit_cast(bf16x8, bload(q2, off));
        }
    }
    // the resident row's own -l log2(e) and -D (dQ)
    float nl = 0.f, nd = 0.f;
    if constexpr (!KV) {
        const float* rows = a.rows + (int64_t)bh * 2 * a.Nr;
        if (row < a.Nr) {
            nl = rows[row] * a.c2;
            nd = rows[a.Nr + row];
        }
    }

    // tile loads: piece n of this wave fills chunks 64 ins .. of a tile; chunk
    // p is row p / CH, logical chunk (p % CH) ^ swz(row)
    uint32_t dma_off[C::DMA_PER_WAVE];
#pragma unroll
    for (int n = 0; n < C::DMA_PER_WAVE; ++n) {
        const int p = 64 * (wave + n * NW) + lane;
        const int r = p / C::CH;
        dma_off[n] = (uint32_t)r * rowb + 16 * ((p % C::CH) ^ C::swz(r));
    }
    auto load_tile = [&](int t, int s) {
        const int lo = (tb + t) * BN;
        const Rsrc q1 = rows_rsrc(a.t1, a.Nt, lo), q2 = rows_rsrc(a.t2, a.Nt, lo);
#pragma unroll
        for (int n = 0; n < C::DMA_PER_WAVE; ++n) {
            const int ins = wave + n * NW;
            if (C::DMA_PER_TILE % NW == 0 || ins < C::DMA_PER_TILE) {
                dma16(q1, lds + s * C::REGION + 1024 * ins, dma_off[n]);
                dma16(q2, lds + C::T2BASE + s * C::REGION + 1024 * ins, dma_off[n]);
            }
        }
        if constexpr (KV) {
            // slot x of a block holds the row that accumulator row x is: 32
            // values of -l sqrt(d), then 32 of -D, per block; the last wave's work
            if (wave == NW - 1) {
                const Rsrc qr = rsrc(a.rows + (int64_t)bh * 2 * a.Nt, (uint32_t)a.Nt * 8);
#pragma unroll
                for (int kb = 0; kb < NB; ++kb) {
                    const int j = lo + 32 * kb + krow<C::PERM>(c);
                    const uint32_t off = j < a.Nt ? 4u * (uint32_t)(j + (hf ? a.Nt : 0)) : kOOB;
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(qr, (lds_void*)(lds + C::ROWBASE + s * C::ROWREGION + 256 * kb), 4,
                                                             off, 0, 0, 0);
                }
            }
        }
    };
    // at most the loads of the N youngest tiles are in flight
    constexpr int LOADS = 2 * (C::DMA_PER_TILE / NW);                       // of a wave without extras
    constexpr int FIRST = LOADS + (C::DMA_PER_TILE % NW ? 2 : 0);           // waves that take a left-over piece
    constexpr int LAST = LOADS + (KV ? NB : 0);
    static_assert(C::DMA_PER_TILE % NW <= 1, "one wave takes a left-over piece");
    auto wait_tiles = [&](auto n_c) {
        constexpr int N = decltype(n_c)::value;
        if (FIRST != LOADS && wave == 0) wait_vmem<N * FIRST>();
        else if (LAST != LOADS && wave == NW - 1) wait_vmem<N * LAST>();
        else wait_vmem<N * LOADS>();
    };

    // LDS addresses of this lane's operand reads in stage 0.  Swizzled rows
    // start at multiples of their own size, so chunks 2kk away are the first
    // one's address with 32kk exclusive-ored in (dims 32db away: 64db); rows
    // of d = 72 take them as offsets.
    const int gi = lane & 15, grp = lane >> 4;
    uint32_t k0, kpad = 0, v0[2], taddr = 0;
    {
        const int r = krow<C::PERM>(c);
        k0 = lds_u32 + r * C::ROWB + 16 * (hf ^ C::swz(r));
        // the chunk past d of the last k-step meets zeros of the resident
        // operand: any finite values do (the last chunk's)
        if constexpr (C::CH % 2 != 0) kpad = lds_u32 + r * C::ROWB + 16 * (C::CH - 1);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int dim = 16 * (grp & 1) + 4 * (gi & 3);
        const int r = krow<C::PERM>(4 * hf + (gi >> 2)) + C::E_ROWS * e;
        v0[e] = lds_u32 + r * C::ROWB + 16 * ((dim >> 3) ^ C::swz(r)) + 2 * (dim & 7);
    }
    // tail (d = 72): group g reads dims 64..71 of the rows of k-step g & 1, half g >> 1
    if constexpr (C::TAIL) {
        const int r = krow<C::PERM>(4 * (grp >> 1) + (gi >> 2)) + 16 * (grp & 1);
        taddr = lds_u32 + r * C::ROWB + 2 * (32 * DBLK + 4 * (gi & 1));
    }
    uint32_t ra = lds_u32 + C::ROWBASE + 16 * hf;  // the rows' scalars
    constexpr int T2OFF = C::T2BASE;

    f32x16 acc1[KV ? DBLK : 1], acc2[DBLK];
    f32x4 tail1[2] = {}, tail2[2] = {};
#pragma unroll
    for (int db = 0; db < DBLK; ++db) {
        if constexpr (KV) acc1[db] = f32x16{};
        acc2[db] = f32x16{};
    }

    // The LDS reads of a block are issued by hand, ahead of their products, in
    // this order: the rows' scalars (KV), the 2 KSTEPS operands of X and Y, the
    // transposed operands of the sums.  They complete in issue order, so each
    // product waits for all but the reads issued after its own.
    // PIPE (d <= 72, where registers allow): the products of X and Y of a block
    // run among the exponentials of the block before it.
    constexpr bool PIPE = D <= 96;
    // operands of X and Y, and how far ahead they are read; products of the sums
    // (full blocks), how far ahead theirs, and how many of these before P and
    // dS: less in the sweeps of dK/dV whose registers would not do
    constexpr int OPS = 2 * KSTEPS, PF = !KV || D <= 64 ? 4 : 2;
    constexpr int SUMS = (KV ? 4 : 2) * DBLK, GF = 4, GP = KV && D > 96 ? 2 : GF;
    u32x4 ring[PF];
    // Addresses of the current stage: a register per operand where there are
    // few (one addition each per tile), otherwise derived at each read.
    constexpr bool HOLD = C::SWIZZLED && D <= 96;
    uint32_t ka[HOLD ? KSTEPS : 1], va0[HOLD ? DBLK : 1][2], kp = 0, ta = 0;
    auto k_stage = [&](uint32_t so) {
#pragma unroll
        for (int kk = 0; kk < (HOLD ? KSTEPS : 1); ++kk) ka[kk] = (k0 ^ (32 * kk)) + so;
        if constexpr (!C::SWIZZLED) kp = kpad + so;
    };
    auto v_stage = [&](uint32_t so) {
#pragma unroll
        for (int db = 0; db < (HOLD ? DBLK : 1); ++db)
#pragma unroll
            for (int e = 0; e < 2; ++e) va0[db][e] = (v0[e] ^ (64 * db)) + so;
        if constexpr (C::TAIL) ta = taddr + so;
    };
    // operand j of X (even) and Y (odd), block at OFF
    auto read_op = [&](auto off_c, auto j_c) {
        constexpr int OFF = decltype(off_c)::value, j = decltype(j_c)::value, kk = j / 2;
        constexpr int O = OFF + (j & 1 ? T2OFF : 0);
        if constexpr (HOLD) ring[j % PF] = lds_b128<O>(ka[kk]);
        else if constexpr (C::SWIZZLED) ring[j % PF] = lds_b128<O>(ka[0] ^ (32 * kk));
        else if constexpr (2 * kk + 1 < C::CH) ring[j % PF] = lds_b128<O + 32 * kk>(ka[0]);
        else ring[j % PF] = lds_b128<O>(kp);
    };
    auto first_ops = [&](auto off_c) {
        static_for<0, PF>([&](auto j) { read_op(off_c, j); });
    };
    u32x2 gr[GF][2], gt[2][2];
    // transposed operand m: acc1's (T2) blocks, k-step by k-step, then acc2's (T1)
    auto read_sum = [&](auto off_c, auto m_c) {
        constexpr int OFF = decltype(off_c)::value, m = decltype(m_c)::value;
        constexpr bool second = KV && m < 2 * DBLK;
        constexpr int ks = m / DBLK % 2, db = m % DBLK;
        constexpr int O = OFF + (second ? T2OFF : 0) + 16 * ks * C::ROWB;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if constexpr (HOLD) gr[m % GF][e] = tr_read<O>(va0[db][e]);
            else if constexpr (C::SWIZZLED) gr[m % GF][e] = tr_read<O>(va0[0][e] ^ (64 * db));
            else gr[m % GF][e] = tr_read<O + 64 * db>(va0[0][e]);
        }
    };
    auto read_tails = [&](auto off_c) {
        constexpr int OFF = decltype(off_c)::value;
        if constexpr (C::TAIL) {
            if constexpr (KV) {
                gt[0][0] = tr_read<OFF + T2OFF>(ta);
                gt[0][1] = tr_read<OFF + T2OFF + C::E_ROWS * C::ROWB>(ta);
            }
            gt[1][0] = tr_read<OFF>(ta);
            gt[1][1] = tr_read<OFF + C::E_ROWS * C::ROWB>(ta);
        }
    };
    // the tail's 16 rows: W of 32 streamed rows regrouped to the 16x16x32 layout
    auto tail_product = [&](const u32x2 (&t)[2], const bf16x8 (&w)[2], f32x4 (&tail)[2]) {
        const u32x4 x = __builtin_bit_cast(u32x4, w[0]), y = __builtin_bit_cast(u32x4, w[1]);
        u32x4 b0, b1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto r = __builtin_amdgcn_permlane16_swap(x[i], y[i], false, false);
            b0[i] = r[0];
            b1[i] = r[1];
        }
        const bf16x8 va = __builtin_bit_cast(bf16x8, u32x4{t[0][0], t[0][1], t[1][0], t[1][1]});
        tail[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, b0), tail[0], 0, 0, 0);
        tail[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, b1), tail[1], 0, 0, 0);
    };

    f32x16 ndv;  // what Y of dQ starts from: -D of the lane's row
    u32x4 xi[4], yi[4];  // and X and Y of dK/dV: the rows' scalars
    auto read_rows = [&](int t, auto kb_c) {
        constexpr int O = 256 * decltype(kb_c)::value;
        const uint32_t base = ra + (uint32_t)(t % NST) * C::ROWREGION;
        static_for<0, 4>([&](auto g_c) {
            constexpr int g = decltype(g_c)::value;
            xi[g] = lds_b128<O + 32 * g>(base);
            yi[g] = lds_b128<O + 128 + 32 * g>(base);
        });
    };
    auto start_rows = [&](f32x16& x, f32x16& y) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            asm volatile("" : "+v"(xi[g]), "+v"(yi[g]));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[4 * g + i] = __uint_as_float(xi[g][i]);
                y[4 * g + i] = __uint_as_float(yi[g][i]);
            }
        }
    };
    // the first reads of block kb of tile t
    auto start_block = [&](int t, auto kb_c) {
        constexpr int kb = decltype(kb_c)::value;
        if constexpr (kb == 0) k_stage((uint32_t)(t % NST) * C::REGION);
        if constexpr (KV && PIPE) read_rows(t, kb_c);
        first_ops(std::integral_constant<int, 32 * kb * C::ROWB>{});
    };
    // X and Y of block kb of tile t, whose first reads are in flight;
    // between(j) goes behind product j
    auto products = [&](int t, auto kb_c, f32x16& x, f32x16& y, auto&& between) {
        constexpr int kb = decltype(kb_c)::value;
        using Off = std::integral_constant<int, 32 * kb * C::ROWB>;
        // (opaque: the addresses derived from this are not kept in registers)
        if constexpr (C::SWIZZLED && !HOLD) asm volatile("" : "+v"(ka[0]));
        if constexpr (KV && !PIPE) {
            read_rows(t, kb_c);
            lds_wait_upto<0>();
            start_rows(x, y);
        }
        if constexpr (!KV) {
            x = f32x16{};
            y = ndv;
        }
        static_for<0, OPS>([&](auto j_c) {
            constexpr int j = decltype(j_c)::value;
            lgkm_wait_v4<(OPS - 1 - j < PF - 1 ? OPS - 1 - j : PF - 1)>(ring[j % PF]);
            if constexpr (KV && PIPE && j == 0) start_rows(x, y);  // read before the operand
            const bf16x8 op = __builtin_bit_cast(bf16x8, ring[j % PF]);
            if constexpr (j & 1) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, r2[j / 2], y, 0, 0, 0);
            else x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, r1[j / 2], x, 0, 0, 0);
            if constexpr (j + PF < OPS) read_op(Off{}, std::integral_constant<int, j + PF>{});
            between(j_c);
        });
    };
    // P and dS of 16 streamed rows of block kb of tile t (values 8ks .. 8ks + 7)
    bf16x8 pb[2], zb[2];
    auto weights = [&](int t, auto kb_c, auto ks_c, const f32x16& x, const f32x16& y) {
        constexpr int kb = decltype(kb_c)::value, ks = decltype(ks_c)::value;
        float p[8], z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            p[e] = __builtin_amdgcn_exp2f(KV ? x[8 * ks + e] * a.c2 : __builtin_fmaf(x[8 * ks + e], a.c2, nl));
        if constexpr (!KV)
            if ((tb + t + 1) * BN > a.Nt)  // streamed keys past the end have no probability
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 8 * ks + e;
                    if ((tb + t) * BN + 32 * kb + krow<C::PERM>(8 * (i >> 2) + 4 * hf + (i & 3)) >= a.Nt) p[e] = 0.f;
                }
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = p[e] * y[8 * ks + e];
        u32x4 pw, zw;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (KV) pw[w] = pack_bf16x2(p[2 * w], p[2 * w + 1]);
            zw[w] = pack_bf16x2(z[2 * w], z[2 * w + 1]);
        }
        if constexpr (KV) pb[ks] = __builtin_bit_cast(bf16x8, pw);
        zb[ks] = __builtin_bit_cast(bf16x8, zw);
    };
    // The sums over block kb of tile t (GP operands are in flight).  next()
    // issues the first reads of the block after the next products' one, behind
    // the last operand of the sums.
    auto sums = [&](auto kb_c, auto n_next, auto&& next) {
        constexpr int kb = decltype(kb_c)::value, NEXT = decltype(n_next)::value;  // reads that next() issues
        using Off = std::integral_constant<int, 32 * kb * C::ROWB>;
        static_for<GP, GF>([&](auto m) { read_sum(Off{}, m); });
        constexpr int LEFT = SUMS - GF;  // from here on no more operands are asked for, then the tails'
        constexpr int TAILS = C::TAIL ? (KV ? 4 : 2) : 0;
        static_for<0, SUMS>([&](auto m_c) {
            constexpr int m = decltype(m_c)::value;
            constexpr bool second = KV && m < 2 * DBLK;
            constexpr int ks = m / DBLK % 2, db = m % DBLK;
            if constexpr (m == LEFT) read_tails(Off{});
            if constexpr (m < LEFT) {
                lds_wait_upto<2 * (GF - 1)>(gr[m % GF][0], gr[m % GF][1]);
            } else {
                lds_wait_upto<2 * (SUMS - 1 - m) + TAILS + (m > LEFT ? NEXT : 0)>(gr[m % GF][0], gr[m % GF][1]);
                if constexpr (m == LEFT) next();
            }
            const bf16x8 va =
                __builtin_bit_cast(bf16x8, u32x4{gr[m % GF][0][0], gr[m % GF][0][1], gr[m % GF][1][0], gr[m % GF][1][1]});
            if constexpr (second) acc1[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[ks], acc1[db], 0, 0, 0);
            else acc2[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, zb[ks], acc2[db], 0, 0, 0);
            if constexpr (m + GF < SUMS) read_sum(Off{}, std::integral_constant<int, m + GF>{});
        });
        if constexpr (C::TAIL) {
            lds_wait_upto<NEXT>(gt[0][0], gt[0][1], gt[1][0], gt[1][1]);
            if constexpr (KV) tail_product(gt[0], pb, tail1);
            tail_product(gt[1], zb, tail2);
        }
    };
    // Tile t + 1 has landed in every wave (tile t + 2 may be in flight), and
    // every wave is done with tile t - 1, whose stage takes tile t + NST - 1.
    auto turn = [&](int t) {
        wait_tiles(std::integral_constant<int, NST - 3>{});
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load_tile(t + NST - 1, (t + NST - 1) % NST);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    constexpr int FIRST_READS = PF + (KV && PIPE ? 8 : 0);  // of start_block

    if (ntiles > 0) {
        // the first NST-1 tiles load whether or not there are that many (past
        // the end they read zeros, into stages nobody reads)
#pragma unroll
        for (int t = 0; t < NST - 1; ++t) load_tile(t, t);
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) asm volatile("" : "+v"(r1[kk]), "+v"(r2[kk]));
        asm volatile("" : "+v"(nl), "+v"(nd));
        if constexpr (!KV) {
            // a register per value, so that the first product takes it as it stands
#pragma unroll
            for (int i = 0; i < 16; ++i) ndv[i] = nd;
            asm volatile("" : "+v"(ndv));
        }
        wait_tiles(std::integral_constant<int, NST - 2>{});
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        f32x16 x0, y0, x1, y1;
        auto nothing = [](auto) {};
        using Reads = std::integral_constant<int, FIRST_READS>;
        if (rt * kRows + wave * 32 >= a.Nr) {
            // a wave whose rows all lie past the end only loads its share
            for (int t = 0; t < ntiles; ++t) turn(t);
        } else if constexpr (PIPE) {
            start_block(0, I0{});
            static_assert(!PIPE || NB == 2, "two blocks of a tile take turns");
            products(0, I0{}, x0, y0, nothing);
            start_block(0, I1{});
            for (int t = 0; t < ntiles; ++t) {
                // the exponentials of one block, eight at a time, behind the products
                // of the next block; the sums' first operands behind the last ones
                auto among = [&](auto kb_c, const f32x16& x, const f32x16& y) {
                    return [&, kb_c](auto j_c) {
                        constexpr int j = decltype(j_c)::value;
                        if constexpr (j == 0) weights(t, kb_c, I0{}, x, y);
                        if constexpr (j == OPS / 2) weights(t, kb_c, I1{}, x, y);
                        if constexpr (j == OPS - 1)
                            static_for<0, GP>([&](auto m) { read_sum(std::integral_constant<int, 32 * decltype(kb_c)::value * C::ROWB>{}, m); });
                    };
                };
                v_stage((uint32_t)(t % NST) * C::REGION);
                products(t, I1{}, x1, y1, among(I0{}, x0, y0));
                sums(I0{}, Reads{}, [&] {
                    turn(t);
                    start_block(t + 1, I0{});
                });
                products(t + 1, I0{}, x0, y0, among(I1{}, x1, y1));
                sums(I1{}, Reads{}, [&] { start_block(t + 1, I1{}); });
            }
        } else {
            static_assert(PIPE || NB == 1, "one block per tile");
            start_block(0, I0{});
            for (int t = 0; t < ntiles; ++t) {
                v_stage((uint32_t)(t % NST) * C::REGION);
                if constexpr (C::SWIZZLED && !HOLD) asm volatile("" : "+v"(va0[0][0]), "+v"(va0[0][1]));
                products(t, I0{}, x0, y0, nothing);
                static_for<0, GP>([&](auto m) { read_sum(I0{}, m); });
                turn(t);
                weights(t, I0{}, I0{}, x0, y0);
                weights(t, I0{}, I1{}, x0, y0);
                sums(I0{}, Reads{}, [&] { start_block(t + 1, I0{}); });
            }
        }
    }
    // the last block's look-ahead reads and the tiles past the end
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < PF; ++j) asm volatile("" : "+v"(ring[j]));
    if constexpr (KV && PIPE)
#pragma unroll
        for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(xi[g]), "+v"(yi[g]));
    wait_vmem<0>();

    // Results: lane c holds resident row 32 wave + c, dims 32db + 8g + 4hf + i;
    // the tail's lanes row 32 wave + 16h + (lane & 15), dims 64 + 4 (lane >> 4) + i
    auto put = [&](void* dst, int64_t part0, int r, int dim, f32x4 v) {
        if (r >= a.Nr) return;
        const int64_t at = ((int64_t)b * a.Nr + r) * rs + headoff + dim;
        if (a.splits > 1) {
            *(f32x4*)(a.part + part0 + (int64_t)sp * a.part_elems + at) = v;
        } else if (a.accum) {
            f32x4* p = (f32x4*)((float*)dst + at);
            *p = *p + v;
        } else {
            *(u32x2*)((uint16_t*)dst + at) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        }
    };
    auto result = [&](void* dst, int64_t part0, const f32x16* acc, const f32x4* tail, float f) {
        if (a.splits == 1 && !a.accum) {
            // stores of 16 bytes, 32 together: half hf takes both halves' dims
            // 8 (g + hf) .. + 7 (2 x 24 heads of 64, 128 x 4429: 46 us, 51 with
            // stores of 8 bytes; whole rows by way of LDS: the same)
#pragma unroll
            for (int db = 0; db < DBLK; ++db)
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    u32x4 w;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int v = 4 * g + 2 * i;
                        const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16x2(acc[db][v] * f, acc[db][v + 1] * f),
                                                                        pack_bf16x2(acc[db][v + 4] * f, acc[db][v + 5] * f), false, false);
                        w[i] = r[0];
                        w[2 + i] = r[1];
                    }
                    if (row < a.Nr)
                        *(u32x4*)((uint16_t*)dst + ((int64_t)b * a.Nr + row) * rs + headoff + 32 * db + 8 * (g + hf)) = w;
                }
        } else {
#pragma unroll
            for (int db = 0; db < DBLK; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    put(dst, part0, row, 32 * db + 8 * g + 4 * hf,
                        f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]} * f);
        }
        if constexpr (C::TAIL)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (grp < 2) put(dst, part0, rt * kRows + wave * 32 + 16 * h + gi, 32 * DBLK + 4 * grp, tail[h] * f);
    };
    result(a.o2, 0, acc2, tail2, a.scale);
    if constexpr (KV) result(a.o1, a.splits * a.part_elems, acc1, tail1, 1.f);
}

// Both sweeps in one launch: they need nothing of each other, and the shorter
// workgroups fill the CUs that the last of the longer ones leave.  The first
// n_first workgroups are those of the sweep whose workgroups take longer, dK/dV
// if kv_first.
template <int D>
__global__ __launch_bounds__(256, 2) void attn_bwd_kernel(BwdArgs kv, BwdArgs q, int n_first, int kv_first) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[BCfg<D, true>::LDS_BYTES];
    const int first = (int)blockIdx.x < n_first;
    const int id = first ? blockIdx.x : blockIdx.x - n_first, n = first ? n_first : gridDim.x - n_first;
    if (first == kv_first) sweep<D, true>(kv, lds, xcd_remap(id, n));
    else sweep<D, false>(q, lds, xcd_remap(id, n));
}

// Per query row: -l sqrt(d) and -D = e - g . o.  A row whose l is -inf (no
// key) gives -inf and 0: its probabilities are 0, and its o is not read.
// One row of a head per L lanes; a wave's rows are consecutive rows of one head.
struct RowsArgs {
    const char* out;
    const char* dout;
    const float* lse;
    const float* dlse;
    float* rows;
    int H, Nq, blocks;  // blocks of rows per head
    float root;         // sqrt(d)
};

template <int D, int ES>
__global__ __launch_bounds__(256) void bwd_rows_kernel(RowsArgs a) {
    constexpr int CH = D * ES / 16;                       // 16-byte chunks of a row
    constexpr int L = CH <= 8 ? 8 : CH <= 16 ? 16 : 32;   // lanes of a row
    constexpr int R = 256 / L;                            // rows at a time
    const int p = threadIdx.x % L, r = threadIdx.x / L;
    const int bh = blockIdx.x / a.blocks, blk = blockIdx.x % a.blocks;
    const int hh = bh % a.H;
    const int64_t b = bh / a.H;
    const int i = blk * R + r;
    if (i >= a.Nq) return;
    const int64_t at = (((b * a.Nq + i) * a.H + hh) * CH + p) * 16;
    const int64_t li = (int64_t)bh * a.Nq + i;
    const float l = a.lse[li];
    float s = 0.f;
    if (p < CH) {
        const u32x4 x = *(const u32x4*)(a.out + at), g = *(const u32x4*)(a.dout + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (ES == 2) {
                s = __builtin_fmaf(__uint_as_float(x[e] << 16), __uint_as_float(g[e] << 16), s);
                s = __builtin_fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(g[e] & 0xffff0000u), s);
            } else {
                s = __builtin_fmaf(__uint_as_float(x[e]), __uint_as_float(g[e]), s);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < L; o *= 2) s += __shfl_xor(s, o);
    if (p == 0) {
        const bool none = l == -INFINITY;
        float* rows = a.rows + (int64_t)bh * 2 * a.Nq;
        rows[i] = none ? -INFINITY : -l * a.root;
        rows[a.Nq + i] = none ? 0.f : (a.dlse ? a.dlse[li] - s : -s);
    }
}

// The sums of cut sweeps' partials, in order, into the results (blockIdx.y).
struct JoinArgs {
    const float* part[3];
    void* dst[3];
    int64_t elems[3];
    int splits[3], accum[3];
};

template <bool BF16>
__global__ __launch_bounds__(256) void bwd_join_kernel(JoinArgs a) {
    const int y = blockIdx.y;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, n = a.elems[y];
    if (i >= n) return;
    const float* part = a.part[y] + i;
    f32x4 v = *(const f32x4*)part;
    for (int s = 1; s < a.splits[y]; ++s) v += *(const f32x4*)(part + s * n);
    if (a.accum[y]) {
        f32x4* p = (f32x4*)((float*)a.dst[y] + i);
        *p = *p + v;
    } else if (BF16) {
        *(u32x2*)((uint16_t*)a.dst[y] + i) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    } else {
        *(f32x4*)((float*)a.dst[y] + i) = v;
    }
}

template <int D>
hipError_t launch_rows(const AttnBwdParams& p, const RowsArgs& a0, hipStream_t s) {
    RowsArgs a = a0;
    const int es = p.bf16 ? 2 : 4, ch = D * es / 16;
    const int R = 256 / (ch <= 8 ? 8 : ch <= 16 ? 16 : 32);
    a.blocks = (p.Nq + R - 1) / R;
    const dim3 grid((unsigned)((int64_t)p.B * p.H * a.blocks)), block(256);
    if (p.bf16) hipLaunchKernelGGL((bwd_rows_kernel<D, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((bwd_rows_kernel<D, 4>), grid, block, 0, s, a);
    return hipGetLastError();
}

// kv: the dK/dV sweep's arguments, else the dQ sweep's
BwdArgs sweep_args(const AttnBwdParams& p, bool kv) {
    BwdArgs a{};
    a.r1 = (const uint16_t*)(kv ? p.k : p.q);
    a.r2 = (const uint16_t*)(kv ? p.v : p.dout);
    a.t1 = (const uint16_t*)(kv ? p.q : p.k);
    a.t2 = (const uint16_t*)(kv ? p.dout : p.v);
    a.rows = p.rows;
    a.o1 = p.dv;
    a.o2 = kv ? p.dk : p.dq;
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

int64_t workgroups(const BwdArgs& a) { return (int64_t)a.B * a.H * a.r_tiles * a.splits; }

template <int D>
hipError_t launch_sweeps(const BwdArgs& kv, const BwdArgs& q, hipStream_t s) {
    const int64_t n_kv = workgroups(kv), n_q = workgroups(q);
    if (n_kv + n_q == 0) return hipSuccess;
    const int kv_first = 4 * (int64_t)kv.Nt * q.splits >= 3 * (int64_t)q.Nt * kv.splits;
    hipLaunchKernelGGL(attn_bwd_kernel<D>, dim3((unsigned)(n_kv + n_q)), dim3(256), 0, s, kv, q,
                       (int)(kv_first ? n_kv : n_q), kv_first);
    return hipGetLastError();
}

}  // namespace

// Ranks the cuts of a call by a model of its launch, in units near a microsecond
// but no times: of its own choice it gives 0.6 to 1.5 times what is measured.  A
// workgroup takes 6 (operands, first tiles, results) plus, per block of 32 streamed
// rows, `unit` for each of its products (4 for dK and dV, 3 for dQ) with another
// workgroup on its CU.  512 workgroups run at once (float32 at d <= 72: up to 768,
// counted as 512); where they are fewer, the longest decides, at 0.65 of its time
// if it has its CU to itself; more of them take their sum's share and most of one
// of the shorter ones, which come last, or as long as the longest.  Cut sweeps add
// the join: a launch, and partials written and read at 2 TB/s.
// Measured in one part, and in the best, us: 2 x 16 heads of 72, 1024 x 1024 47
// (dQ in 2: 53); 24 heads of 128, 512 x 4224 112, dQ in 2 101; 2 x 24 heads of
// 64, 333 x 4429 81; 24 heads of 64, 1 x 4429 54, dQ in 4 24; 24 heads of 128,
// 4224 x 64 129, dK/dV in 8 45; 3 heads of 128, 4224 x 4224 127, dQ in 3 and
// dK/dV in 2 101; one head of 64, 8000 x 8000 118, dQ in 4 and dK/dV in 4 65;
// float32, 2 heads of 64, 256 x 64 25, dQ in 2 and dK/dV in 8 13.  (One state per
// call and short runs; calls among others on states in turn take 43 and 83 for the
// first and the third.)  Over 86 calls timed under all cuts the choice takes 2.0 %
// more time than the best in the mean; farthest off are float32, 12 heads of
// 128, 85 x 592 (dQ in 6 38, in 4 29) and then four calls by 8 to 11 %; one, 12
// heads of 128, 1100 x 4000, takes 6 % more than uncut.
BwdSplits bwd_splits(int64_t bh, int64_t Nq, int64_t Nk, int D, bool bf16) {
    BwdSplits best{1, 1, bf16 ? kRows : 64};
    const int tile = bf16 && D <= 96 ? 64 : 32;
    const double unit = bf16 ? (D == 64 ? 0.247 : D == 72 ? 0.296 : 0.465) : (D == 64 ? 1.15 : D == 72 ? 1.33 : 2.2);
    constexpr int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16};
    constexpr int64_t kSlots = 512;
    const int64_t wgs[2] = {bh * ((Nq + best.rows - 1) / best.rows), bh * ((Nk + best.rows - 1) / best.rows)};
    const int64_t tiles[2] = {(Nk + tile - 1) / tile, (Nq + tile - 1) / tile};
    double each[2][8], join[2][8];
    for (int w = 0; w < 2; ++w)
        for (int i = 0; i < 8; ++i) {
            const int s = kParts[i];
            each[w][i] = s > 1 && (s > tiles[w] || s * wgs[w] > 2 * kSlots)
                             ? -1.
                             : 6. + (double)((tiles[w] + s - 1) / s * (tile / 32) * (w ? 4 : 3)) * unit;
            join[w][i] = s > 1 ? 2. * (w ? 8. : 4.) * (double)(bh * (w ? Nk : Nq) * D) * s / 2e6 : 0.;
        }
    double least = INFINITY;
    for (int i = 0; i < 8; ++i)
        for (int j = 0; j < 8; ++j) {
            const double q = each[0][i], k = each[1][j];
            if (q < 0. || k < 0.) continue;
            const int64_t nq = wgs[0] * kParts[i], nk = wgs[1] * kParts[j], n = nq + nk;
            const double sum = ((double)nq * q + (double)nk * k) / kSlots;
            const double longest = wgs[0] == 0 ? k : wgs[1] == 0 ? q : fmax(q, k), shortest = fmin(q, k);
            double t = n <= kSlots / 2 ? 0.65 * longest
                       : n <= kSlots   ? fmax(sum, longest * (0.65 + 0.35 * (double)(n - kSlots / 2) / (kSlots / 2)))
                                       : fmax(sum + 0.7 * shortest, longest);
            if (i + j > 0) t += 4. + join[0][i] + join[1][j];
            if (t < least) {
                least = t;
                best.q = kParts[i];
                best.kv = kParts[j];
            }
        }
    return best;
}

hipError_t launch_bwd_join(const AttnBwdParams& p, hipStream_t s) {
    JoinArgs a{};
    int n = 0;
    int64_t most = 0;
    auto add = [&](const float* part, void* dst, int64_t elems, int splits, int accum) {
        a.part[n] = part, a.dst[n] = dst, a.elems[n] = elems, a.splits[n] = splits, a.accum[n] = accum;
        if (elems > most) most = elems;
        ++n;
    };
    const int64_t nq = (int64_t)p.B * p.Nq * p.H * p.D, nk = (int64_t)p.B * p.Nk * p.H * p.D;
    if (p.q_splits > 1) add(p.q_part, p.dq, nq, p.q_splits, p.accum_q);
    if (p.kv_splits > 1) {
        add(p.kv_part, p.dk, nk, p.kv_splits, p.accum_kv);
        add(p.kv_part + p.kv_splits * nk, p.dv, nk, p.kv_splits, p.accum_kv);
    }
    if (most == 0) return hipSuccess;
    const dim3 grid((unsigned)((most / 4 + 255) / 256), (unsigned)n), block(256);
    if (p.bf16) hipLaunchKernelGGL(bwd_join_kernel<true>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(bwd_join_kernel<false>, grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_bwd_rows(const AttnBwdParams& p, hipStream_t s) {
    RowsArgs a{};
    a.out = (const char*)p.out, a.dout = (const char*)p.dout, a.lse = p.lse, a.dlse = p.dlse, a.rows = p.rows;
    a.H = p.H, a.Nq = p.Nq, a.root = sqrtf((float)p.D);
    if ((int64_t)p.B * p.H * p.Nq == 0) return hipSuccess;
    if (p.D == 64) return launch_rows<64>(p, a, s);
    if (p.D == 72) return launch_rows<72>(p, a, s);
    return launch_rows<128>(p, a, s);
}

hipError_t launch_attn_bwd_bf16(const AttnBwdParams& p, hipStream_t s) {
    const BwdArgs kv = sweep_args(p, true), q = sweep_args(p, false);
    if (p.D == 64) return launch_sweeps<64>(kv, q, s);
    if (p.D == 72) return launch_sweeps<72>(kv, q, s);
    return launch_sweeps<128>(kv, q, s);
}

}  // namespace xdit
