// C = P Q^T on the 16-bit matrix cores (v_mfma_f32_16x16x32, sums in 32 bits), for operands whose rows run along the inner
// dimension in slabs of 128 bytes (weights_internal.h). One slice: the ordinary product. Two slices of fp16 (value = first +
// second, 22 bits and more): the products first*first, first*second and second*first of the same fragments, which leaves out
// what is below 2^-22 of a term; a slab then holds both slices of 32 positions, so loads and shared memory are the same and only
// the pairs differ.
//
// A workgroup owns a BM x BN tile. A slab of its rows of P and Q is brought into LDS by direct loads (1 KiB = 8 rows a wavefront and load;
// the lane that fetches 16-byte piece c of row r puts it at place c ^ (r % 8), so that the 16 lanes of a fragment read, ds_read_b128, meet
// all banks), STAGES - 1 slabs ahead of the one that is multiplied: one barrier per slab. Rows beyond the last are read from the last one
// and their results dropped. With fewer tiles than run at a time, or a last round of them that is far from full, several workgroups share a
// tile's inner dimension; their sums go through memory and a second launch adds them up in a fixed order (4096 x 4096 symmetric, 528 tiles
// of 128 where 512 run at a time: 253 us whole). The fragments of Q are the MFMA's first operand: a lane then holds four consecutive
// columns of one row of C.
#pragma once

#include <algorithm>

#include "half_common.h"

namespace ozimmu {
namespace {

// How the tiles of all matrices (numbered through) are dealt to workgroups: the first `whole` to one each, the others to `parts` each, with
// `part_slabs` slabs of the inner dimension.
struct NtPlan {
    int tiles_m, tiles_n, tiles;   // of a matrix
    int whole, parts, part_slabs;
};

__device__ __forceinline__ void nt_tile(const NtArgs& a, const NtPlan& p, int tile, int& tm, int& tn, int& z) {
    z = tile / p.tiles;
    tile -= z * p.tiles;
    if (a.symmetric) {   // tiles on and above the diagonal, row by row of tiles
        for (tm = 0; tile >= p.tiles_m - tm; ++tm) tile -= p.tiles_m - tm;
        tn = tm + tile;
    } else {
        tile_of_logical(tile, p.tiles_m, p.tiles_n, tm, tn);
    }
}

// What becomes of the sums of four neighbouring elements C[row][col .. col + 3]. Two slices: `both` receives them, the first in the low
// half; the transposed matrix is the caller's.
template <int RESULT>
__device__ __forceinline__ void nt_finish(const NtArgs& a, int z, int r, int c, const v4f& acc, unsigned (&both)[4]) {
    if constexpr (RESULT == kOutSlices) {
        const int m_pad = (a.m + 31) & ~31, n_pad = (a.n + 31) & ~31;
        if (c >= n_pad || r >= m_pad) return;
        unsigned short* C = a.C + z * a.batch_c;
        const int64_t at = (int64_t)r * a.ldc + (c >> 5) * 64 + (c & 31);
        unsigned short h[4], l[4];
        unsigned short ih[4] = {}, il[4] = {};
        if (a.in && r < a.m) {
            const unsigned short* in = a.in + z * a.batch_c;
            *reinterpret_cast<v2u*>(ih) = *reinterpret_cast<const v2u*>(in + at);
            *reinterpret_cast<v2u*>(il) = *reinterpret_cast<const v2u*>(in + at + 32);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = a.factor * acc[e];
            if (a.in) v = fmaf(a.beta, f16_to_f32(ih[e]) + f16_to_f32(il[e]), v);
            if (r == c + e) v += a.diagonal;
            if (c + e >= a.n || r >= a.m) v = 0.f;   // the padding of a row holds zeros
            two_slices(v, h[e], l[e]);
            both[e] = (unsigned)h[e] | (unsigned)l[e] << 16;
        }
        if (r < a.m) {
            *reinterpret_cast<v2u*>(C + at) = *reinterpret_cast<v2u*>(h);
            *reinterpret_cast<v2u*>(C + at + 32) = *reinterpret_cast<v2u*>(l);
        }
    } else {
        typedef Elem<RESULT == kOutF32 ? OZIMMU_F32 : RESULT == kOutBf16 ? OZIMMU_BF16 : OZIMMU_F16> E;
        typedef typename E::raw raw;
        typedef raw raw4 __attribute__((ext_vector_type(4)));
        if (r >= a.m || c >= a.n) return;
        raw* out = reinterpret_cast<raw*>(a.out) + z * a.batch_o;
        const bool wide = (a.ldo & 3) == 0 && (a.batch_o & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & (4 * sizeof(raw) - 1)) == 0;
        const int ep = RESULT == kOutF32 && a.exp_p ? a.exp_p[r] : 0;
        raw4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = a.factor * acc[e];
            if (RESULT == kOutF32 && a.exp_p) x = ldexpf(x, ep + a.exp_q[min(c + e, a.n - 1) / a.q_run]);
            v[e] = E::store(x);
        }
        raw* at = out + (int64_t)r * a.ldo + c;
        if (wide && c + 4 <= a.n)
            *reinterpret_cast<raw4*>(at) = v;
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.n) at[e] = v[e];
    }
}

// When a wavefront reads its fragments of a slab from LDS: in the slab, all of them in the one before, or those that its first MFMAs need
// in the one before.
enum NtWalk { kReadOnTime, kReadAhead, kFirstReadsAhead };

template <int BM, int BN, int WM, int WN, int STAGES, int WALK, int SLICES, bool BF16, int RESULT>
__launch_bounds__(WM * WN * 64)
__global__ void nt_product_kernel(NtArgs a, NtPlan plan) {
    constexpr int W = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LP = BM / 8 / W, LQ = BN / 8 / W;   // direct loads per wavefront and slab
    constexpr unsigned kStage = (BM + BN) * 128;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile, slab0 = 0, slabs = a.slabs;
    const bool shared = (int)blockIdx.x >= plan.whole;
    if (shared) {
        const int b = blockIdx.x - plan.whole, part = b % plan.parts;
        tile = plan.whole + b / plan.parts;
        slab0 = part * plan.part_slabs;
        slabs = min(plan.part_slabs, a.slabs - slab0);
    } else {
        int first, count;
        xcd_tile_range(blockIdx.x & 7, plan.whole, first, count);
        tile = first + (blockIdx.x >> 3);
    }
    int tm, tn, z;
    nt_tile(a, plan, tile, tm, tn, z);
    const int row0 = tm * BM, col0 = tn * BN;
    const unsigned char* P = reinterpret_cast<const unsigned char*>(a.P + z * a.batch_p + (int64_t)row0 * a.ldp) + (int64_t)slab0 * 128;
    const unsigned char* Q = reinterpret_cast<const unsigned char*>(a.Q + z * a.batch_q + (int64_t)col0 * a.ldq) + (int64_t)slab0 * 128;
    const unsigned piece = ((lane & 7) ^ (lane >> 3)) * 16;
    unsigned voff_p[LP], voff_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) voff_p[i] = (unsigned)min((wave * LP + i) * 8 + (lane >> 3), a.m - 1 - row0) * (unsigned)(2 * a.ldp) + piece;
#pragma unroll
    for (int i = 0; i < LQ; ++i) voff_q[i] = (unsigned)min((wave * LQ + i) * 8 + (lane >> 3), a.n - 1 - col0) * (unsigned)(2 * a.ldq) + piece;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);

    // direct load `i` of this wavefront's LP + LQ for a slab
    auto load = [&](int i, int slab, int stage) {
        const unsigned at = lds0 + stage * kStage;
        if (i < LP)
            dma_load16<0>(P + (int64_t)slab * 128, voff_p[i], at + (wave * LP + i) * 1024);
        else
            dma_load16<0>(Q + (int64_t)slab * 128, voff_q[i - LP], at + BM * 128 + (wave * LQ + i - LP) * 1024);
    };

    const int wm = wave / WN, wn = wave % WN;
    // a lane's 16 bytes of a fragment: row lane % 16, piece lane / 16 (+ 4 for the second half of the slab)
    const unsigned frag0 = (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) * 16);
    const unsigned frag1 = (lane & 15) * 128 + ((((lane >> 4) + 4) ^ (lane & 7)) * 16);
    v4f acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    auto row_of_products = [&](int i, const v4u& a0, const v4u& a1, const v4u (&q0)[NI], const v4u (&q1)[NI]) {
        if constexpr (SLICES == 1) {
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], a0, acc[i][j]);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q1[j], a1, acc[i][j]);
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q1[j], a0, acc[i][j]);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], a1, acc[i][j]);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], a0, acc[i][j]);
        }
    };
    constexpr int AHEAD = WALK == kReadAhead ? STAGES : STAGES - 1;   // slabs requested before the first is multiplied
    for (int i = 0; i < AHEAD; ++i)
        if (i < slabs)
#pragma unroll
            for (int l = 0; l < LP + LQ; ++l) load(l, i, i);
    if constexpr (WALK == kReadAhead) {
        // The fragments of the next slab are read from LDS while this one's are multiplied; a slab's stage is requested anew as soon as its
        // fragments are in registers.
        struct Frags {
            v4u p0[MI], p1[MI], q0[NI], q1[NI];
        } f[2];
        auto read = [&](Frags& to, int stage) {
            const unsigned char* at_p = lds + stage * kStage + wm * (BM / WM) * 128;
            const unsigned char* at_q = lds + stage * kStage + BM * 128 + wn * (BN / WN) * 128;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                to.q0[j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag0);
                to.q1[j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag1);
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                to.p0[i] = *reinterpret_cast<const v4u*>(at_p + i * 2048 + frag0);
                to.p1[i] = *reinterpret_cast<const v4u*>(at_p + i * 2048 + frag1);
            }
        };
        if (AHEAD <= slabs)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * (LP + LQ)) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read(f[0], 0);
        int stage = 0;
        auto step = [&](int slab, Frags& now, Frags& next) {
            // the next slab has landed and this one's fragments are in registers; behind the barrier, everyone's
            if (slab + STAGES <= slabs)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * (LP + LQ)) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int free = stage;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (slab + 1 < slabs) read(next, stage);
            const bool more = slab + STAGES < slabs;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (more)
#pragma unroll
                    for (int l = (LP + LQ) * i / MI; l < (LP + LQ) * (i + 1) / MI; ++l) load(l, slab + STAGES, free);
                row_of_products(i, now.p0[i], now.p1[i], now.q0, now.q1);
            }
        };
        int slab = 0;
        for (; slab + 1 < slabs; slab += 2) {
            step(slab, f[0], f[1]);
            step(slab + 1, f[1], f[0]);
        }
        if (slab < slabs) step(slab, f[0], f[1]);
    } else if constexpr (WALK == kFirstReadsAhead) {
        // Two stages, two barriers a slab: behind the first nobody reads the other stage any more, and its loads go out between the first
        // rows of MFMAs; behind the second, near the end, they have landed, and the next slab's first fragments are read under the last
        // MFMAs.
        static_assert(STAGES == 2 && MI >= 4);
        v4u q0[2][NI], q1[2][NI], p0[2], p1[2];
        auto first_reads = [&](int stage, int to) {
            const unsigned char* at_p = lds + stage * kStage + wm * (BM / WM) * 128;
            const unsigned char* at_q = lds + stage * kStage + BM * 128 + wn * (BN / WN) * 128;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                q0[to][j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag0);
                q1[to][j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag1);
            }
            p0[0] = *reinterpret_cast<const v4u*>(at_p + frag0);
            p1[0] = *reinterpret_cast<const v4u*>(at_p + frag1);
        };
        constexpr int kLoadRows = MI / 2;
        auto step = [&](int slab, auto odd) {
            constexpr int now = decltype(odd)::value;
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const bool more = slab + 1 < slabs;
            const unsigned char* at_p = lds + now * kStage + wm * (BM / WM) * 128;
            static_for<0, MI>([&](auto row) {
                constexpr int i = decltype(row)::value;
                const v4u a0 = p0[i & 1], a1 = p1[i & 1];
                if constexpr (i + 1 < MI) {
                    p0[(i + 1) & 1] = *reinterpret_cast<const v4u*>(at_p + (i + 1) * 2048 + frag0);
                    p1[(i + 1) & 1] = *reinterpret_cast<const v4u*>(at_p + (i + 1) * 2048 + frag1);
                }
                if constexpr (i < kLoadRows) {
                    if (more)
#pragma unroll
                        for (int l = (LP + LQ) * i / kLoadRows; l < (LP + LQ) * (i + 1) / kLoadRows; ++l) load(l, slab + 1, now ^ 1);
                }
                if constexpr (i + 1 == MI) {
                    if (more) {
                        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
                        first_reads(now ^ 1, now ^ 1);
                    }
                }
                row_of_products(i, a0, a1, q0[now], q1[now]);
            });
        };
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        first_reads(0, 0);
        int slab = 0;
        for (; slab + 1 < slabs; slab += 2) {
            step(slab, std::integral_constant<int, 0>{});
            step(slab + 1, std::integral_constant<int, 1>{});
        }
        if (slab < slabs) step(slab, std::integral_constant<int, 0>{});
    } else {
        int stage = 0;
        for (int slab = 0; slab < slabs; ++slab) {
            // this wavefront's loads of the slab have landed (later ones may be on their way) and its reads of the stage that is loaded
            // next are done; behind the barrier, everyone's
            if (slab + AHEAD <= slabs)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * (LP + LQ)) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int to = stage == 0 ? AHEAD : stage - 1;
            const unsigned char* at_p = lds + stage * kStage + wm * (BM / WM) * 128;
            const unsigned char* at_q = lds + stage * kStage + BM * 128 + wn * (BN / WN) * 128;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (slab + AHEAD < slabs)
#pragma unroll
                for (int l = 0; l < LP + LQ; ++l) load(l, slab + AHEAD, to);
            v4u q0[NI], q1[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                q0[j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag0);
                q1[j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + frag1);
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const v4u p0 = *reinterpret_cast<const v4u*>(at_p + i * 2048 + frag0);
                const v4u p1 = *reinterpret_cast<const v4u*>(at_p + i * 2048 + frag1);
                row_of_products(i, p0, p1, q0, q1);
            }
        }
    }

    // ---- results: lane holds C[row][col .. col + 3]
    if (shared) {
        v4f* to = reinterpret_cast<v4f*>(a.partial) + (int64_t)(blockIdx.x - plan.whole) * (MI * NI * W * 64) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) to[(i * NI + j) * (W * 64)] = acc[i][j];
        return;
    }
    const int r0 = wm * (BM / WM) + (lane & 15), c0 = wn * (BN / WN) + (lane >> 4) * 4;   // in the tile
    // The transposed tile goes through LDS, which nobody reads any more: stored from the registers it would be two bytes at a time (4096 x
    // 4096: 27 us of 323). kAtOnce columns of it fit; value (row, col) lies at row ^ 16 (col / 4 % 4) of its column, so that the four
    // quarters of a wavefront meet different banks.
    constexpr int kAtOnce = STAGES * (BM + BN) * 128 / (BM * 4) < BN ? BN / 2 : BN;
    static_assert(kAtOnce * BM * 4 <= STAGES * (BM + BN) * 128 && kAtOnce % (BN / WN) == 0);
    unsigned* const turned = reinterpret_cast<unsigned*>(lds);
    const bool mirror = RESULT == kOutSlices && a.CT && !(a.symmetric && tm == tn);
#pragma unroll 1
    for (int part = 0; part < BN / kAtOnce; ++part) {
        if (mirror) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (wn / (kAtOnce / (BN / WN)) == part) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    unsigned both[4] = {};
                    const int r = r0 + 16 * i, c = c0 + 16 * j;
                    nt_finish<RESULT>(a, z, row0 + r, col0 + c, acc[i][j], both);
                    if (mirror) {
                        const int here = c - part * kAtOnce;
#pragma unroll
                        for (int e = 0; e < 4; ++e) turned[(here + e) * BM + (r ^ ((here >> 2 & 3) << 4))] = both[e];
                    }
                }
        }
        if (!mirror) continue;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        unsigned short* CT = a.CT + z * a.batch_ct;
        const int m_pad = (a.m + 31) & ~31;
        for (int piece = threadIdx.x; piece < kAtOnce * BM / 8; piece += W * 64) {
            const int here = piece / (BM / 8), r = piece % (BM / 8) * 8;
            const int64_t col = col0 + part * kAtOnce + here, row = row0 + r;
            if (col >= a.n || row >= m_pad) continue;
            const unsigned* from = turned + here * BM + (r ^ ((here >> 2 & 3) << 4));
            const v4u x = reinterpret_cast<const v4u*>(from)[0], y = reinterpret_cast<const v4u*>(from)[1];
            unsigned short* to = CT + col * a.ldct + (row >> 5) * 64 + (row & 31);
            *reinterpret_cast<v4u*>(to) = v4u{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u),
                                              __builtin_amdgcn_perm(y[1], y[0], 0x05040100u), __builtin_amdgcn_perm(y[3], y[2], 0x05040100u)};
            *reinterpret_cast<v4u*>(to + 32) = v4u{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u),
                                                   __builtin_amdgcn_perm(y[1], y[0], 0x07060302u), __builtin_amdgcn_perm(y[3], y[2], 0x07060302u)};
        }
    }
}

// The shared tiles: parts added up in order, a workgroup per 16 x 16 result of its wavefronts.
template <int BM, int BN, int WM, int WN, int RESULT>
__launch_bounds__(WM * WN * 64)
__global__ void nt_join_kernel(NtArgs a, NtPlan plan) {
    constexpr int W = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
    const int i = blockIdx.y / NI, j = blockIdx.y % NI;
    int tm, tn, z;
    nt_tile(a, plan, plan.whole + blockIdx.x, tm, tn, z);
    const v4f* from = reinterpret_cast<const v4f*>(a.partial) + ((int64_t)blockIdx.x * plan.parts * (MI * NI) + blockIdx.y) * (W * 64) + threadIdx.x;
    v4f sum = from[0];
    for (int p = 1; p < plan.parts; ++p) {
        const v4f x = from[(int64_t)p * (MI * NI * W * 64)];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    const int r = tm * BM + wm * (BM / WM) + (lane & 15) + 16 * i, c = tn * BN + wn * (BN / WN) + (lane >> 4) * 4 + 16 * j;
    unsigned both[4] = {};
    nt_finish<RESULT>(a, z, r, c, sum, both);
    if (RESULT == kOutSlices && a.CT && !(a.symmetric && tm == tn) && r < ((a.m + 31) & ~31)) {
        unsigned short* CT = a.CT + z * a.batch_ct;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.n) {
                const int64_t t = (int64_t)(c + e) * a.ldct + (r >> 5) * 64 + (r & 31);
                CT[t] = (unsigned short)both[e];
                CT[t + 32] = (unsigned short)(both[e] >> 16);
            }
    }
}

// A tile shape as the choice sees it: how many workgroups run at a time, and what a slab takes then and with one workgroup to a compute
// unit (us).
struct NtShape {
    int tile, slots;
    double full, alone;
};
struct NtChoice {
    NtPlan plan;
    double us;
};
inline NtChoice nt_choose(const NtArgs& a, const NtShape& s, size_t part_bytes) {
    NtChoice c{};
    c.plan.tiles_m = (a.m + s.tile - 1) / s.tile;
    c.plan.tiles_n = (a.n + s.tile - 1) / s.tile;
    const int64_t one = a.symmetric ? (int64_t)c.plan.tiles_m * (c.plan.tiles_m + 1) / 2 : (int64_t)c.plan.tiles_m * c.plan.tiles_n, all = one * a.batch;
    c.us = 1e30;
    if (all > INT32_MAX / 64) return c;
    c.plan.tiles = (int)one;
    auto round_us = [&](int64_t workgroups, int64_t slabs) {   // of a round of at most s.slots: what the fullest compute unit takes
        const double deepest = (double)((workgroups + kComputeUnits - 1) / kComputeUnits), most = (double)(s.slots / kComputeUnits);
        return (double)slabs * (s.alone + (s.full - s.alone) * (most > 1.0 ? (deepest - 1.0) / (most - 1.0) : 0.0));
    };
    const int64_t rounds = all / s.slots, rest = all % s.slots;
    c.plan.whole = (int)all;
    c.plan.parts = 1;
    c.plan.part_slabs = a.slabs;
    c.us = rounds * round_us(s.slots, a.slabs) + (rest ? round_us(rest, a.slabs) : 0.0);
    // the tiles of a last round that is not full may be shared, at the price of their sums' way through memory and of a launch
    if (rest && a.partial) {
        for (int64_t parts = 2; parts <= 32 && rest * parts <= s.slots && parts * 4 <= a.slabs; ++parts) {
            const int64_t slabs = (a.slabs + parts - 1) / parts, used = (a.slabs + slabs - 1) / slabs;
            const double bytes = (double)(rest * used) * s.tile * s.tile * sizeof(float);
            if (used != parts || bytes > (double)part_bytes) continue;
            const double us = rounds * round_us(s.slots, a.slabs) + round_us(rest * parts, slabs) + 5.0 + 2.0 * bytes / 4.0e6;
            if (us < c.us) {
                c.us = us;
                c.plan.whole = (int)(all - rest);
                c.plan.parts = (int)parts;
                c.plan.part_slabs = (int)slabs;
            }
        }
    }
    return c;
}

template <int BM, int BN, int WM, int WN, int STAGES, int WALK, int SLICES, bool BF16, int RESULT>
hipError_t launch_nt_tile(const NtArgs& a, const NtPlan& plan, hipStream_t st) {
    constexpr auto kernel = nt_product_kernel<BM, BN, WM, WN, STAGES, WALK, SLICES, BF16, RESULT>;
    constexpr int bytes = STAGES * (BM + BN) * 128;
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
    const int rest = plan.tiles * a.batch - plan.whole;
    kernel<<<dim3((unsigned)(plan.whole + rest * plan.parts)), dim3(WM * WN * 64), bytes, st>>>(a, plan);
    if (rest) nt_join_kernel<BM, BN, WM, WN, RESULT><<<dim3((unsigned)rest, BM / WM / 16 * (BN / WN / 16)), dim3(WM * WN * 64), 0, st>>>(a, plan);
    return hipGetLastError();
}

// A larger tile moves fewer bytes through LDS per product, a smaller one keeps more compute units busy: by an estimate from what a slab
// takes each shape (two slices, one slice; measured with products of one to four rounds). 64 x 64 tiles come in two forms: with about one
// workgroup to a compute unit nothing else hides a wavefront's LDS reads, and they run a slab ahead; with more, the registers and LDS of
// that cost the co-residents that do (2048 x 2048 x 8192, 528 tiles, 131 us against 162).
template <int SLICES, bool BF16, int RESULT>
hipError_t launch_nt(const NtArgs& a, hipStream_t st) {
    if (a.m <= 0 || a.n <= 0 || a.slabs <= 0 || a.batch <= 0 || (a.symmetric && a.m != a.n)) return hipErrorInvalidValue;
    constexpr bool two = SLICES == 2;
    const NtShape shapes[] = {{256, 256, two ? 2.41 : 1.73, two ? 2.41 : 1.73}, {128, 512, two ? 1.31 : 0.95, two ? 0.92 : 0.62}, {64, 1280, two ? 1.0 : 0.9, two ? 0.40 : 0.37}, {64, 768, two ? 0.75 : 0.66, two ? 0.31 : 0.27}};
    NtChoice best{};
    int which = -1;
    for (int i = 0; i < 4; ++i) {
        const NtChoice c = nt_choose(a, shapes[i], a.partial_bytes);
        if (which < 0 || c.us < best.us) {
            best = c;
            which = i;
        }
    }
    if (best.us >= 1e30) return hipErrorInvalidConfiguration;
    switch (which) {
        case 0: return launch_nt_tile<256, 256, 2, 4, 2, kFirstReadsAhead, SLICES, BF16, RESULT>(a, best.plan, st);
        case 1: return launch_nt_tile<128, 128, 2, 2, 2, kReadOnTime, SLICES, BF16, RESULT>(a, best.plan, st);
        case 2: return launch_nt_tile<64, 64, 2, 2, 2, kReadOnTime, SLICES, BF16, RESULT>(a, best.plan, st);
        default: return launch_nt_tile<64, 64, 2, 2, 3, kReadAhead, SLICES, BF16, RESULT>(a, best.plan, st);
    }
}

}  // namespace
}  // namespace ozimmu
