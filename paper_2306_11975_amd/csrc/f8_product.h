// R = P Q^T for codes in 8-bit floating point, tile by tile (gfx950). Rows of both operands run along the inner dimension, in slabs of 128
// positions (128 bytes) that have one scale each.
//
// A workgroup owns a BM x BN tile. Slabs come into LDS by direct loads, swizzled and double-buffered as in nt_product.h (16-byte piece c of row
// r lies at place c ^ (r % 8)); a lane's fragment of a slab is pieces lane / 16 and lane / 16 + 4 of row lane % 16, of either operand alike, so
// that positions meet. Two ways of multiplying:
//   16-bit results: v_mfma_scale_f32_16x16x128_f8f6f4, which takes a power-of-two scale for every row and 32 positions: a slab is one
//     instruction and its scales cost nothing. It cuts each product toward zero to a multiple of 2^(E - 13), E the largest sum of two codes' exponents
//     among eight neighbouring products (those of zeros apart; subnormal codes count with -6), and adds the eights up in 32 bits: measured, on every
//     one of 2 10^5 random eights. For normally distributed values that is 2^-19 of the sum of magnitudes, 2^-10.2 of it at worst, 2^-7.2 beside
//     subnormal codes. It is taken for 16-bit results alone, of values whose own rounding to codes lost up to 2^-4 of each, for two and a half times
//     the speed; 32-bit results are the way to exact products.
//   32-bit results (EXACT): the codes become fp16, which holds each of them, four MFMAs a slab, at half the rate; a slab's sum is scaled and
//     added to the tile's on the vector units.
// Scales of the weights in 32 bits (WIDE): their exponents go the way of the bytes, their significands are multiplied on the vector units.
// A lane's scales of four slabs are one word. Bound: the way of the operands through LDS and, where tiles are few, latency. us, 16-bit results, tiles
// of 128, 64 x 128, 64: 2048 x 2048 x 8192 53, 47, 59; 2048 x 4096 x 4096 42, 53, 62; 32-bit results 4096 x 8192 x 4096 309 with the cut.
//
// Over experts the tiles are counted on the GPU from the offsets: every wavefront scans them once. The launch is as large as they could make
// it; what is left over ends at once.
#pragma once

#include <algorithm>

#include "f8_common.h"

namespace ozimmu {
namespace {

// How the tiles are dealt: the first `whole` to a workgroup each, the others to `parts` each, with part_slabs (a multiple of four) slabs.
struct F8Plan {
    int tiles_m, tiles_n, whole, parts, part_slabs;
};

// A workgroup's items: tiles, and parts of those that are shared. Every XCD has a contiguous run of them (tile_of_block).
struct F8Tile {
    int expert, first, count, row0, col0;   // rows first .. first + count are the expert's; row0 from there on
    int slab0, slabs, before;               // `before`: slab from which the expert's runs begin (along_rows)
    int shared;                             // number among the shared parts, or -1
};
template <int BM>
__device__ __forceinline__ int f8_items(const F8Args& a, const F8Plan& p) {
    const int tiles = p.tiles_m * p.tiles_n;
    if (a.along_rows && a.experts) return a.experts * tiles;
    if (a.experts) return count_units(a.offsets, a.experts, a.rows, BM) * p.tiles_n;
    return p.whole + (tiles - p.whole) * p.parts;
}
template <int BM, int BN>
__device__ __forceinline__ F8Tile f8_tile(const F8Args& a, const F8Plan& p, int items, int item) {
    F8Tile t;
    t.expert = t.first = t.before = t.slab0 = 0;
    t.count = a.rows;
    t.slabs = a.slabs;
    t.shared = -1;
    int tm, tn;
    if (a.along_rows && a.experts) {
        const int one = p.tiles_m * p.tiles_n;
        t.expert = item / one;
        tile_of_logical(item - t.expert * one, p.tiles_m, p.tiles_n, tm, tn);
        over_experts(a.offsets, a.experts, a.t, 128, 4, [&](int e, int, int count, int, int before) {
            const unsigned long long here = __builtin_amdgcn_ballot_w64(e == t.expert);
            if (!here) return;
            t.slabs = (__builtin_amdgcn_readlane(count, __builtin_ctzll(here)) + 127) >> 7;
            t.before = __builtin_amdgcn_readlane(before, __builtin_ctzll(here));
        });
    } else if (a.experts) {
        tile_of_logical(item, items / p.tiles_n, p.tiles_n, tm, tn);
        Segment s{};
        find_unit(a.offsets, a.experts, a.rows, BM, 1, tm, s);
        t.expert = s.expert;
        t.first = s.first;
        t.count = s.count;
        tm = s.unit;
    } else {
        int tile = item;
        if (item >= p.whole) {
            t.shared = item - p.whole;
            tile = p.whole + t.shared / p.parts;
            t.slab0 = t.shared % p.parts * p.part_slabs;
            t.slabs = min(p.part_slabs, a.slabs - t.slab0);
        }
        tile_of_logical(tile, p.tiles_m, p.tiles_n, tm, tn);
    }
    t.row0 = tm * BM;
    t.col0 = tn * BN;
    return t;
}

template <int BM, int BN, int WM, int WN, bool EXACT, bool WIDE, bool Q_ROWS>
__launch_bounds__(WM * WN * 64)
__global__ void f8_product_kernel(F8Args a, F8Plan plan) {
    static_assert(!(WIDE && Q_ROWS) && BN / WN <= 128);
    constexpr int W = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LP = BM / 8 / W, LQ = BN / 8 / W;   // direct loads per wavefront and slab
    constexpr unsigned kStage = (BM + BN) * 128;
    constexpr int SQ = Q_ROWS ? NI : 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int items = f8_items<BM>(a, plan);
    int item, mine;
    xcd_tile_range(blockIdx.x & 7, items, item, mine);
    if ((int)(blockIdx.x >> 3) >= mine) return;
    const F8Tile t = f8_tile<BM, BN>(a, plan, items, item + (blockIdx.x >> 3));
    const int slabs = t.slabs;

    // operands: P's rows from `first` on (or by source), Q's from the expert's first
    const int64_t p_row = a.along_rows ? t.row0 : a.source ? 0 : (int64_t)t.first + t.row0;
    const int64_t q_row = a.along_rows ? t.col0 : (int64_t)t.expert * a.n + t.col0;
    const int64_t slab_first = t.before + t.slab0;
    const uint8_t* P = a.P + p_row * a.ldp + slab_first * 128;
    const uint8_t* Q = a.Q + q_row * a.ldq + slab_first * 128;
    auto row_of = [&](int r) {   // row of P, from p_row, of row r of the tile
        r = min(r, t.count - 1 - t.row0);
        if (!a.source || a.along_rows) return r;
        const int s = a.source[t.first + t.row0 + r];
        return (unsigned)s < (unsigned)a.t ? s : 0;
    };
    const unsigned piece = ((lane & 7) ^ (lane >> 3)) * 16;
    unsigned voff_p[LP], voff_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) voff_p[i] = (unsigned)row_of((wave * LP + i) * 8 + (lane >> 3)) * (unsigned)a.ldp + piece;
#pragma unroll
    for (int i = 0; i < LQ; ++i) voff_q[i] = (unsigned)min((wave * LQ + i) * 8 + (lane >> 3), a.n - 1 - t.col0) * (unsigned)a.ldq + piece;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
    auto load = [&](int i, int slab, int stage) {
        const unsigned at = lds0 + stage * kStage;
        if (i < LP)
            dma_load16<0>(P + (int64_t)slab * 128, voff_p[i], at + (wave * LP + i) * 1024);
        else
            dma_load16<0>(Q + (int64_t)slab * 128, voff_q[i - LP], at + BM * 128 + (wave * LQ + i - LP) * 1024);
    };

    const int wm = wave / WN, wn = wave % WN;
    const unsigned frag0 = (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) * 16);
    const unsigned frag1 = (lane & 15) * 128 + ((((lane >> 4) + 4) ^ (lane & 7)) * 16);

    // scales: words of four slabs
    const uint8_t* SP = a.sp + p_row * a.ldsp + slab_first;
    unsigned voff_sp[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) voff_sp[i] = (unsigned)row_of(wm * (BM / WM) + 16 * i + (lane & 15)) * (unsigned)a.ldsp;
    const uint8_t* SQB = nullptr;
    const float* SQF = nullptr;
    unsigned voff_sq[SQ] = {};
    if constexpr (Q_ROWS) {
        SQB = static_cast<const uint8_t*>(a.sq) + q_row * a.ldsq + slab_first;
#pragma unroll
        for (int j = 0; j < NI; ++j) voff_sq[j] = (unsigned)min(wn * (BN / WN) + 16 * j + (lane & 15), a.n - 1 - t.col0) * (unsigned)a.ldsq;
    } else {
        const int64_t at = ((int64_t)t.expert * ((a.n + 127) >> 7) + min((t.col0 + wn * (BN / WN)) >> 7, (a.n - 1) >> 7)) * a.ldsq + slab_first;
        if constexpr (WIDE)
            SQF = static_cast<const float*>(a.sq) + at;
        else
            SQB = static_cast<const uint8_t*>(a.sq) + at;
    }
    // The words of the next four slabs are asked for a slab ahead, with the direct loads, whose wait they share.
    unsigned sp[MI], sq[SQ], sp_next[MI], sq_next[WIDE ? 4 : SQ];
    float sig = 1.0f;
    auto request_scales = [&](int slab) {
#pragma unroll
        for (int i = 0; i < MI; ++i) sp_next[i] = *reinterpret_cast<const unsigned*>(SP + slab + voff_sp[i]);
        if constexpr (WIDE) {
#pragma unroll
            for (int s = 0; s < 4; ++s) sq_next[s] = __float_as_uint(SQF[min(slab + s, slabs - 1)]);
        } else {
#pragma unroll
            for (int j = 0; j < SQ; ++j) sq_next[j] = *reinterpret_cast<const unsigned*>(SQB + slab + voff_sq[j]);
        }
    };
    auto next_scales = [&]() {
#pragma unroll
        for (int i = 0; i < MI; ++i) sp[i] = sp_next[i];
        if constexpr (!WIDE)
#pragma unroll
            for (int j = 0; j < SQ; ++j) sq[j] = sq_next[j];
    };
    auto scales = [&](int slab) {   // those of `slab` in the low bytes
        if ((slab & 3) == 0) {
            next_scales();
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i) sp[i] >>= 8;
            if constexpr (!WIDE)
#pragma unroll
                for (int j = 0; j < SQ; ++j) sq[j] >>= 8;
        }
        if constexpr (WIDE) {
            int byte;
            const unsigned w = (slab & 2) ? (slab & 1) ? sq_next[3] : sq_next[2] : (slab & 1) ? sq_next[1] : sq_next[0];
            scale_parts(w, sig, byte);
            sq[0] = (unsigned)byte;
        }
        if ((slab & 3) == 3 && slab + 1 < slabs) request_scales(slab + 1);
    };

    v4f acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

    struct Operand {
        v4u a, b;
    };
    auto read = [&](Operand& x, const unsigned char* at) {
        x.a = *reinterpret_cast<const v4u*>(at + frag0);
        x.b = *reinterpret_cast<const v4u*>(at + frag1);
    };
    auto both = [](const Operand& x) { return v8i{(int)x.a[0], (int)x.a[1], (int)x.a[2], (int)x.a[3], (int)x.b[0], (int)x.b[1], (int)x.b[2], (int)x.b[3]}; };
    auto row_of_products = [&](int i, const Operand& p, const Operand (&q)[NI]) {
        if constexpr (EXACT) {
            v8h ph[4];
            halves16(p.a, ph[0], ph[1]);
            halves16(p.b, ph[2], ph[3]);
            // (a byte of 255 is a NaN: the sums of two others end at 254; columns that were cut here have none)
            const int sp_now = (int)(sp[i] & 255u), e_p = Q_ROWS || sp_now < 255 ? sp_now : 512;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                v8h qh[4];
                halves16(q[j].a, qh[0], qh[1]);
                halves16(q[j].b, qh[2], qh[3]);
                v4f part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 4; ++h) part = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh[h], ph[h], part, 0, 0, 0);
                // (a word of Q_ROWS is the lane's own row of Q; the sums are of its columns 4 (lane / 16) + 0 .. 3)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int byte = (int)((Q_ROWS ? (unsigned)__shfl((int)sq[j], (lane >> 4) * 4 + e) : sq[0]) & 255u);
                    float x = part[e];
                    if constexpr (WIDE) x *= sig;
                    const int exponent = e_p + (Q_ROWS || byte < 255 ? byte : 512) - 254;
                    x = __builtin_amdgcn_ldexpf(x, exponent);
                    acc[i][j][e] += !Q_ROWS && exponent > 254 ? __builtin_nanf("") : x;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if constexpr (WIDE) {
                    const v4f part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(q[j]), both(p), v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, (int)sq[0], 0, (int)sp[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[e], sig, acc[i][j][e]);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(q[j]), both(p), acc[i][j], 0, 0, 0, (int)sq[Q_ROWS ? j : 0], 0, (int)sp[i]);
                }
            }
        }
    };

    if (slabs > 0) {
#pragma unroll
        for (int l = 0; l < LP + LQ; ++l) load(l, 0, 0);
        request_scales(0);
        for (int slab = 0; slab < slabs; ++slab) {
            // the slab has landed and this wavefront's reads of the other stage are done; behind the barrier, everyone's
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int stage = slab & 1;
            scales(slab);
            if (slab + 1 < slabs)
#pragma unroll
                for (int l = 0; l < LP + LQ; ++l) load(l, slab + 1, stage ^ 1);
            const unsigned char* at_p = lds + stage * kStage + wm * (BM / WM) * 128;
            const unsigned char* at_q = lds + stage * kStage + BM * 128 + wn * (BN / WN) * 128;
            Operand q[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) read(q[j], at_q + j * 2048);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                Operand p;
                read(p, at_p + i * 2048);
                row_of_products(i, p, q);
            }
        }
    }
    // The compiler may move the last MFMAs down to where their results are stored, under a condition that lanes differ in; the instruction
    // takes its operands from all lanes. So the sums are complete here.
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) asm volatile("" : "+a"(acc[i][j]));

    // ---- results: lane holds R[row][col .. col + 3]
    if (t.shared >= 0) {
        v4f* to = reinterpret_cast<v4f*>(a.partial) + (int64_t)t.shared * (MI * NI * W * 64) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) to[(i * NI + j) * (W * 64)] = acc[i][j];
        return;
    }
    const int64_t first_row = a.along_rows ? (int64_t)t.expert * a.rows : (int64_t)t.first;
    auto has_source = [&](int r) { return !a.source || a.along_rows || (unsigned)a.source[t.first + min(r, t.count - 1)] < (unsigned)a.t; };
    if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int r = t.row0 + wm * (BM / WM) + 16 * i + (lane & 15);
            const bool there = has_source(r);
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int c = t.col0 + wn * (BN / WN) + 16 * j + (lane >> 4) * 4;
                if (r < t.count && c < a.n) store_four(a, first_row + r, c, acc[i][j], there);
            }
        }
    } else {   // 16 bits: by way of LDS, so that stores are of whole lines (gradients of 8192 x 4096 weights from one token 34 -> 29 us)
        constexpr unsigned kPitch = BN * 2 + 16;
        static_assert(BM * kPitch <= 2 * kStage);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // everyone's reads of the last slab are done
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int r = wm * (BM / WM) + 16 * i + (lane & 15);
            const bool there = has_source(t.row0 + r);
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const v4f& x = acc[i][j];
                v2u y;
                if (a.out_type == OZIMMU_BF16)
                    y = v2u{two_as<OZIMMU_BF16>(x[0], x[1]), two_as<OZIMMU_BF16>(x[2], x[3])};
                else
                    y = v2u{two_as<OZIMMU_F16>(x[0], x[1]), two_as<OZIMMU_F16>(x[2], x[3])};
                *reinterpret_cast<v2u*>(lds + r * kPitch + (wn * (BN / WN) + 16 * j + (lane >> 4) * 4) * 2) = there ? y : v2u{0, 0};
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int i = 0; i < BM * BN / 8 / (W * 64); ++i) {
            const int piece = i * (W * 64) + threadIdx.x, r = piece / (BN / 8), c = piece % (BN / 8) * 8;
            if (t.row0 + r >= t.count || t.col0 + c >= a.n) continue;
            const unsigned char* from = lds + r * kPitch + c * 2;
            unsigned short* to = static_cast<unsigned short*>(a.out) + (first_row + t.row0 + r) * a.ldo + t.col0 + c;
            if (t.col0 + c + 8 <= a.n)
                *reinterpret_cast<v4u_any*>(to) = *reinterpret_cast<const v4u*>(from);
            else
                for (int e = 0; t.col0 + c + e < a.n; ++e) to[e] = reinterpret_cast<const unsigned short*>(from)[e];
        }
    }
}

// The shared tiles: parts added up in order, a workgroup for a 16 x 16 result of each wavefront.
template <int BM, int BN, int WM, int WN>
__launch_bounds__(WM * WN * 64)
__global__ void f8_join_kernel(F8Args a, F8Plan plan) {
    constexpr int W = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
    const int i = blockIdx.y / NI, j = blockIdx.y % NI;
    int tm, tn;
    tile_of_logical(plan.whole + blockIdx.x, plan.tiles_m, plan.tiles_n, tm, tn);
    const v4f* from = reinterpret_cast<const v4f*>(a.partial) + ((int64_t)blockIdx.x * plan.parts * (MI * NI) + blockIdx.y) * (W * 64) + threadIdx.x;
    v4f sum = from[0];
    for (int p = 1; p < plan.parts; ++p) {
        const v4f x = from[(int64_t)p * (MI * NI * W * 64)];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    const int r = tm * BM + wm * (BM / WM) + (lane & 15) + 16 * i, c = tn * BN + wn * (BN / WN) + (lane >> 4) * 4 + 16 * j;
    if (r < a.rows && c < a.n) store_four(a, r, c, sum, true);
}

// Items of a product, at most (over experts the offsets tell how many), by eights.
template <int BM, int BN>
int64_t f8_most_items(const F8Args& a, F8Plan& plan) {
    plan.tiles_m = (a.rows + BM - 1) / BM;
    plan.tiles_n = (a.n + BN - 1) / BN;
    const int64_t tiles = (int64_t)plan.tiles_m * plan.tiles_n;
    if (a.along_rows && a.experts) return pad_to(tiles * a.experts, 8);
    if (a.experts) return pad_to(tiles + (int64_t)std::min(a.experts, a.rows) * plan.tiles_n, 8);
    return pad_to(plan.whole + (tiles - plan.whole) * plan.parts, 8);
}

template <int BM, int BN, int WM, int WN, bool EXACT, bool WIDE, bool Q_ROWS>
hipError_t launch_f8_shape(const F8Args& a, const F8Plan& plan, int64_t grid, hipStream_t st) {
    constexpr auto kernel = f8_product_kernel<BM, BN, WM, WN, EXACT, WIDE, Q_ROWS>;
    constexpr int bytes = 2 * (BM + BN) * 128;
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
    kernel<<<dim3((unsigned)grid), dim3(WM * WN * 64), bytes, st>>>(a, plan);
    const int rest = a.experts ? 0 : plan.tiles_m * plan.tiles_n - plan.whole;
    if (rest) f8_join_kernel<BM, BN, WM, WN><<<dim3((unsigned)rest, BM / WM / 16 * (BN / WN / 16)), dim3(WM * WN * 64), 0, st>>>(a, plan);
    return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, bool EXACT>
hipError_t launch_f8_tile(const F8Args& a, F8Plan plan, hipStream_t st) {
    const int64_t grid = f8_most_items<BM, BN>(a, plan);
    if (grid <= 0 || grid > INT32_MAX) return hipErrorInvalidConfiguration;
    if (a.along_rows) return launch_f8_shape<BM, BN, WM, WN, EXACT, false, true>(a, plan, grid, st);
    if (a.scale_type == OZIMMU_F32) return launch_f8_shape<BM, BN, WM, WN, EXACT, true, false>(a, plan, grid, st);
    return launch_f8_shape<BM, BN, WM, WN, EXACT, false, false>(a, plan, grid, st);
}

}  // namespace
}  // namespace ozimmu
