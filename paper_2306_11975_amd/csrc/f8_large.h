// R = P Q^T for codes in 8-bit floating point on tiles of 256 x 256 (gfx950): the products of many rows with 16-bit results. What is common
// with the smaller tiles is in f8_product.h.
//
// Bound: the matrix cores, through the clock that the power limit grants, and the way of the operands into LDS. (A register-only loop of their
// instruction reaches 4.1 PFLOP/s on normal values, 4.9 on zeros, 3.7 with LDS reads beside it; the loads alone take 80 us for 4096 x 4096 x 8192.)
// Four wavefronts, one to a SIMD, own 128 x 128 each: a slab then costs LDS 128 KiB of reads and 64 of writes, three quarters of the time that the
// MFMAs take (wavefronts of 128 x 64 would take all of it). The sums fill the accumulation registers, so the MFMAs
// (v_mfma_scale_f32_32x32x64_f8f6f4) are written out with their sums in place.
//
// LDS holds two slabs. A slab's fragments are all read into registers while the slab before is multiplied, each as soon as the fragment whose place
// it takes has had its last MFMA. So early in a slab's 32 MFMAs (slot kFree, behind a barrier) its own place in LDS is free, and the loads of the
// slab after the next go there, one in the shadow of each MFMA; they are waited for in the middle of the next slab (slot kLanded, another barrier),
// 29 MFMAs after the last of them, 45 after the first. (All loads at once were 7 % slower: they stand in each other's way. Waiting at the slab's end
// with one barrier: 4 %.) Past the end the last slab is fetched again, so that all waits are alike. Scales come by direct loads too, a word (four
// slabs) to a row; the loop takes four slabs a round, and the instruction picks the byte. Workgroups stay for as many tiles as there are to each
// compute unit: the next tile's first slabs come while this one's results go. 4096 x 8192 x 4096: 106 us, 2.6 PFLOP/s (a library product of 8-bit
// matrices, without blocks' scales: 110); tile by tile with stores of 8 bytes 130, of 32-byte pieces 111; 128 x 128 tiles 145.
#pragma once

#include "f8_product.h"

namespace ozimmu {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

// acc += the products of 64 positions, the scales taken from byte BYTE of their words; in place. What it needs around it: mfma16_acc.
template <int BYTE>
__device__ __forceinline__ void mfma_scaled(const v8i& a, const v8i& b, v16f& acc, unsigned sa, unsigned sb) {
    if constexpr (BYTE == 0)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
    else if constexpr (BYTE == 1)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
    else if constexpr (BYTE == 2)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0]" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0]" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
__device__ __forceinline__ float sum_read(float a) {
    float v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
    return v;
}
// One word to a lane, as dma_load16.
__device__ __forceinline__ void dma_load4(const void* gbase, unsigned voff, unsigned lds_addr) {
    asm volatile(
        "s_add_u32 m0, %2, 0\n\t"
        "s_nop 4\n\t"
        "global_load_lds_dword %1, %0"
        :
        : "s"(gbase), "v"(voff), "s"(lds_addr)
        : "memory", "scc");
}

constexpr int kLargeTile = 256;
constexpr int kFree = 3, kLanded = 16;   // slots of a slab's 32 MFMAs (see below; 2 to 6 and 16 to 23 were within 4 %)
constexpr unsigned kLargeStage = 2 * kLargeTile * 128, kLargeScales = 2 * kLargeStage, kLargeTurn = kLargeScales + 2 * 2 * kLargeTile * 4;
// Each wavefront's 32 x 64 results on their way to memory; rows of 128 bytes, 16 apart, meet no bank twice.
constexpr unsigned kTurnPitch = 144, kLargeBytes = kLargeTurn + 4 * 32 * kTurnPitch;

template <bool Q_ROWS, int TYPE>
__launch_bounds__(256)
__global__ void f8_large_kernel(F8Args a, F8Plan plan) {
    constexpr int B = kLargeTile, SQN = Q_ROWS ? 4 : 1;
    typedef typename Elem<TYPE>::raw raw;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int items = f8_items<B>(a, plan);
    int first, mine, at_item = blockIdx.x >> 3;
    xcd_tile_range(blockIdx.x & 7, items, first, mine);
    if (at_item >= mine) return;

    F8Tile t;
    int slabs;
    const uint8_t *P, *Q, *SP, *SQ;
    unsigned voff_p[8], voff_q[8], voff_sp, voff_sq;
    // (the lane number is formed anew outside the walk: what comes of it has no registers to wait in, and reloads would wait for loads and stores)
    auto take = [&](int item) {   // a tile's operands
        const int lane = lane_here();
        t = f8_tile<B, B>(a, plan, items, item);
        slabs = t.slabs;
        const int64_t p_row = a.along_rows ? t.row0 : a.source ? 0 : (int64_t)t.first + t.row0;
        const int64_t q_row = a.along_rows ? t.col0 : (int64_t)t.expert * a.n + t.col0;
        const int64_t slab_first = t.before + t.slab0;
        P = a.P + p_row * a.ldp + slab_first * 128;
        Q = a.Q + q_row * a.ldq + slab_first * 128;
        SP = a.sp + p_row * a.ldsp + slab_first;
        SQ = static_cast<const uint8_t*>(a.sq) + (Q_ROWS ? q_row : (int64_t)t.expert * ((a.n + 127) >> 7) + (t.col0 >> 7)) * a.ldsq + slab_first;
        auto row_of = [&](int r) {   // row of P, from p_row, of row r of the tile
            r = min(r, t.count - 1 - t.row0);
            if (!a.source || a.along_rows) return r;
            const int s = a.source[t.first + t.row0 + r];
            return (unsigned)s < (unsigned)a.t ? s : 0;
        };
        auto col_of = [&](int c) { return min(c, a.n - 1 - t.col0); };
        const unsigned piece = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            voff_p[i] = (unsigned)row_of((wave * 8 + i) * 8 + (lane >> 3)) * (unsigned)a.ldp + piece;
            voff_q[i] = (unsigned)col_of((wave * 8 + i) * 8 + (lane >> 3)) * (unsigned)a.ldq + piece;
        }
        // scales: a wavefront fetches the words of 64 rows of P, and of Q's; where Q's have one word for 128 rows, that of each row's
        voff_sp = (unsigned)row_of(wave * 64 + lane) * (unsigned)a.ldsp;
        voff_sq = (unsigned)(Q_ROWS ? col_of(wave * 64 + lane) : col_of(wave * 64 + lane) >> 7) * (unsigned)a.ldsq;
    };
    const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
    auto load = [&](int i, int slab, int to) {   // direct load i of sixteen
        const int64_t at = (int64_t)min(slab, slabs - 1) * 128;
        if (i < 8)
            dma_load16<0>(P + at, voff_p[i], lds0 + to * kLargeStage + (wave * 8 + i) * 1024);
        else
            dma_load16<0>(Q + at, voff_q[i - 8], lds0 + to * kLargeStage + B * 128 + (wave * 8 + i - 8) * 1024);
    };
    auto load_scales = [&](int slab, int to) {
        const int64_t at = min(slab, (slabs - 1) & ~3);
        dma_load4(SP + at, voff_sp, lds0 + kLargeScales + to * 2 * B * 4 + wave * 256);
        dma_load4(SQ + at, voff_sq, lds0 + kLargeScales + to * 2 * B * 4 + B * 4 + wave * 256);
    };
    auto first_loads = [&]() {
        if (slabs == 0) return;
        load_scales(0, 0);
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 16; ++i) load(i, s, s);
    };

    const int wm = wave >> 1, wn = wave & 1;
    const unsigned char* const at_p = lds + (wm * 128 + (lane & 31)) * 128;
    const unsigned char* const at_q = lds + (B + wn * 128 + (lane & 31)) * 128;
    const unsigned char* const at_sp = lds + kLargeScales + (wm * 128 + (lane & 31)) * 4;
    const unsigned char* const at_sq = lds + kLargeScales + B * 4 + (wn * 128 + (lane & 31)) * 4;
    // a lane's fragment of half a slab: pieces lane / 32 and lane / 32 + 2 of its four
    auto fragment = [&](const unsigned char* at, int half) {
        const int c = half * 4 + (lane >> 5);
        return __builtin_shufflevector(*reinterpret_cast<const v4i*>(at + ((c ^ (lane & 7)) * 16)), *reinterpret_cast<const v4i*>(at + (((c + 2) ^ (lane & 7)) * 16)), 0, 1, 2, 3, 4, 5, 6, 7);
    };

    take(first + at_item);
    first_loads();
    for (;;) {
        v16f acc[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        if (slabs > 0) {
            v8i p[2][4], q[2][4];
            unsigned sp[4], sq[SQN];
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    p[h][i] = fragment(at_p + i * 4096, h);
                    q[h][i] = fragment(at_q + i * 4096, h);
                }
                sp[i] = *reinterpret_cast<const unsigned*>(at_sp + i * 128);
                if (i < SQN) sq[i] = *reinterpret_cast<const unsigned*>(at_sq + i * 128);
            }
            for (int slab = 0; slab < slabs; slab += 4) {
                static_for<0, 4>([&](auto number) {
                    constexpr int n = decltype(number)::value, now = n & 1, next = now ^ 1;
                    if (slab + n >= slabs) return;
                    const unsigned char *next_p = at_p + next * kLargeStage, *next_q = at_q + next * kLargeStage;
                    const unsigned round = ((slab >> 2) + 1) & 1;
                    static_for<0, 32>([&](auto place) {
                        constexpr int slot = decltype(place)::value, h = slot / 16, i = slot / 4 % 4, j = slot % 4;
                        if constexpr (slot == kFree) {   // this wavefront's fragments of this slab are in registers; behind the barrier, everyone's
                            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                            if constexpr (n == 1) load_scales(slab + 4, round);
                        }
                        if constexpr (slot == kLanded)   // the next slab has landed; later loads may be on their way
                            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLanded - kFree + (n == 1 ? 2 : 0)) : "memory");
                        mfma_scaled<n>(q[h][j], p[h][i], acc[i][j], sq[Q_ROWS ? j : 0], sp[i]);
                        if constexpr (slot >= kFree && slot < kFree + 16) load(slot - kFree, slab + n + 2, now);
                        if constexpr (slot >= kLanded && slot < kLanded + 4) p[0][slot - kLanded] = fragment(next_p + (slot - kLanded) * 4096, 0);
                        if constexpr (slot >= kLanded + 4 && slot < kLanded + 8) q[0][slot - kLanded - 4] = fragment(next_q + (slot - kLanded - 4) * 4096, 0);
                        if constexpr (h == 1 && j == 3) {
                            p[1][i] = fragment(next_p + i * 4096, 1);
                            if constexpr (n == 3) sp[i] = *reinterpret_cast<const unsigned*>(at_sp + round * 2 * B * 4 + i * 128);
                        }
                        if constexpr (h == 1 && i == 3) {
                            q[1][j] = fragment(next_q + j * 4096, 1);
                            if constexpr (n == 3 && (Q_ROWS || j == 3)) sq[Q_ROWS ? j : 0] = *reinterpret_cast<const unsigned*>(at_sq + round * 2 * B * 4 + (Q_ROWS ? j * 128 : 0));
                        }
                    });
                });
            }
        }
        mfma_results_ready();
        // the next tile's first slabs come while this one's results go: behind the barrier nobody reads LDS, and nothing is on its way to it
        const F8Tile done = t;
        const int lane = lane_here();
        unsigned no_source = 0;   // bit i: row 32 i + lane % 32 of this wavefront's has none (read before other loads and stores are on their way)
        if (a.source && !a.along_rows)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                no_source |= (unsigned)a.source[done.first + min(done.row0 + wm * 128 + 32 * i + (lane & 31), done.count - 1)] >= (unsigned)a.t ? 1u << i : 0u;
        at_item += gridDim.x >> 3;
        const bool more = at_item < mine;
        if (more) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            take(first + at_item);
            first_loads();
        }

        // ---- results: lane holds R[row][col + 8 g + 4 (lane / 32) .. + 3], g = 0 .. 3, of row lane % 32
        // 32 x 64 at a time by way of LDS, so that stores are of whole lines; while a piece is read back the next is rounded.
        unsigned char* const turn = lds + kLargeTurn + wave * (32 * kTurnPitch);
        const int row0 = done.row0 + wm * 128, col0 = done.col0 + wn * 128;
        const bool whole = row0 + 128 <= done.count && col0 + 128 <= a.n;
        raw* const out = static_cast<raw*>(a.out) + ((a.along_rows ? (int64_t)done.expert * a.rows : (int64_t)done.first) + row0) * a.ldo + col0;
        const unsigned lane_out = (unsigned)(lane >> 3) * (unsigned)a.ldo * sizeof(raw) + (lane & 7) * 16;
        v4u piece[4], y[4];
        auto round = [&](auto number) {
            constexpr int i = decltype(number)::value / 2, half = decltype(number)::value % 2;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int g = 0; g < 4; g += 2) {   // the halves of the wavefront exchange: eight columns to a lane
                    unsigned x[2][2];
#pragma unroll
                    for (int f = 0; f < 2; ++f)
#pragma unroll
                        for (int e = 0; e < 2; ++e) x[f][e] = two_as<TYPE>(sum_read(acc[i][2 * half + j][4 * (g + f) + 2 * e]), sum_read(acc[i][2 * half + j][4 * (g + f) + 2 * e + 1]));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const auto z = __builtin_amdgcn_permlane32_swap(x[0][e], x[1][e], false, false);
                        piece[2 * j + g / 2][e] = z[0];
                        piece[2 * j + g / 2][2 + e] = z[1];
                    }
                }
            if (no_source >> i & 1)
#pragma unroll
                for (int x = 0; x < 4; ++x) piece[x] = v4u{0, 0, 0, 0};
        };
        auto by_lds = [&]() {
#pragma unroll
            for (int x = 0; x < 4; ++x) *reinterpret_cast<v4u*>(turn + (lane & 31) * kTurnPitch + (2 * x + (lane >> 5)) * 16) = piece[x];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = *reinterpret_cast<const v4u*>(turn + (q * 8 + (lane >> 3)) * kTurnPitch + (lane & 7) * 16);
        };
        auto store = [&](auto number) {   // eight rows at a time
            constexpr int i = decltype(number)::value / 2, half = decltype(number)::value % 2;
            if (whole) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<v4u_any*>(reinterpret_cast<unsigned char*>(out + (int64_t)(32 * i + 8 * q) * a.ldo + 64 * half) + lane_out) = y[q];
            } else {
#pragma unroll 1
                for (int q = 0; q < 4; ++q) {
                    const int r = 32 * i + q * 8 + (lane >> 3), c = 64 * half + (lane & 7) * 8;
                    const raw* from = reinterpret_cast<const raw*>(turn + (q * 8 + (lane >> 3)) * kTurnPitch + (lane & 7) * 16);
                    if (row0 + r >= done.count) continue;
                    if (col0 + c + 8 <= a.n)
                        *reinterpret_cast<v4u_any*>(out + (int64_t)r * a.ldo + c) = *reinterpret_cast<const v4u*>(from);
                    else
#pragma unroll 1
                        for (int e = 0; e < 8; ++e)
                            if (col0 + c + e < a.n) out[(int64_t)r * a.ldo + c + e] = from[e];
                }
            }
        };
        static_for<0, 8>([&](auto number) {
            round(number);
            __builtin_amdgcn_sched_barrier(0);   // (all sums at once would take as many ordinary registers)
            if constexpr (decltype(number)::value > 0) store(std::integral_constant<int, decltype(number)::value - 1>{});
            by_lds();
            __builtin_amdgcn_sched_barrier(0);
        });
        store(std::integral_constant<int, 7>{});
        if (!more) return;
    }
}

}  // namespace
}  // namespace ozimmu
