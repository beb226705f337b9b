// C = P Q^T on the 16-bit matrix cores (v_mfma_f32_16x16x32, sums in 32 bits), for operands whose rows run along the inner
// dimension in slabs of 128 bytes (weights_internal.h). One slice: the ordinary product. Two slices of fp16 (value = first +
// second, 22 bits and more): the products first*first, first*second and second*first of the same fragments, which leaves out
// what is below 2^-22 of a term; a slab then holds both slices of 32 positions, so loads and shared memory are the same and only
// the pairs differ.
//
// A workgroup owns a BM x BN tile. A slab of its rows of P and Q is brought into LDS by direct loads (1 KiB = 8 rows a
// wavefront and load; the lane that fetches 16-byte piece c of row r puts it at place c ^ (r % 8), so that the 16 lanes of a
// fragment read, ds_read_b128, meet all banks), STAGES - 1 slabs ahead of the one that is multiplied: one barrier per slab. Rows
// beyond the last are read from the last one and their results dropped.
// The fragments of Q are the MFMA's first operand: a lane then holds four consecutive columns of one row of C.
#pragma once

#include "half_common.h"

namespace ozimmu {
namespace {

template <int BM, int BN, int WM, int WN, int STAGES, bool PIPE, int SLICES, bool BF16, int RESULT>
__launch_bounds__(WM * WN * 64)
__global__ void nt_product_kernel(NtArgs a, int tiles_m, int tiles_n) {
    constexpr int W = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LP = BM / 8 / W, LQ = BN / 8 / W;   // direct loads per wavefront and slab
    constexpr unsigned kStage = (BM + BN) * 128;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tm, tn;
    if (a.symmetric) {   // tiles on and above the diagonal, row by row of tiles
        int first, count;
        xcd_tile_range(blockIdx.x & 7, tiles_m * (tiles_m + 1) / 2, first, count);
        int left = first + (blockIdx.x >> 3);
        for (tm = 0; left >= tiles_m - tm; ++tm) left -= tiles_m - tm;
        tn = tm + left;
    } else {
        tile_of_block(blockIdx.x, tiles_m, tiles_n, tm, tn);
    }
    const int64_t z = blockIdx.y;
    const int row0 = tm * BM, col0 = tn * BN;
    const unsigned char* P = reinterpret_cast<const unsigned char*>(a.P + z * a.batch_p + (int64_t)row0 * a.ldp);
    const unsigned char* Q = reinterpret_cast<const unsigned char*>(a.Q + z * a.batch_q + (int64_t)col0 * a.ldq);
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
    constexpr int AHEAD = PIPE ? STAGES : STAGES - 1;   // slabs requested before the first is multiplied
    for (int i = 0; i < AHEAD; ++i)
        if (i < a.slabs)
#pragma unroll
            for (int l = 0; l < LP + LQ; ++l) load(l, i, i);
    if constexpr (PIPE) {
        // The fragments of the next slab are read from LDS while this one's are multiplied; a slab's stage is requested anew as soon as its fragments are in registers.
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
        if (AHEAD <= a.slabs)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * (LP + LQ)) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read(f[0], 0);
        int stage = 0;
        auto step = [&](int slab, Frags& now, Frags& next) {
            // the next slab has landed and this one's fragments are in registers; behind the barrier, everyone's
            if (slab + STAGES <= a.slabs)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * (LP + LQ)) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int free = stage;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (slab + 1 < a.slabs) read(next, stage);
            const bool more = slab + STAGES < a.slabs;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (more)
#pragma unroll
                    for (int l = (LP + LQ) * i / MI; l < (LP + LQ) * (i + 1) / MI; ++l) load(l, slab + STAGES, free);
                row_of_products(i, now.p0[i], now.p1[i], now.q0, now.q1);
            }
        };
        int slab = 0;
        for (; slab + 1 < a.slabs; slab += 2) {
            step(slab, f[0], f[1]);
            step(slab + 1, f[1], f[0]);
        }
        if (slab < a.slabs) step(slab, f[0], f[1]);
    } else {
        int stage = 0;
        for (int slab = 0; slab < a.slabs; ++slab) {
            // this wavefront's loads of the slab have landed (later ones may be on their way) and its reads of the stage that is loaded next are done;
            // behind the barrier, everyone's
            if (slab + AHEAD <= a.slabs)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * (LP + LQ)) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int to = stage == 0 ? AHEAD : stage - 1;
            const unsigned char* at_p = lds + stage * kStage + wm * (BM / WM) * 128;
            const unsigned char* at_q = lds + stage * kStage + BM * 128 + wn * (BN / WN) * 128;
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (slab + AHEAD < a.slabs)
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
    const int r0 = row0 + wm * (BM / WM) + (lane & 15), c0 = col0 + wn * (BN / WN) + (lane >> 4) * 4;
    if constexpr (RESULT == kOutSlices) {
        unsigned short* C = a.C + z * a.batch_c;
        const unsigned short* in = a.in ? a.in + z * a.batch_c : nullptr;
        unsigned short* CT = a.CT ? a.CT + z * a.batch_ct : nullptr;
        const int m_pad = (a.m + 31) & ~31, n_pad = (a.n + 31) & ~31;
        const bool mirror = CT && !(a.symmetric && tm == tn);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = r0 + 16 * i, c = c0 + 16 * j;
                if (c >= n_pad || r >= m_pad) continue;
                const int64_t at = (int64_t)r * a.ldc + (c >> 5) * 64 + (c & 31);
                float v[4];
                unsigned short h[4], l[4];
                unsigned short ih[4] = {}, il[4] = {};
                if (in && r < a.m) {
                    *reinterpret_cast<v2u*>(ih) = *reinterpret_cast<const v2u*>(in + at);
                    *reinterpret_cast<v2u*>(il) = *reinterpret_cast<const v2u*>(in + at + 32);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = a.factor * acc[i][j][e];
                    if (in) v[e] = fmaf(a.beta, f16_to_f32(ih[e]) + f16_to_f32(il[e]), v[e]);
                    if (r == c + e) v[e] += a.diagonal;
                    if (c + e >= a.n || r >= a.m) v[e] = 0.f;   // the padding of a row holds zeros
                    two_slices(v[e], h[e], l[e]);
                }
                if (r < a.m) {
                    *reinterpret_cast<v2u*>(C + at) = *reinterpret_cast<v2u*>(h);
                    *reinterpret_cast<v2u*>(C + at + 32) = *reinterpret_cast<v2u*>(l);
                }
                if (mirror) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (c + e >= a.n) continue;
                        const int64_t t = (int64_t)(c + e) * a.ldct + (r >> 5) * 64 + (r & 31);
                        CT[t] = h[e];
                        CT[t + 32] = l[e];
                    }
                }
            }
    } else {
        typedef Elem<RESULT == kOutF32 ? OZIMMU_F32 : RESULT == kOutBf16 ? OZIMMU_BF16 : OZIMMU_F16> E;
        typedef typename E::raw raw;
        typedef raw raw4 __attribute__((ext_vector_type(4)));
        raw* out = reinterpret_cast<raw*>(a.out) + z * a.batch_o;
        const bool wide = (a.ldo & 3) == 0 && (a.batch_o & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & (4 * sizeof(raw) - 1)) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int r = r0 + 16 * i;
            if (r >= a.m) continue;
            const int ep = a.exp_p ? a.exp_p[r] : 0;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int c = c0 + 16 * j;
                if (c >= a.n) continue;
                raw4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = a.factor * acc[i][j][e];
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
    }
}

template <int BM, int BN, int WM, int WN, int STAGES, bool PIPE, int SLICES, bool BF16, int RESULT>
hipError_t launch_nt_tile(const NtArgs& a, hipStream_t st) {
    constexpr auto kernel = nt_product_kernel<BM, BN, WM, WN, STAGES, PIPE, SLICES, BF16, RESULT>;
    constexpr int bytes = STAGES * (BM + BN) * 128;
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
    if (a.m <= 0 || a.n <= 0 || a.slabs <= 0 || (a.symmetric && (BM != BN || a.m != a.n))) return hipErrorInvalidValue;
    const int tiles_m = (a.m + BM - 1) / BM, tiles_n = (a.n + BN - 1) / BN;
    const int64_t tiles = a.symmetric ? (int64_t)tiles_m * (tiles_m + 1) / 2 : (int64_t)tiles_m * tiles_n;
    if (tiles > INT32_MAX || a.batch > 65535) return hipErrorInvalidConfiguration;
    kernel<<<dim3((unsigned)tiles, a.batch), dim3(WM * WN * 64), bytes, st>>>(a, tiles_m, tiles_n);
    return hipGetLastError();
}

template <int SLICES, bool BF16, int RESULT>
hipError_t launch_nt(const NtArgs& a, hipStream_t st) {
    auto tiles = [&](int64_t b) {
        const int64_t x = (a.m + b - 1) / b, y = (a.n + b - 1) / b;
        return (a.symmetric ? x * (x + 1) / 2 : x * y) * a.batch;
    };
    // A larger tile moves fewer bytes through LDS per product, a smaller one keeps more compute units busy. Measured, two slices, us: 4096^3 on tiles of 256, 128, 64
    // 309, 336, 412; 2048 x 4096 x 4096 (128, 512, 2048 tiles) 247, 167, 206; 1024 x 1024 x 4096 (16, 64, 256) 250, 86, 42. One slice: 1024 x 4096 x 4096
    // (64, 256, 1024 tiles) 98, 44, 47.
    if (tiles(256) >= 200) return launch_nt_tile<256, 256, 2, 4, 2, false, SLICES, BF16, RESULT>(a, st);
    if (tiles(128) >= 256) return launch_nt_tile<128, 128, 2, 2, 2, false, SLICES, BF16, RESULT>(a, st);
    // With about one workgroup to a compute unit nothing else hides a wavefront's LDS reads: they run a slab ahead (1024 x 1024 x 4096 56 -> 42, 6 x 520 x 520 x 1024 21.1 -> 17.6).
    // With more, their registers and LDS cost the co-residents that do (2048 x 2048 x 8192, 528 tiles, 131 against 162).
    if (tiles(64) <= 320) return launch_nt_tile<64, 64, 2, 2, 3, true, SLICES, BF16, RESULT>(a, st);
    return launch_nt_tile<64, 64, 2, 2, 2, false, SLICES, BF16, RESULT>(a, st);
}

}  // namespace
}  // namespace ozimmu
