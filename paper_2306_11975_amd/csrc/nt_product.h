// C = P Q^T on the 16-bit matrix cores (v_mfma_f32_16x16x32, sums in 32 bits), for operands whose rows run along the inner
// dimension in slabs of 128 bytes (weights_internal.h). One slice: the ordinary product. Two slices of fp16 (value = first +
// second, 22 bits and more): the products first*first, first*second and second*first of the same fragments, which leaves out
// what is below 2^-22 of a term; a slab then holds both slices of 32 positions, so loads and shared memory are the same and only
// the pairs differ.
//
// A workgroup owns a BM x BN tile. A slab of its rows of P and Q is brought into LDS by direct loads (1 KiB = 8 rows a
// wavefront and load; the lane that fetches 16-byte piece c of row r puts it at place c ^ (r % 8), so that the 16 lanes of a
// fragment read, ds_read_b128, meet all banks), a stage ahead of the one that is multiplied: one barrier per slab. Rows
// beyond the last are read from the last one and their results dropped.
// The fragments of Q are the MFMA's first operand: a lane then holds four consecutive columns of one row of C.
#pragma once

#include "half_common.h"

namespace ozimmu {
namespace {

template <int BM, int BN, int WM, int WN, int SLICES, bool BF16, int RESULT>
__launch_bounds__(WM * WN * 64, (BM == 256 ? 2 : 2))
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

    auto load_slab = [&](int slab) {
        const unsigned at = lds0 + (slab & 1) * kStage;
        const unsigned char* p = P + (int64_t)slab * 128;
        const unsigned char* q = Q + (int64_t)slab * 128;
#pragma unroll
        for (int i = 0; i < LP; ++i) dma_load16<0>(p, voff_p[i], at + (wave * LP + i) * 1024);
#pragma unroll
        for (int i = 0; i < LQ; ++i) dma_load16<0>(q, voff_q[i], at + BM * 128 + (wave * LQ + i) * 1024);
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

    load_slab(0);
    for (int slab = 0; slab < a.slabs; ++slab) {
        // this wavefront's loads have landed and its reads of the other stage are done; behind the barrier, everyone's
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (slab + 1 < a.slabs) load_slab(slab + 1);
        const unsigned char* at_p = lds + (slab & 1) * kStage + wm * (BM / WM) * 128;
        const unsigned char* at_q = lds + (slab & 1) * kStage + BM * 128 + wn * (BN / WN) * 128;
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
            if constexpr (SLICES == 1) {
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], p0, acc[i][j]);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q1[j], p1, acc[i][j]);
            } else {
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q1[j], p0, acc[i][j]);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], p1, acc[i][j]);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(q0[j], p0, acc[i][j]);
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

template <int BM, int BN, int WM, int WN, int SLICES, bool BF16, int RESULT>
hipError_t launch_nt_tile(const NtArgs& a, hipStream_t st) {
    constexpr auto kernel = nt_product_kernel<BM, BN, WM, WN, SLICES, BF16, RESULT>;
    constexpr int bytes = 2 * (BM + BN) * 128;
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
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
    if (tiles(256) >= 200) return launch_nt_tile<256, 256, 2, 4, SLICES, BF16, RESULT>(a, st);
    if (tiles(128) >= 256) return launch_nt_tile<128, 128, 2, 2, SLICES, BF16, RESULT>(a, st);
    return launch_nt_tile<64, 64, 2, 2, SLICES, BF16, RESULT>(a, st);
}

}  // namespace
}  // namespace ozimmu
