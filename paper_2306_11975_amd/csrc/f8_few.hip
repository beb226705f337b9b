// R = P Q^T for codes in 8-bit floating point, few rows of P to an expert: one token and up, straight from memory (gfx950).
//
// Bound: the bytes of Q. A wavefront takes 16 rows of P and 16 of Q (COLS: once or twice) at a time; a lane reads 16 bytes of a row of either and
// the 16 that lie 64 further on, so that 16 rows of 128 bytes, a slab, come by whole lines. Tokens that are not codes yet are cut on the way, each
// wavefront for itself: a lane's 32 values of a slab and those of the three other lanes of its row are a run of 128. That saves a launch and a way
// through memory (one token of bf16 through 2048 x 2048: 5.1 us; cut before, 6.9).
// The matrix cores' 8-bit instruction cuts products beside larger ones (f8_product.h); here, where the bytes are what takes time, the codes become
// fp16, which holds each of them, and the sums of a slab's 128 products are 32-bit ones. They are scaled and added slab by slab. Up
// to sixteen wavefronts share the inner dimension, a slab at a time, so that every SIMD has some, and add up in order at the end.
#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kMostWaves = 16;

// A lane's 32 positions of a slab: codes, and the byte of the run's scale.
template <int TYPE>
struct Slab {   // as they lie
    Eight<TYPE> raw[4];
};
template <>
struct Slab<OZIMMU_E4M3> {
    v4u raw[2];
};
template <int TYPE>
__device__ __forceinline__ void load_slab(const void* row, int64_t at, int64_t k, Slab<TYPE>& x) {
    if constexpr (TYPE == OZIMMU_E4M3) {
        x.raw[0] = *reinterpret_cast<const v4u*>(static_cast<const uint8_t*>(row) + at);
        x.raw[1] = *reinterpret_cast<const v4u*>(static_cast<const uint8_t*>(row) + at + 64);
    } else {
        typedef typename Elem<TYPE>::raw raw;
#pragma unroll
        for (int e = 0; e < 4; ++e) load8<TYPE>(static_cast<const raw*>(row), at + (e & 1) * 8 + (e >> 1) * 64, k, x.raw[e]);
    }
}
template <int TYPE>
__device__ __forceinline__ void cut_slab(const Slab<TYPE>& x, v4u (&codes)[2], int& byte) {
    if constexpr (TYPE == OZIMMU_E4M3) {
        codes[0] = x.raw[0];
        codes[1] = x.raw[1];
    } else {
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, top8<TYPE>(x.raw[e]));
        const auto a = __builtin_amdgcn_permlane32_swap(top, top, false, false);   // the four lanes of a row
        top = max(a[0], a[1]);
        const auto b = __builtin_amdgcn_permlane16_swap(top, top, false, false);
        byte = scale_byte(max(b[0], b[1]));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const v2u c = code8<TYPE>(x.raw[e], byte);
            codes[e >> 1][(e & 1) * 2] = c[0];
            codes[e >> 1][(e & 1) * 2 + 1] = c[1];
        }
    }
}

template <int TYPE, bool WIDE, int COLS>
__launch_bounds__(kMostWaves * 64)
__global__ void f8_few_kernel(F8Args a, int tiles_n) {
    __shared__ v4f sums[kMostWaves - 1][COLS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int tile = blockIdx.x / tiles_n, col0 = (blockIdx.x % tiles_n) * 16 * COLS;
    int first = 0, count = a.rows, unit = tile, expert = 0;
    if (a.experts) {
        Segment s;
        if (!find_unit(a.offsets, a.experts, a.rows, 16, 1, tile, s)) return;
        first = s.first;
        count = s.count;
        unit = s.unit;
        expert = s.expert;
    }
    const int r = unit * 16 + (lane & 15);
    int64_t row = first + min(r, count - 1);
    bool there = r < count;
    const int64_t out_row = row;
    if (a.source) {
        const int s = a.source[row];
        const bool in = (unsigned)s < (unsigned)a.t;
        row = in ? s : 0;
        there = there && in;
    }
    const int piece = (lane >> 4) * 16;
    const char* p = static_cast<const char*>(a.V) + row * a.ldv * (int)(TYPE == OZIMMU_E4M3 ? 1 : TYPE == OZIMMU_F32 ? 4 : 2);
    const uint8_t* sp = a.sp + row * a.ldsp;
    const uint8_t* q[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) q[c] = a.Q + ((int64_t)expert * a.n + min(col0 + 16 * c + (lane & 15), a.n - 1)) * a.ldq + piece;
    const int64_t sq = ((int64_t)expert * ((a.n + 127) >> 7) + (col0 >> 7)) * a.ldsq;
    v4f acc[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int slab = wave; slab < a.slabs; slab += waves) {
        const int64_t at = (int64_t)slab * 128;
        v4u y[COLS][2];
        Slab<TYPE> x;
        int e_x = 0, byte;
        float m;
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            y[c][0] = *reinterpret_cast<const v4u*>(q[c] + at);
            y[c][1] = *reinterpret_cast<const v4u*>(q[c] + at + 64);
        }
        load_slab<TYPE>(p, at + piece, a.k, x);
        if constexpr (TYPE == OZIMMU_E4M3) e_x = sp[slab];
        scale_parts<WIDE>(a.sq, sq + slab, m, byte);
        if (TYPE == OZIMMU_E4M3 && e_x == 255) m = __builtin_nanf("");
        v4u codes[2];
        cut_slab<TYPE>(x, codes, e_x);
        v8h h[4];
        halves16(codes[0], h[0], h[1]);
        halves16(codes[1], h[2], h[3]);
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            v4f part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                v8h y0, y1;
                halves16(y[c][g], y0, y1);
                part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y0, h[2 * g], part, 0, 0, 0);
                part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y1, h[2 * g + 1], part, 0, 0, 0);
            }
            // (a lane's sums are of row lane % 16 of P, whose scale it has)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c][i] += __builtin_amdgcn_ldexpf(part[i] * m, e_x + byte - 254);
        }
    }
    if (wave)
#pragma unroll
        for (int c = 0; c < COLS; ++c) sums[wave - 1][c][lane] = acc[c];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        for (int w = 1; w < waves; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c][i] += sums[w - 1][c][lane][i];
        const int col = col0 + 16 * c + (lane >> 4) * 4;
        if (r < count && col < a.n) store_four(a, out_row, col, acc[c], there);
    }
}

template <int TYPE, int COLS>
hipError_t launch(const F8Args& a, int64_t tiles, hipStream_t st) {
    const int64_t tiles_n = (a.n + 16 * COLS - 1) / (16 * COLS), grid = tiles * tiles_n;
    if (grid <= 0 || grid > INT32_MAX) return hipErrorInvalidConfiguration;
    const int waves = a.slabs < 1 ? 1 : a.slabs < kMostWaves ? a.slabs : kMostWaves;
    auto kernel = a.scale_type == OZIMMU_F32 ? f8_few_kernel<TYPE, true, COLS> : f8_few_kernel<TYPE, false, COLS>;
    kernel<<<dim3((unsigned)grid), dim3(waves * 64), 0, st>>>(a, (int)tiles_n);
    return hipGetLastError();
}
// Two tiles of columns to a wavefront, where that leaves every compute unit a workgroup: the tokens are cut half as often. bf16, one row, us, one tile
// of columns or two: 8192 x 4096 11.7, 9.7; 8192 x 2048 6.7, 6.5.
template <int TYPE>
hipError_t launch_by_columns(const F8Args& a, hipStream_t st) {
    const int64_t tiles = a.experts ? a.rows / 16 + (a.experts < a.rows ? a.experts : a.rows) : ((int64_t)a.rows + 15) / 16;
    return ((int64_t)a.n + 31) / 32 * tiles >= kComputeUnits ? launch<TYPE, 2>(a, tiles, st) : launch<TYPE, 1>(a, tiles, st);
}

}  // namespace

hipError_t launch_f8_few(const F8Args& a, hipStream_t st) {
    switch (a.v_type) {
        case OZIMMU_F32: return launch_by_columns<OZIMMU_F32>(a, st);
        case OZIMMU_BF16: return launch_by_columns<OZIMMU_BF16>(a, st);
        case OZIMMU_F16: return launch_by_columns<OZIMMU_F16>(a, st);
        default: return launch_by_columns<OZIMMU_E4M3>(a, st);
    }
}

}  // namespace ozimmu
