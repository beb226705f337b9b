// R = P Q^T for codes in 8-bit floating point, few rows of P to an expert: one token and up, straight from memory (gfx950).
//
// Bound: the bytes of Q. A wavefront takes 16 rows of P and 16 of Q (COLS: once or twice) at a time; a lane reads 16 bytes of a row of either and
// the 16 that lie 64 further on, so that 16 rows of 128 bytes, a slab, come by whole lines. Tokens that are not codes yet are cut on the way, each
// wavefront for itself: a lane's 32 values of a slab and those of the three other lanes of its row are a run of 128. That saves a launch and a way
// through memory (one token of bf16 through 2048 x 2048: 5.1 us; cut before, 6.9).
// The matrix cores' 8-bit products drop what is below 2^-13 of the largest of eight; here, where the bytes are what takes time, the codes become
// fp16, which holds each of them, and the sums of a slab's 128 products are 32-bit ones. They are scaled and added slab by slab. Four
// to sixteen wavefronts share the inner dimension and add up in order at the end.
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

template <int TYPE, bool WIDE, int COLS, int DEPTH>
__launch_bounds__((DEPTH == 1 ? kMostWaves : 4) * 64)
__global__ void f8_few_kernel(F8Args a, int tiles_n) {
    __shared__ v4f sums[(DEPTH == 1 ? kMostWaves : 4) - 1][COLS][64];
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
    for (int slab0 = wave * DEPTH; slab0 < a.slabs; slab0 += waves * DEPTH) {
        const int slabs = min(DEPTH, a.slabs - slab0);
        v4u y[DEPTH][COLS][2];
        Slab<TYPE> x[DEPTH];
        unsigned ep[DEPTH] = {};
#pragma unroll
        for (int s = 0; s < DEPTH; ++s)
            if (s < slabs) {
                const int64_t at = (int64_t)(slab0 + s) * 128;
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    y[s][c][0] = *reinterpret_cast<const v4u*>(q[c] + at);
                    y[s][c][1] = *reinterpret_cast<const v4u*>(q[c] + at + 64);
                }
                load_slab<TYPE>(p, at + piece, a.k, x[s]);
                if constexpr (TYPE == OZIMMU_E4M3) ep[s] = sp[slab0 + s];
            }
#pragma unroll
        for (int s = 0; s < DEPTH; ++s)
            if (s < slabs) {
                float m;
                int byte, e;
                scale_parts<WIDE>(a.sq, sq + slab0 + s, m, byte);
                v4u codes[2];
                e = (int)ep[s];
                if (TYPE == OZIMMU_E4M3 && e == 255) m = __builtin_nanf("");
                cut_slab<TYPE>(x[s], codes, e);
                v8h h[4];
                halves16(codes[0], h[0], h[1]);
                halves16(codes[1], h[2], h[3]);
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    v4f part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        v8h y0, y1;
                        halves16(y[s][c][g], y0, y1);
                        part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y0, h[2 * g], part, 0, 0, 0);
                        part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y1, h[2 * g + 1], part, 0, 0, 0);
                    }
                    // (a lane's sums are of row lane % 16 of P, whose scale it has)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[c][i] += __builtin_amdgcn_ldexpf(part[i] * m, e + byte - 254);
                }
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

// Two tiles of columns to a wavefront, where that leaves a compute unit four workgroups and more: the tokens are cut half as often.
int few_columns(const F8Args& a) { return ((int64_t)a.n + 31) / 32 * ((a.rows + 15) / 16) >= 4 * 256 ? 2 : 1; }

template <int TYPE, int COLS, int DEPTH>
hipError_t launch(const F8Args& a, int waves, hipStream_t st) {
    const int64_t tiles_n = (a.n + 16 * COLS - 1) / (16 * COLS), tiles = ((int64_t)a.rows + 15) / 16 + (a.experts < a.rows ? a.experts : a.rows), grid = tiles * tiles_n;
    if (grid <= 0 || grid > INT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = a.scale_type == OZIMMU_F32 ? f8_few_kernel<TYPE, true, COLS, DEPTH> : f8_few_kernel<TYPE, false, COLS, DEPTH>;
    kernel<<<dim3((unsigned)grid), dim3(waves * 64), 0, st>>>(a, (int)tiles_n);
    return hipGetLastError();
}
// Few workgroups: up to sixteen wavefronts to each, a slab at a time, so that the chip has some for every SIMD; else four wavefronts that ask for
// four slabs at a time.
template <int TYPE>
hipError_t launch_by_columns(const F8Args& a, hipStream_t st) {
    if (few_columns(a) == 2) return launch<TYPE, 2, 4>(a, 4, st);
    const int64_t workgroups = ((int64_t)a.n + 15) / 16 * ((a.rows + 15) / 16);
    if (workgroups > 512) return launch<TYPE, 1, 4>(a, 4, st);
    return launch<TYPE, 1, 1>(a, a.slabs < 1 ? 1 : a.slabs < kMostWaves ? a.slabs : kMostWaves, st);
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
