// R = P Q^T for codes in 8-bit floating point, few rows of P to an expert: one token and up, straight from memory (gfx950).
//
// Bound: the bytes of Q. A wavefront takes 16 rows of P and 16 of Q at a time; a lane reads 16 bytes of a row of either and the 16 that lie 64
// further on, so that 16 rows of 128 bytes, a slab, come by whole lines. The matrix cores' 8-bit products drop what is below 2^-13 of the
// largest of eight; here, where the bytes are what takes time, the codes become fp16, which holds each of them, and the sums of a slab's 128
// products are 32-bit ones. They are scaled and added slab by slab. Four wavefronts share the inner dimension, 512 positions at a time (a word
// of scales), and add up in order at the end.
#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kWaves = 4;

template <bool WIDE>
__launch_bounds__(kWaves * 64)
__global__ void f8_few_kernel(F8Args a, int tiles_n) {
    __shared__ v4f sums[kWaves - 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x / tiles_n, col0 = (blockIdx.x % tiles_n) * 16;
    int first = 0, count = a.rows, unit = tile, expert = 0;
    if (a.experts) {
        Segment s;
        if (!find_unit(a.offsets, a.experts, a.rows, 16, 1, tile, s)) return;
        first = s.first;
        count = s.count;
        unit = s.unit;
        expert = s.expert;
    }
    const int r = unit * 16 + (lane & 15), col = col0 + (lane & 15);
    int64_t row = first + min(r, count - 1);
    bool there = r < count;
    const int64_t out_row = row;
    if (a.source) {
        const int s = a.source[row];
        const bool in = (unsigned)s < (unsigned)a.t;
        row = in ? s : 0;
        there = there && in;
    }
    const unsigned piece = (lane >> 4) * 16;
    const uint8_t* p = a.P + row * a.ldp + piece;
    const uint8_t* sp = a.sp + row * a.ldsp;
    const uint8_t* q = a.Q + ((int64_t)expert * a.n + min(col, a.n - 1)) * a.ldq + piece;
    const int64_t sq = ((int64_t)expert * ((a.n + 127) >> 7) + (col0 >> 7)) * a.ldsq;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    for (int slab0 = wave * 4; slab0 < a.slabs; slab0 += kWaves * 4) {
        const int slabs = min(4, a.slabs - slab0);
        const unsigned ep = *reinterpret_cast<const unsigned*>(sp + slab0);
        v4u x[4][2], y[4][2];
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (s < slabs) {
                const int64_t at = (int64_t)(slab0 + s) * 128;
                y[s][0] = *reinterpret_cast<const v4u*>(q + at);
                y[s][1] = *reinterpret_cast<const v4u*>(q + at + 64);
                x[s][0] = *reinterpret_cast<const v4u*>(p + at);
                x[s][1] = *reinterpret_cast<const v4u*>(p + at + 64);
            }
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (s < slabs) {
                float m;
                int byte;
                scale_parts<WIDE>(a.sq, sq + slab0 + s, m, byte);
                v4f part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v8h x0, x1, y0, y1;
                    halves16(x[s][h], x0, x1);
                    halves16(y[s][h], y0, y1);
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y0, x0, part, 0, 0, 0);
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(y1, x1, part, 0, 0, 0);
                }
                const int e = (int)(ep >> (8 * s) & 255u) + byte - 254;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] += __builtin_amdgcn_ldexpf(part[i] * m, e);
            }
    }
    if (wave) sums[wave - 1][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += sums[w][lane][i];
    if (r < count) store_four(a, out_row, col0 + (lane >> 4) * 4, acc, there);
}

}  // namespace

hipError_t launch_f8_few(const F8Args& a, hipStream_t st) {
    const int64_t tiles_n = (a.n + 15) / 16, tiles = ((int64_t)a.rows + 15) / 16 + (a.experts < a.rows ? a.experts : a.rows), grid = tiles * tiles_n;
    if (grid <= 0 || grid > INT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = a.scale_type == OZIMMU_F32 ? f8_few_kernel<true> : f8_few_kernel<false>;
    kernel<<<dim3((unsigned)grid), dim3(kWaves * 64), 0, st>>>(a, (int)tiles_n);
    return hipGetLastError();
}

}  // namespace ozimmu
