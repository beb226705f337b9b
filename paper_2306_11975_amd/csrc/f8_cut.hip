// The cut into 8-bit floating point, its inverse, and the transposed operands of gradients (gfx950).
//
// A block of 1 x 128 or 128 x 128 values has the scale 2^e, e the least integer in [-127, 127] with max |x| <= 448 2^e over its finite values;
// the codes are RNE(x 2^-e) in e4m3. x 2^-e is exact, so a code is rounded once. Everything here is one pass over memory, which bounds it. us (a copy of as
// many bytes): cut of 8192 x 8192 bf16 by blocks 41 to 47 (39), its inverse 30 (39, from the last-level cache); 4096 x 4096 bf16 by rows 10.8 (9.8);
// operands of the gradient of 4096 x 8192 x 4096 34 (33), those of its weights' 28 to 31 (29).
#include <algorithm>

#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ unsigned max16(unsigned x) {   // over sixteen neighbouring lanes, in all of them
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));
}

// Runs of a row: a wavefront takes 512 positions of kRows rows, eight to a lane, sixteen lanes to a run.
constexpr int kRows = 4;
template <int TYPE>
__device__ __forceinline__ void split_rows(int64_t n, int64_t k, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds, int64_t block, int64_t chunk) {
    typedef typename Elem<TYPE>::raw raw;
    const int lane = threadIdx.x & 63;
    const int64_t row0 = (block * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kRows, at = chunk * 512 + lane * 8;
    if (row0 >= n) return;
    Eight<TYPE> x[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) load8<TYPE>(static_cast<const raw*>(W) + min(row0 + r, n - 1) * ldw, at, k, x[r]);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (row0 + r >= n) break;
        const int byte = scale_byte(max16(top8<TYPE>(x[r])));
        if (at < ((k + 127) & ~int64_t(127))) *reinterpret_cast<v2u*>(codes + (row0 + r) * ldq + at) = code8<TYPE>(x[r], byte);
        const unsigned four = (unsigned)__builtin_amdgcn_readlane(byte, 0) | (unsigned)__builtin_amdgcn_readlane(byte, 16) << 8 |
                              (unsigned)__builtin_amdgcn_readlane(byte, 32) << 16 | (unsigned)__builtin_amdgcn_readlane(byte, 48) << 24;
        if (lane == 0) *reinterpret_cast<unsigned*>(scales + (row0 + r) * lds + chunk * 4) = four;
    }
}
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void f8_split_rows_kernel(int64_t n, int64_t k, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds) {
    split_rows<TYPE>(n, k, W, ldw, codes, ldq, scales, lds, blockIdx.x, blockIdx.y);
}

// Blocks: a workgroup each; a thread holds eight positions of every sixteenth row.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void f8_split_blocks_kernel(int64_t n, int64_t k, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds, int groups) {
    typedef typename Elem<TYPE>::raw raw;
    __shared__ unsigned tops[kThreads / 64];
    const int64_t row0 = (int64_t)(blockIdx.x / groups) * 128;
    const int group = blockIdx.x % groups;
    const int64_t at = (int64_t)group * 128 + (threadIdx.x & 15) * 8;
    const int r0 = threadIdx.x >> 4;
    Eight<TYPE> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) load8<TYPE>(static_cast<const raw*>(W) + min(row0 + r0 + 16 * i, n - 1) * ldw, at, k, x[i]);
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, top8<TYPE>(x[i]));   // (rows beyond the last repeat it)
    top = max16(top);
    top = max(max((unsigned)__builtin_amdgcn_readlane((int)top, 0), (unsigned)__builtin_amdgcn_readlane((int)top, 16)),
              max((unsigned)__builtin_amdgcn_readlane((int)top, 32), (unsigned)__builtin_amdgcn_readlane((int)top, 48)));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    const int byte = scale_byte(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (row0 + r0 + 16 * i >= n) break;
        *reinterpret_cast<v2u*>(codes + (row0 + r0 + 16 * i) * ldq + at) = code8<TYPE>(x[i], byte);
    }
    if (threadIdx.x == 0) {
        uint8_t* s = scales + (row0 >> 7) * lds;
        s[group] = (uint8_t)byte;
        if (group == groups - 1)
            for (int g = groups; g < ((groups + 3) & ~3); ++g) s[g] = 0;
    }
}

// Values: a wavefront takes 512 positions of kRows rows, eight to a lane.
template <int TYPE, bool WIDE>
__launch_bounds__(kThreads)
__global__ void f8_expand_kernel(int64_t n, int64_t k, int shift, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds, void* W, int64_t ldw) {
    typedef typename Elem<TYPE>::raw raw;
    const int lane = threadIdx.x & 63;
    const int64_t row0 = ((int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kRows, at = (int64_t)blockIdx.y * 512 + lane * 8;
    if (row0 >= n || at >= k) return;
    v2u c[kRows];
    float s[kRows];      // (32 bits hold 2^-127, as a subnormal value, and a product with any scale is rounded once)
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t row = min(row0 + i, n - 1);
        c[i] = *reinterpret_cast<const v2u*>(codes + row * ldq + at);
        s[i] = scale_value<WIDE>(scales, (row >> shift) * lds + (at >> 7));
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (row0 + i >= n) break;
        float f[8];
        values4(c[i][0], *reinterpret_cast<float(*)[4]>(f));
        values4(c[i][1], *reinterpret_cast<float(*)[4]>(f + 4));
        raw r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = f[e] * s[i];
            asm("" : "+v"(x));      // (in one instruction with the rounding to fp16 the product would not be rounded to 32 bits first)
            r[e] = Elem<TYPE>::store(x);
        }
        raw* out = static_cast<raw*>(W) + (row0 + i) * ldw + at;
        if (at + 8 <= k) {
            *reinterpret_cast<v4u_any*>(out) = *reinterpret_cast<const v4u*>(r);
            if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u_any*>(out + 4) = *reinterpret_cast<const v4u*>(r + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < k) out[e] = r[e];
        }
    }
}

// Transposed weights: a workgroup turns a block of 128 x 128 in LDS, four by four bytes to a thread. The rows of a gradient are cut in the same launch,
// by the workgroups behind those.
struct Turn {
    int64_t n, k;
    const uint8_t* codes;
    int64_t ldq;
    const void* scales;
    int64_t lds;
    uint8_t* codes_t;
    void* scales_t;
    int64_t ld_t, lds_t;
    int nb, kb, blocks;
};
struct Rows {
    int64_t n, k;
    const void* V;
    int64_t ldv;
    uint8_t* codes;
    int64_t ld;
    uint8_t* scales;
    int64_t lds;
    int chunks;
};
template <int TYPE, bool WIDE>
__launch_bounds__(kThreads)
__global__ void f8_gradient_operands_kernel(Turn t, Rows v) {
    __shared__ unsigned block[128][33];
    if ((int)blockIdx.x >= t.blocks) {
        const int b = blockIdx.x - t.blocks;
        split_rows<TYPE>(v.n, v.k, v.V, v.ldv, v.codes, v.ld, v.scales, v.lds, b / v.chunks, b % v.chunks);
        return;
    }
    const int line = blockIdx.x / t.kb, bk = blockIdx.x - line * t.kb, expert = line / t.nb, bn = line - expert * t.nb;
    const uint8_t* from = t.codes + (expert * t.n + (int64_t)bn * 128) * t.ldq + (int64_t)bk * 128;
    const int rows = (int)min<int64_t>(128, t.n - (int64_t)bn * 128), cols = (int)min<int64_t>(128, t.k - (int64_t)bk * 128);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = (threadIdx.x >> 3) + 32 * i, p = threadIdx.x & 7;
        v4u x = {0, 0, 0, 0};
        if (r < rows) x = *reinterpret_cast<const v4u*>(from + r * t.ldq + p * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) block[r][p * 4 + e] = x[e];
    }
    __syncthreads();
    uint8_t* to = t.codes_t + (expert * t.k + (int64_t)bk * 128) * t.ld_t + (int64_t)bn * 128;
    const int r4 = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c4 = (threadIdx.x >> 5) + 8 * i;
        unsigned x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = block[4 * r4 + e][c4];
        const unsigned a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);   // bytes 0 and 1 of each pair
        const unsigned c = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);   // bytes 2 and 3
        const unsigned y[4] = {__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x05040100u),
                               __builtin_amdgcn_perm(d, c, 0x07060302u)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (4 * c4 + e < cols) *reinterpret_cast<unsigned*>(to + (int64_t)(4 * c4 + e) * t.ld_t + 4 * r4) = y[e];
    }
    if (threadIdx.x == 0) {
        const int64_t at = ((int64_t)expert * t.nb + bn) * t.lds + bk, at_t = ((int64_t)expert * t.kb + bk) * t.lds_t + bn;
        if constexpr (WIDE)
            static_cast<float*>(t.scales_t)[at_t] = static_cast<const float*>(t.scales)[at];
        else
            static_cast<uint8_t*>(t.scales_t)[at_t] = static_cast<const uint8_t*>(t.scales)[at];
    }
}

// Runs along the tokens: a workgroup takes 128 tokens of an expert and 64 columns; a thread holds eight columns of four neighbouring tokens,
// whose codes are a word of the transposed row.
// Both operands of a weights' gradient in one launch.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void f8_cut_tokens_kernel(int rows, int experts, const int* offsets, F8Columns dy, F8Columns x, int runs) {
    typedef typename Elem<TYPE>::raw raw;
    const int dy_tiles = (int)((dy.n + 63) / 64), first_x = runs * dy_tiles;
    const bool second = (int)blockIdx.x >= first_x;
    const int tiles = second ? (int)((x.n + 63) / 64) : dy_tiles, number = second ? blockIdx.x - first_x : blockIdx.x, t = second ? x.t : dy.t;
    const int64_t n = second ? x.n : dy.n, ldv = second ? x.ldv : dy.ldv, ld = (int64_t)runs * 128, lds = runs;
    const int* source = second ? x.source : dy.source;
    const void* V = second ? x.V : dy.V;
    uint8_t *codes = second ? x.codes : dy.codes, *scales = second ? x.scales : dy.scales;
    __shared__ unsigned tops[kThreads / 64][64];
    __shared__ unsigned turned[64][33];
    const int run = number / tiles, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col0 = (int64_t)(number % tiles) * 64;
    int first = 0, count = rows, unit = run;
    if (experts) {
        Segment s;
        if (!find_unit(offsets, experts, rows, 128, 4, run, s)) return;
        first = s.first;
        count = s.count;
        unit = s.unit;
    }
    if (unit * 128 >= count) return;
    const int token0 = unit * 128 + (threadIdx.x >> 3) * 4;   // within the expert's
    const int64_t at = col0 + (threadIdx.x & 7) * 8;
    float f[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int64_t row = first + min(token0 + i, count - 1);
        bool there = token0 + i < count;
        if (source) {
            const int s = source[row];
            there = there && (unsigned)s < (unsigned)t;
            row = there ? s : 0;
        }
        Eight<TYPE> x;
        load8<TYPE>(static_cast<const raw*>(V) + row * ldv, at, n, x);
        floats<TYPE>(x, f[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[i][e] = there ? f[i][e] : 0.f;
    }
    unsigned top[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        top[e] = max(max(finite_bits(f[0][e]), finite_bits(f[1][e])), max(finite_bits(f[2][e]), finite_bits(f[3][e])));
#pragma unroll
        for (int d = 8; d < 64; d <<= 1) top[e] = max(top[e], (unsigned)__shfl_xor((int)top[e], d));
        if (lane < 8) tops[wave][lane * 8 + e] = top[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = (threadIdx.x & 7) * 8 + e;
        const int byte = scale_byte(max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c])));
        const float x[4] = {f[0][e], f[1][e], f[2][e], f[3][e]};
        turned[c][threadIdx.x >> 3] = code4(x, byte);
    }
    if (threadIdx.x < 64 && col0 + threadIdx.x < n)
        scales[(col0 + threadIdx.x) * lds + run] = (uint8_t)scale_byte(max(max(tops[0][threadIdx.x], tops[1][threadIdx.x]), max(tops[2][threadIdx.x], tops[3][threadIdx.x])));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (threadIdx.x >> 3) + 32 * i, p = (threadIdx.x & 7) * 4;
        if (col0 + c < n) *reinterpret_cast<v4u*>(codes + (col0 + c) * ld + (int64_t)run * 128 + p * 4) = v4u{turned[c][p], turned[c][p + 1], turned[c][p + 2], turned[c][p + 3]};
    }
}

template <class F>
hipError_t by_type(int type, F&& f) {
    switch (type) {
        case OZIMMU_F32: f(std::integral_constant<int, OZIMMU_F32>{}); break;
        case OZIMMU_BF16: f(std::integral_constant<int, OZIMMU_BF16>{}); break;
        default: f(std::integral_constant<int, OZIMMU_F16>{}); break;
    }
    return hipGetLastError();
}
bool too_many(int64_t workgroups) { return workgroups <= 0 || workgroups > INT32_MAX; }

}  // namespace

hipError_t launch_f8_split(int64_t n, int64_t k, int block_rows, const void* W, int type, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds, hipStream_t st) {
    const int64_t groups = f8_groups(k), blocks = (n + 127) / 128 * groups;
    const dim3 rows((unsigned)((n + 4 * kRows - 1) / (4 * kRows)), (unsigned)((k + 511) / 512));
    if (too_many(blocks)) return hipErrorInvalidConfiguration;
    return by_type(type, [&](auto kind) {
        constexpr int T = decltype(kind)::value;
        if (block_rows == 1)
            f8_split_rows_kernel<T><<<rows, dim3(kThreads), 0, st>>>(n, k, W, ldw, codes, ldq, scales, lds);
        else
            f8_split_blocks_kernel<T><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(n, k, W, ldw, codes, ldq, scales, lds, (int)groups);
    });
}

hipError_t launch_f8_expand(int64_t n, int64_t k, int block_rows, const uint8_t* codes, int64_t ldq, int scale_type, const void* scales, int64_t lds, void* W, int type, int64_t ldw, hipStream_t st) {
    const dim3 grid((unsigned)((n + 4 * kRows - 1) / (4 * kRows)), (unsigned)((k + 511) / 512));
    return by_type(type, [&](auto kind) {
        constexpr int T = decltype(kind)::value;
        auto kernel = scale_type == OZIMMU_F32 ? f8_expand_kernel<T, true> : f8_expand_kernel<T, false>;
        kernel<<<grid, dim3(kThreads), 0, st>>>(n, k, block_rows == 1 ? 0 : 7, codes, ldq, scales, lds, W, ldw);
    });
}

hipError_t launch_f8_gradient_operands(int64_t experts, int64_t n, int64_t k, const uint8_t* codes, int64_t ldq, int scale_type, const void* scales, int64_t lds, uint8_t* codes_t,
                                       void* scales_t, int64_t rows, const void* V, int type, int64_t ldv, uint8_t* v_codes, uint8_t* v_scales, hipStream_t st) {
    const int64_t nb = f8_groups(n), kb = f8_groups(k), blocks = experts * nb * kb, chunks = (n + 511) / 512, cuts = v_codes ? (rows + 4 * kRows - 1) / (4 * kRows) * chunks : 0;
    if (too_many(blocks + cuts)) return hipErrorInvalidConfiguration;
    const Turn t{n, k, codes, ldq, scales, lds, codes_t, scales_t, f8_row_bytes(n), f8_scale_bytes(n), (int)nb, (int)kb, (int)blocks};
    const Rows v{rows, n, V, ldv, v_codes, f8_row_bytes(n), v_scales, f8_scale_bytes(n), (int)chunks};
    return by_type(type, [&](auto kind) {
        constexpr int T = decltype(kind)::value;
        auto kernel = scale_type == OZIMMU_F32 ? f8_gradient_operands_kernel<T, true> : f8_gradient_operands_kernel<T, false>;
        kernel<<<dim3((unsigned)(blocks + cuts)), dim3(kThreads), 0, st>>>(t, v);
    });
}

hipError_t launch_f8_cut_tokens(int64_t rows, int64_t experts, const int* offsets, int type, const F8Columns& dy, const F8Columns& x, int64_t runs, hipStream_t st) {
    const int64_t grid = runs * ((dy.n + 63) / 64 + (x.n + 63) / 64);
    if (too_many(grid)) return hipErrorInvalidConfiguration;
    return by_type(type, [&](auto kind) { f8_cut_tokens_kernel<decltype(kind)::value><<<dim3((unsigned)grid), dim3(kThreads), 0, st>>>((int)rows, (int)experts, offsets, dy, x, (int)runs); });
}

}  // namespace ozimmu
