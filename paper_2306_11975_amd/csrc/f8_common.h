// Device helpers for 8-bit floating point (e4m3: sign, four bits of exponent, three of fraction; 448 is the largest value, 0x7f a NaN, no
// infinities) under power-of-two scales, and for rows sorted by expert (gfx950 only).
#pragma once

#include "eight_internal.h"
#include "half_common.h"

namespace ozimmu {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v2i __attribute__((ext_vector_type(2)));

// Byte e + 127 of the least e in [-127, 127] with top <= 448 2^e, for the bits of a finite top >= 0: 448 is 1.75 2^8, so the exponent goes up
// where the fraction exceeds that of 1.75.
__device__ __forceinline__ int scale_byte(unsigned top) { return max(0, (int)((top + 0x1fffffu) >> 23) - 8); }
// The magnitude's bits where it is finite, else 0.
__device__ __forceinline__ unsigned finite_bits(float x) {
    const unsigned a = __float_as_uint(x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}
// Four codes as a word, under the scale of a byte. The conversion takes the scale's exponent: x 2^-e is exact, or far below the least code, and is
// rounded once, to nearest, ties to even. What is not finite becomes a NaN.
typedef short v2s __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned code4(const float* x, int byte) {
    const float scale = __uint_as_float((unsigned)byte << 23);
    v2s w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[0], x[1], scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[2], x[3], scale, true);
    return __builtin_bit_cast(unsigned, w);
}
template <int TYPE>
struct Eight {   // eight consecutive values as they lie
    v4u raw[TYPE == OZIMMU_F32 ? 2 : 1];
};
template <int TYPE>
__device__ __forceinline__ void load8(const typename Elem<TYPE>::raw* row, int64_t at, int64_t len, Eight<TYPE>& x) {
    typedef typename Elem<TYPE>::raw raw;
    if (at + 8 <= len) {
        x.raw[0] = *reinterpret_cast<const v4u_any*>(row + at);
        if constexpr (TYPE == OZIMMU_F32) x.raw[1] = *reinterpret_cast<const v4u_any*>(row + at + 4);
    } else {
        raw r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = at + e < len ? row[at + e] : raw(0);
        x = __builtin_bit_cast(Eight<TYPE>, r);
    }
}
template <int TYPE>
__device__ __forceinline__ void floats(const Eight<TYPE>& x, float (&f)[8]) {
    if constexpr (TYPE == OZIMMU_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(x.raw[e >> 2][e & 3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = Elem<TYPE>::load((unsigned short)(x.raw[0][e] & 0xffffu));
            f[2 * e + 1] = Elem<TYPE>::load((unsigned short)(x.raw[0][e] >> 16));
        }
    }
}
// Codes of eight values as they lie.
template <int TYPE>
__device__ __forceinline__ v2u code8(const Eight<TYPE>& x, int byte) {
    const float scale = __uint_as_float((unsigned)byte << 23);
    v2u out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v2s w = {0, 0};
        const unsigned first = x.raw[0][2 * h], second = x.raw[0][2 * h + 1];   // (a bit cast of a vector's element takes element 0)
        if constexpr (TYPE == OZIMMU_F32) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, __uint_as_float(x.raw[h][0]), __uint_as_float(x.raw[h][1]), scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, __uint_as_float(x.raw[h][2]), __uint_as_float(x.raw[h][3]), scale, true);
        } else if constexpr (TYPE == OZIMMU_BF16) {
            typedef __bf16 v2b __attribute__((ext_vector_type(2)));
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(v2b, first), scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(v2b, second), scale, true);
        } else {
            typedef _Float16 v2h __attribute__((ext_vector_type(2)));
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(v2h, first), scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(v2h, second), scale, true);
        }
        out[h] = __builtin_bit_cast(unsigned, w);
    }
    return out;
}
// The largest finite magnitude's bits (of 32-bit floats) among eight values as they lie.
template <int TYPE>
__device__ __forceinline__ unsigned top8(const Eight<TYPE>& x) {
    unsigned t = 0;
    if constexpr (TYPE == OZIMMU_BF16) {   // bits order like magnitudes: the halves of the words each for themselves
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned low = x.raw[0][e] << 16 & 0x7fffffffu, high = x.raw[0][e] & 0x7fff0000u;
            t = max(t, max(low < 0x7f800000u ? low : 0u, high < 0x7f800000u ? high : 0u));
        }
    } else {
        float f[8];
        floats<TYPE>(x, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) t = max(t, finite_bits(f[e]));
    }
    return t;
}
// The values of a word of codes.
__device__ __forceinline__ void values4(unsigned w, float (&x)[4]) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
// Sixteen codes as fp16, which holds each of them.
__device__ __forceinline__ void halves16(const v4u& w, v8h& first, v8h& second) {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    v2h h[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[i], 1.0f, false);
        h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[i], 1.0f, true);
    }
    first = v8h{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
    second = v8h{h[4][0], h[4][1], h[5][0], h[5][1], h[6][0], h[6][1], h[7][0], h[7][1]};
}

// A scale of the weights as significand and exponent byte: value = m 2^(byte - 127). Bytes: m = 1. A NaN or infinity: byte 255.
__device__ __forceinline__ void scale_parts(unsigned bits, float& m, int& byte) {   // of 32 bits
    byte = (int)(bits >> 23 & 255u);
    m = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
    if (byte == 0) {   // subnormal: fraction 2^-126
        byte = 1;
        m = __builtin_amdgcn_ldexpf((float)(bits & 0x7fffffu), -23);
    }
    m = bits >> 31 ? -m : m;
    if (byte == 255) m = __builtin_nanf("");
}
template <bool WIDE>
__device__ __forceinline__ void scale_parts(const void* scales, int64_t at, float& m, int& byte) {
    if constexpr (WIDE) {
        scale_parts(static_cast<const unsigned*>(scales)[at], m, byte);
    } else {
        byte = static_cast<const uint8_t*>(scales)[at];
        m = byte == 255 ? __builtin_nanf("") : 1.0f;
    }
}
// The scale itself; a NaN where it is not finite.
template <bool WIDE>
__device__ __forceinline__ float scale_value(const void* scales, int64_t at) {
    unsigned bits;
    if constexpr (WIDE) {
        bits = static_cast<const unsigned*>(scales)[at];
    } else {
        const unsigned byte = static_cast<const uint8_t*>(scales)[at];
        bits = byte ? byte << 23 : 0x400000u;
    }
    return (bits >> 23 & 255u) == 255u ? __builtin_nanf("") : __uint_as_float(bits);
}

// ---- rows sorted by expert

__device__ __forceinline__ int wave_scan(int x) {   // inclusive sum over the lanes before and this one: within rows of sixteen, then the rows' last
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
}
// The experts' rows, whatever the offsets hold: an offset is taken as at least the largest before it and within [0, rows], so that no two
// experts share rows. Units are of `unit` rows, counted in multiples of `to` for each expert. Every lane of a wavefront calls these with the same
// arguments.
struct Segment {
    int expert, first, count;   // its rows
    int unit;                   // the unit's number within the expert
    int before;                 // units of the experts before it
};
template <class F>
__device__ __forceinline__ int over_experts(const int* offsets, int experts, int rows, int unit, int to, F&& f) {
    const int lane = threadIdx.x & 63;
    int base = 0, least = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        int first = rows, end = rows;
        if (e < experts) {
            first = min(max(offsets[e], 0), rows);
            end = min(max(offsets[e + 1], 0), rows);
        }
        if (__builtin_amdgcn_ballot_w64(end < first || first < least)) {   // some fall: the largest so far instead
            first = max(first, least);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_up(first, d);
                first = lane >= d ? max(first, y) : first;
            }
            end = max(first, end);
        }
        least = __builtin_amdgcn_readlane(end, 63);
        const int count = e < experts ? end - first : 0;
        int units = (count + unit - 1) / unit;
        units = (units + to - 1) / to * to;
        const int sum = wave_scan(units);
        f(e, first, count, units, base + sum - units);
        base += __builtin_amdgcn_readlane(sum, 63);
    }
    return base;
}
__device__ __forceinline__ int count_units(const int* offsets, int experts, int rows, int unit) {
    return over_experts(offsets, experts, rows, unit, 1, [](int, int, int, int, int) {});
}
__device__ __forceinline__ bool find_unit(const int* offsets, int experts, int rows, int unit, int to, int index, Segment& s) {
    bool found = false;
    over_experts(offsets, experts, rows, unit, to, [&](int e, int first, int count, int units, int before) {
        const unsigned long long here = __builtin_amdgcn_ballot_w64(index >= before && index < before + units);
        if (here) {
            const int l = __builtin_ctzll(here);
            s.expert = __builtin_amdgcn_readlane(e, l);
            s.first = __builtin_amdgcn_readlane(first, l);
            s.count = __builtin_amdgcn_readlane(count, l);
            s.before = __builtin_amdgcn_readlane(before, l);
            s.unit = index - s.before;
            found = true;
        }
    });
    return found;
}

// Two values rounded to 16 bits, as a word.
template <int TYPE>
__device__ __forceinline__ unsigned two_as(float x, float y) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    if constexpr (TYPE == OZIMMU_BF16)
        return __builtin_bit_cast(unsigned, __builtin_convertvector(v2f{x, y}, v2b));
    else
        return __builtin_bit_cast(unsigned, __builtin_convertvector(v2f{x, y}, v2h));
}

// R[row][col .. col + 3], rounded once to the result's type; zeros where the row has no source.
template <int TYPE>
__device__ __forceinline__ void store_four_as(const F8Args& a, int64_t row, int col, const v4f& v, bool there) {
    typedef typename Elem<TYPE>::raw raw;
    typedef raw raw4 __attribute__((ext_vector_type(4)));
    typedef raw4 raw4_any __attribute__((aligned(sizeof(raw))));
    raw* at = static_cast<raw*>(a.out) + row * a.ldo + col;
    raw4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = Elem<TYPE>::store(there ? v[e] : 0.f);
    if (col + 4 <= a.n)
        *reinterpret_cast<raw4_any*>(at) = x;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.n) at[e] = x[e];
}
__device__ __forceinline__ void store_four(const F8Args& a, int64_t row, int col, const v4f& v, bool there) {
    if (a.out_type == OZIMMU_F32)
        store_four_as<OZIMMU_F32>(a, row, col, v, there);
    else if (a.out_type == OZIMMU_BF16)
        store_four_as<OZIMMU_BF16>(a, row, col, v, there);
    else
        store_four_as<OZIMMU_F16>(a, row, col, v, there);
}

}  // namespace
}  // namespace ozimmu
