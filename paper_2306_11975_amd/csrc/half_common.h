// Device helpers for 16-bit and mixed types (gfx950 only).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "mfma_common.h"
#include "weights_internal.h"

namespace ozimmu {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
// vectors at the alignment of 16-bit values (global memory takes them at any): rows may start anywhere
typedef v4u v4u_any __attribute__((aligned(2)));
typedef v2u v2u_any __attribute__((aligned(2)));
typedef unsigned u32_any __attribute__((aligned(2)));

__device__ __forceinline__ float f16_to_f32(unsigned short b) { return (float)__builtin_bit_cast(_Float16, b); }
__device__ __forceinline__ unsigned short f32_to_f16(float x) { return __builtin_bit_cast(unsigned short, (_Float16)x); }
__device__ __forceinline__ float bf16_to_f32(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ unsigned short f32_to_bf16(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }   // nearest, ties to even

template <int TYPE> struct Elem;   // one value of an ozimmu_type_t
template <> struct Elem<OZIMMU_F32> {
    typedef float raw;
    static __device__ __forceinline__ float load(raw r) { return r; }
    static __device__ __forceinline__ raw store(float x) { return x; }
};
template <> struct Elem<OZIMMU_BF16> {
    typedef unsigned short raw;
    static __device__ __forceinline__ float load(raw r) { return bf16_to_f32(r); }
    static __device__ __forceinline__ raw store(float x) { return f32_to_bf16(x); }
};
template <> struct Elem<OZIMMU_F16> {
    typedef unsigned short raw;
    static __device__ __forceinline__ float load(raw r) { return f16_to_f32(r); }
    static __device__ __forceinline__ raw store(float x) { return f32_to_f16(x); }
};

// x = first + second, each rounded to fp16: 22 bits and more of x, down to 2^-24 absolutely
__device__ __forceinline__ void two_slices(float x, unsigned short& first, unsigned short& second) {
    const _Float16 h = (_Float16)x;
    first = __builtin_bit_cast(unsigned short, h);
    second = __builtin_bit_cast(unsigned short, (_Float16)(x - (float)h));
}

template <bool BF16>
__device__ __forceinline__ v4f mfma_half(const v4u& a, const v4u& b, const v4f& c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

}  // namespace
}  // namespace ozimmu
