// Weights in four bits: the cut, its inverse, and the operands of their matrix-core product (gfx950).
//
// Group g of row i: s = RN_T(RN_32(max |w| / 7)), c = RNE(w / s) clamped to [-8, 7], stored as c + 8, two to a byte, the even
// position in the low half; a row takes a multiple of 16 bytes (32 codes), what is beyond k stands for zero.
#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;

// Eight consecutive values of a row, zero beyond the end. vec: the row's addresses are 16-byte aligned.
template <int TYPE>
__device__ __forceinline__ void load8(const typename Elem<TYPE>::raw* row, int64_t at, int64_t len, bool vec, float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    if (vec && at + 8 <= len) {
        raw r[8];
        if constexpr (TYPE == OZIMMU_F32) {
            *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u*>(row + at);
            *reinterpret_cast<v4u*>(r + 4) = *reinterpret_cast<const v4u*>(row + at + 4);
        } else {
            *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u*>(row + at);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Elem<TYPE>::load(r[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < len ? Elem<TYPE>::load(row[at + e]) : 0.f;
    }
}
template <int TYPE>
__device__ __forceinline__ void store8(typename Elem<TYPE>::raw* row, int64_t at, int64_t len, bool vec, const float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    raw r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = Elem<TYPE>::store(x[e]);
    if (vec && at + 8 <= len) {
        *reinterpret_cast<v4u*>(row + at) = *reinterpret_cast<const v4u*>(r);
        if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u*>(row + at + 4) = *reinterpret_cast<const v4u*>(r + 4);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < len) row[at + e] = r[e];
    }
}

// The nearest integer to w / s, ties to even: the quotient itself, not one rounded to 32 bits, which may fall onto a border that
// the quotient only comes near. The remainder w - q s of the candidate is exact in 32 bits (|q| <= 16, and it is a multiple of half a
// unit of s no larger than about s), so comparing it with s / 2 decides.
__device__ __forceinline__ int nearest_code(float w, float s, float inv) {
    float q = rintf(fminf(fmaxf(w * inv, -9.f), 8.f));
    const float r = fmaf(-q, s, w), half = 0.5f * s, a = fabsf(r);
    const bool odd = ((int)q & 1) != 0;
    if (a > half || (a == half && odd)) q += r > 0.f ? 1.f : -1.f;
    return (int)fminf(fmaxf(q, -8.f), 7.f);
}

// The largest magnitude of eight values, as bits: those of |w| order like the values, NaN last, so that one that is there stays visible in the scale. As integers the
// largest is the largest positive value, as unsigned ones the largest negative one.
__device__ __forceinline__ unsigned top_bits(const float (&w)[8]) {
    int up = 0;
    unsigned down = 0x80000000u;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        up = max(up, max(__float_as_int(w[e]), __float_as_int(w[e + 1])));
        down = max(down, max(__float_as_uint(w[e]), __float_as_uint(w[e + 1])));
    }
    return max((unsigned)up, down & 0x7fffffffu);
}
// The maximum over N neighbouring lanes (4, 8 or 16), in all of them.
template <int N>
__device__ __forceinline__ unsigned max_of_lanes(unsigned x) {
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));    // lanes 1, 0, 3, 2
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));    // lanes 2, 3, 0, 1
    if constexpr (N >= 8) x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));   // eight mirrored
    if constexpr (N >= 16) x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));  // sixteen mirrored
    return x;
}

// The codes of eight weights as a word. w * (1/s), with a reciprocal that is off by a unit, is off the quotient by less than 2e-6; adding 1.5 * 2^23 rounds it to an integer, ties to
// even, whose low bits then stand in the low bits of the sum. That is the nearest integer to the quotient unless the product lies within 1e-5 of a border and is
// not the quotient itself (a tie, which weights of 8 bits often are): then the remainders decide, as they do where a scale that underflowed lets codes leave their range.
// (Both tests are asked of the wavefront: lane by lane, everyone would pay for them. 8192 x 8192 bf16: with the remainders always 62 us.)
__device__ __forceinline__ unsigned code_word(const float (&w)[8], float s, float top) {
    const float inv = __builtin_amdgcn_rcpf(s);
    float t[8], far = 0.f;
    unsigned sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        t[e] = w[e] * inv;
        const float x = t[e] + 12582912.f;
        sum[e] = __float_as_uint(x);
        far = fmaxf(far, fabsf(t[e] - (x - 12582912.f)));
    }
    bool unsure = !(s >= 0x1p-60f && s <= 3.4028234664e38f) || top * inv > 7.4f;
    if (__builtin_amdgcn_ballot_w64(far > 0.49999f)) {   // the quotients near a border once more, corrected by their remainders: then ties are exact
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = fmaf(fmaf(-t[e], s, w[e]), inv, t[e]), x = q + 12582912.f;
            sum[e] = __float_as_uint(x);
            unsure |= fabsf(q - (x - 12582912.f)) > 0.49999f && fmaf(-q, s, w[e]) != 0.f;
        }
    }
    // bytes of the even positions and of the odd ones
    const unsigned even = __builtin_amdgcn_perm(__builtin_amdgcn_perm(sum[6], sum[4], 0x0c0c0400u), __builtin_amdgcn_perm(sum[2], sum[0], 0x0c0c0400u), 0x05040100u);
    const unsigned odd = __builtin_amdgcn_perm(__builtin_amdgcn_perm(sum[7], sum[5], 0x0c0c0400u), __builtin_amdgcn_perm(sum[3], sum[1], 0x0c0c0400u), 0x05040100u);
    unsigned word = ((even & 0x0f0f0f0fu) | (odd & 0x0f0f0f0fu) << 4) ^ 0x88888888u;
    if (__builtin_amdgcn_ballot_w64(unsure)) {
        const bool usable = s > 0.f && s <= 3.4028234664e38f;
        const float up = s < 0x1p-60f ? 0x1p64f : 1.f;   // (small scales: the reciprocal stays finite and the remainders normal)
        unsigned exact = 0;
#pragma unroll 1
        for (int e = 7; e >= 0; --e) {
            float x = w[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) x = e == i ? w[i] : x;
            exact = exact << 4 | (unsigned)((usable ? nearest_code(x * up, s * up, 1.0f / (s * up)) : 0) + 8);
        }
        if (unsure) word = exact;
    }
    return word;
}

// max |w| / 7, correctly rounded: the product with the rounded reciprocal, corrected by its remainder; very small ones, whose remainder would underflow, and infinities divided.
__device__ __forceinline__ float seventh(float top) {
    constexpr float r = 1.0f / 7.0f;
    const float q = top * r;
    const float exact = fmaf(fmaf(-7.0f, q, top), r, q);
    const bool plain = top > 1e-30f && top <= 3.4028234664e38f;
    if (__builtin_amdgcn_ballot_w64(!plain)) return plain ? exact : top / 7.0f;
    return exact;
}

// A thread cuts eight weights of two rows; the lanes of a group (GROUP / 8 of them, side by side) share its maximum. tx threads along a row.
// Memory-bound: the weights are read once, 16 or 32 bytes a lane, two rows on their way at a time.
template <int TYPE, int STYPE, int GROUP>
__launch_bounds__(kThreads)
__global__ void q4_split_kernel(int64_t n, int64_t k, const void* W, int64_t ldw, bool vec, uint8_t* codes, int64_t ldq, void* scales,
                                int64_t lds, int tx, unsigned across) {
    typedef Elem<TYPE> E;
    typedef Elem<STYPE> S;
    constexpr int ROWS = 2;
    const int ty = kThreads / tx;
    const int64_t row0 = (int64_t)(blockIdx.x / across) * (ROWS * ty) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(blockIdx.x % across) * tx + threadIdx.x % tx) * 8;
    float w[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) load8<TYPE>(reinterpret_cast<const typename E::raw*>(W) + min(row0 + i * ty, n - 1) * ldw, at, k, vec, w[i]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = row0 + i * ty;
        const float top = __uint_as_float(max_of_lanes<GROUP / 8>(top_bits(w[i])));
        const typename S::raw stored = S::store(seventh(top));
        const unsigned word = code_word(w[i], S::load(stored), top);
        if (row < n) {
            if (at < pad_to(k, 32)) *reinterpret_cast<unsigned*>(codes + row * ldq + at / 2) = word;
            if (at < k && at % GROUP == 0) reinterpret_cast<typename S::raw*>(scales)[row * lds + at / GROUP] = stored;
        }
    }
}

__device__ __forceinline__ float code_value(unsigned word, int e) { return (float)((int)(word >> (4 * e) & 15u) - 8); }

// The weights s c, each rounded once to the result's type.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void q4_expand_kernel(int64_t n, int64_t k, int group_log2, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                                 void* W, int64_t ldw, int64_t len, bool vec, int tx, unsigned across) {
    typedef Elem<TYPE> E;
    const int64_t row = (int64_t)(blockIdx.x / across) * (kThreads / tx) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(blockIdx.x % across) * tx + threadIdx.x % tx) * 8;
    if (row >= n || at >= len) return;
    float x[8] = {};
    if (at < k) {
        const unsigned word = *reinterpret_cast<const unsigned*>(codes + row * ldq + at / 2);
        const float s = E::load(reinterpret_cast<const typename E::raw*>(scales)[row * lds + (at >> group_log2)]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < k ? s * code_value(word, e) : 0.f;
    }
    store8<TYPE>(reinterpret_cast<typename E::raw*>(W) + row * ldw, at, len, vec, x);
}

__device__ __forceinline__ int exponent_of(float top) {   // of the power of two just above; 0 for zero
    int e = 0;
    if (top > 0.f) {
        if (top <= 3.4028234664e38f)
            (void)frexpf(top, &e);
        else
            e = 128;
    }
    return e;
}
constexpr int kRowShift = 15;   // rows in two slices of fp16 are scaled to just below 2^15

__device__ __forceinline__ float block_max(float x, float* shared) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = shared[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) x = fmaxf(x, shared[i]);
    __syncthreads();
    return x;
}

// Two slices of eight neighbouring values into a row of slabs (32 positions of the first slice, then of the second).
__device__ __forceinline__ void store_slices8(unsigned short* row, int64_t at, const float (&x)[8]) {
    unsigned short h[8], l[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) two_slices(x[e], h[e], l[e]);
    unsigned short* to = row + (at >> 5) * 64 + (at & 31);
    *reinterpret_cast<v4u*>(to) = *reinterpret_cast<const v4u*>(h);
    *reinterpret_cast<v4u*>(to + 32) = *reinterpret_cast<const v4u*>(l);
}

// Rows of 32-bit values in two slices of fp16 under a power-of-two exponent per row; a workgroup per row, which it reads twice
// (the second time from the caches). NaN does not raise the maximum and stays in its place; so does an infinity.
__launch_bounds__(kThreads)
__global__ void row_slices_kernel(int64_t k, const float* X, int64_t ldx, bool vec, unsigned short* out, int64_t ldo, int* exps) {
    __shared__ float shared[kThreads / 64];
    const int64_t row = blockIdx.x;
    const float* x = X + row * ldx;
    float top = 0.f;
    for (int64_t at = threadIdx.x * 8; at < k; at += kThreads * 8) {
        float v[8];
        load8<OZIMMU_F32>(x, at, k, vec, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
    }
    const int e0 = exponent_of(block_max(top, shared)) - kRowShift;
    if (threadIdx.x == 0) exps[row] = e0;
    const int64_t len = pad_to(k, 32);
    for (int64_t at = threadIdx.x * 8; at < len; at += kThreads * 8) {
        float v[8];
        load8<OZIMMU_F32>(x, at, k, vec, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ldexpf(v[e], -e0);
        store_slices8(out + row * ldo, at, v);
    }
}

// A padded copy of rows of 16-bit values.
__launch_bounds__(kThreads)
__global__ void pad_rows_kernel(int64_t rows, int64_t k, const unsigned short* X, int64_t ldx, bool vec, unsigned short* out, int64_t ldo, int tx, unsigned across) {
    const int64_t row = (int64_t)(blockIdx.x / across) * (kThreads / tx) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(blockIdx.x % across) * tx + threadIdx.x % tx) * 8;
    if (row >= rows || at >= ldo) return;
    const unsigned short* x = X + row * ldx;
    unsigned short r[8] = {};
    if (vec && at + 8 <= k)
        *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u*>(x + at);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < k) r[e] = x[at + e];
    *reinterpret_cast<v4u*>(out + row * ldo + at) = *reinterpret_cast<const v4u*>(r);
}

// Zeros (a product over an empty inner dimension).
template <typename T>
__launch_bounds__(kThreads)
__global__ void zero_rows_kernel(int64_t rows, int64_t cols, T* R, int64_t ld) {
    const int64_t row = blockIdx.x, at = (int64_t)blockIdx.y * kThreads + threadIdx.x;
    if (at < cols) R[row * ld + at] = T(0);
}

// exps[row] for the largest scale of a row of W (a workgroup per row), and exps[group] for the largest one of a group of
// columns (a workgroup per group): |s c| <= 8 s.
__launch_bounds__(kThreads)
__global__ void scale_exponents_kernel(int64_t len, const float* scales, int64_t step, int64_t next, int* exps) {
    __shared__ float shared[kThreads / 64];
    const float* s = scales + (int64_t)blockIdx.x * next;
    float top = 0.f;
    for (int64_t i = threadIdx.x; i < len; i += kThreads) top = fmaxf(top, fabsf(s[i * step]));
    const int e0 = exponent_of(block_max(top, shared)) + 3 - kRowShift;
    if (threadIdx.x == 0) exps[blockIdx.x] = e0;
}

// Rows of W in two slices under the row's exponent.
__launch_bounds__(kThreads)
__global__ void q4_slices_kernel(int64_t n, int64_t k, int group_log2, const uint8_t* codes, int64_t ldq, const float* scales, int64_t lds,
                                 unsigned short* out, int64_t ldo, const int* exps, int tx, unsigned across) {
    const int64_t row = (int64_t)(blockIdx.x / across) * (kThreads / tx) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(blockIdx.x % across) * tx + threadIdx.x % tx) * 8;
    if (row >= n || at >= pad_to(k, 32)) return;
    float x[8] = {};
    if (at < k) {
        const unsigned word = *reinterpret_cast<const unsigned*>(codes + row * ldq + at / 2);
        const float s = ldexpf(scales[row * lds + (at >> group_log2)], -exps[row]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < k ? s * code_value(word, e) : 0.f;
    }
    store_slices8(out + row * ldo, at, x);
}

// Columns of W as rows along n: a 64 x 64 tile through LDS. TYPE OZIMMU_F32: two slices under the exponent of the column's group.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void q4_transposed_kernel(int64_t n, int64_t k, int group_log2, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                                     unsigned short* out, int64_t ldo, const int* exps) {
    typedef Elem<TYPE> E;
    __shared__ float tile[64][65];
    const int64_t n0 = (int64_t)blockIdx.y * 64, k0 = (int64_t)blockIdx.x * 64;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int i = half * 32 + threadIdx.x / 8, j = threadIdx.x % 8 * 8;
        const int64_t row = n0 + i, at = k0 + j;
        float x[8] = {};
        if (row < n && at < k) {
            const unsigned word = *reinterpret_cast<const unsigned*>(codes + row * ldq + at / 2);
            float s = E::load(reinterpret_cast<const typename E::raw*>(scales)[row * lds + (at >> group_log2)]);
            if (TYPE == OZIMMU_F32) s = ldexpf(s, -exps[at >> group_log2]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s * code_value(word, e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) tile[j + e][i] = x[e];
    }
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int j = half * 32 + threadIdx.x / 8, i = threadIdx.x % 8 * 8;
        const int64_t col = k0 + j, at = n0 + i;
        if (col >= k || at >= pad_to(n, TYPE == OZIMMU_F32 ? 32 : 64)) continue;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = tile[j][i + e];
        if constexpr (TYPE == OZIMMU_F32)
            store_slices8(out + col * ldo, at, x);
        else
            store8<TYPE>(out + col * ldo, at, at + 8, true, x);
    }
}

// Threads along a row of `chunks` pieces: a power of two of at least 16 (the lanes of the largest group), so that short rows share a workgroup.
int threads_along(int64_t chunks) {
    int tx = 16;
    while (tx < kThreads && tx < chunks) tx *= 2;
    return tx;
}
// Workgroups over `rows` rows of `chunks` pieces, tx threads along a row: numbered along the rows, so that those that run together read memory in order (by columns first:
// 8192 x 8192 bf16 cut in 62 us).
unsigned across_of(int64_t chunks, int tx) { return (unsigned)((chunks + tx - 1) / tx); }
dim3 grid_for(int64_t rows, int64_t chunks, int tx) { return dim3((unsigned)((rows + kThreads / tx - 1) / (kThreads / tx)) * across_of(chunks, tx)); }
int log2_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

template <int TYPE, int STYPE>
hipError_t split_typed(int64_t n, int64_t k, int group, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, void* scales, int64_t lds, hipStream_t st) {
    const int64_t chunks = pad_to(k, group) / 8;
    const int tx = threads_along(chunks);
    const bool vec = rows_aligned16(W, ldw, sizeof(typename Elem<TYPE>::raw));
    const dim3 grid = grid_for((n + 1) / 2, chunks, tx);
    if (group == 32)
        q4_split_kernel<TYPE, STYPE, 32><<<grid, kThreads, 0, st>>>(n, k, W, ldw, vec, codes, ldq, scales, lds, tx, across_of(chunks, tx));
    else if (group == 64)
        q4_split_kernel<TYPE, STYPE, 64><<<grid, kThreads, 0, st>>>(n, k, W, ldw, vec, codes, ldq, scales, lds, tx, across_of(chunks, tx));
    else
        q4_split_kernel<TYPE, STYPE, 128><<<grid, kThreads, 0, st>>>(n, k, W, ldw, vec, codes, ldq, scales, lds, tx, across_of(chunks, tx));
    return hipGetLastError();
}
template <int TYPE>
hipError_t split_from(int64_t n, int64_t k, int group, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, void* scales, int stype, int64_t lds, hipStream_t st) {
    if (stype == OZIMMU_F32) return split_typed<TYPE, OZIMMU_F32>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
    if (stype == OZIMMU_BF16) return split_typed<TYPE, OZIMMU_BF16>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
    return split_typed<TYPE, OZIMMU_F16>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
}

template <int TYPE>
hipError_t expand_typed(int64_t n, int64_t k, int group, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds, void* W, int64_t ldw,
                        int64_t len, hipStream_t st) {
    const int64_t chunks = pad_to(len, 8) / 8;
    const int tx = threads_along(chunks);
    const bool vec = rows_aligned16(W, ldw, sizeof(typename Elem<TYPE>::raw));
    q4_expand_kernel<TYPE><<<grid_for(n, chunks, tx), kThreads, 0, st>>>(n, k, log2_of(group), codes, ldq, scales, lds, W, ldw, len, vec, tx, across_of(chunks, tx));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_zero_rows(int64_t rows, int64_t cols, void* R, int type, int64_t ld, hipStream_t st) {
    const dim3 grid((unsigned)rows, (unsigned)((cols + kThreads - 1) / kThreads));
    if (type == OZIMMU_F32)
        zero_rows_kernel<<<grid, kThreads, 0, st>>>(rows, cols, reinterpret_cast<float*>(R), ld);
    else
        zero_rows_kernel<<<grid, kThreads, 0, st>>>(rows, cols, reinterpret_cast<unsigned short*>(R), ld);
    return hipGetLastError();
}

hipError_t launch_q4_split(int64_t n, int64_t k, int group, const void* W, int type, int64_t ldw, uint8_t* codes, int64_t ldq,
                           void* scales, int scale_type, int64_t lds, hipStream_t st) {
    if (type == OZIMMU_F32) return split_from<OZIMMU_F32>(n, k, group, W, ldw, codes, ldq, scales, scale_type, lds, st);
    if (type == OZIMMU_BF16) return split_from<OZIMMU_BF16>(n, k, group, W, ldw, codes, ldq, scales, scale_type, lds, st);
    return split_from<OZIMMU_F16>(n, k, group, W, ldw, codes, ldq, scales, scale_type, lds, st);
}

hipError_t launch_q4_expand(int64_t n, int64_t k, int group, const uint8_t* codes, int64_t ldq, const void* scales, int type,
                            int64_t lds, void* W, int64_t ldw, hipStream_t st) {
    if (type == OZIMMU_F32) return expand_typed<OZIMMU_F32>(n, k, group, codes, ldq, scales, lds, W, ldw, k, st);
    if (type == OZIMMU_BF16) return expand_typed<OZIMMU_BF16>(n, k, group, codes, ldq, scales, lds, W, ldw, k, st);
    return expand_typed<OZIMMU_F16>(n, k, group, codes, ldq, scales, lds, W, ldw, k, st);
}

hipError_t launch_q4_operand(int64_t n, int64_t k, int group, const uint8_t* codes, int64_t ldq, const void* scales, int type,
                             int64_t lds, bool transposed, unsigned short* out, int64_t ldo, int* exps, hipStream_t st) {
    const int lg = log2_of(group);
    if (type == OZIMMU_F32) {
        const float* s = reinterpret_cast<const float*>(scales);
        const int64_t groups = (k + group - 1) / group;
        if (transposed)
            scale_exponents_kernel<<<dim3((unsigned)groups), kThreads, 0, st>>>(n, s, lds, 1, exps);
        else
            scale_exponents_kernel<<<dim3((unsigned)n), kThreads, 0, st>>>(groups, s, 1, lds, exps);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (transposed) {
        const dim3 grid((unsigned)((k + 63) / 64), (unsigned)((n + 63) / 64));
        if (type == OZIMMU_F32)
            q4_transposed_kernel<OZIMMU_F32><<<grid, kThreads, 0, st>>>(n, k, lg, codes, ldq, scales, lds, out, ldo, exps);
        else if (type == OZIMMU_BF16)
            q4_transposed_kernel<OZIMMU_BF16><<<grid, kThreads, 0, st>>>(n, k, lg, codes, ldq, scales, lds, out, ldo, exps);
        else
            q4_transposed_kernel<OZIMMU_F16><<<grid, kThreads, 0, st>>>(n, k, lg, codes, ldq, scales, lds, out, ldo, exps);
        return hipGetLastError();
    }
    if (type == OZIMMU_F32) {
        const int64_t chunks = pad_to(k, 32) / 8;
        const int tx = threads_along(chunks);
        q4_slices_kernel<<<grid_for(n, chunks, tx), kThreads, 0, st>>>(n, k, lg, codes, ldq, reinterpret_cast<const float*>(scales), lds, out, ldo, exps, tx, across_of(chunks, tx));
        return hipGetLastError();
    }
    const int64_t len = pad_to(k, 64);
    return type == OZIMMU_BF16 ? expand_typed<OZIMMU_BF16>(n, k, group, codes, ldq, scales, lds, out, ldo, len, st)
                               : expand_typed<OZIMMU_F16>(n, k, group, codes, ldq, scales, lds, out, ldo, len, st);
}

hipError_t launch_row_operand(int64_t rows, int64_t k, const void* X, int type, int64_t ldx, unsigned short* out, int64_t ldo,
                              int* exps, hipStream_t st) {
    if (type == OZIMMU_F32) {
        row_slices_kernel<<<dim3((unsigned)rows), kThreads, 0, st>>>(k, reinterpret_cast<const float*>(X), ldx, rows_aligned16(X, ldx, 4), out, ldo, exps);
    } else {
        const int64_t chunks = pad_to(k, 64) / 8;
        const int tx = threads_along(chunks);
        pad_rows_kernel<<<grid_for(rows, chunks, tx), kThreads, 0, st>>>(rows, k, reinterpret_cast<const unsigned short*>(X), ldx, rows_aligned16(X, ldx, 2), out, ldo, tx, across_of(chunks, tx));
    }
    return hipGetLastError();
}

}  // namespace ozimmu
