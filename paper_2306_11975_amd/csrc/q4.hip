// Weights in four bits: the cut, its inverse, and the operands of their matrix-core product (gfx950).
//
// Group g of row i: s = RN_T(RN_32(max |w| / 7)), c = RNE(w / s) clamped to [-8, 7], stored as c + 8, two to a byte, the even
// position in the low half; a row takes a multiple of 16 bytes (32 codes), what is beyond k stands for zero.
#include <algorithm>

#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;

// Eight consecutive values of a row, zero beyond the end.
template <int TYPE>
__device__ __forceinline__ void load8(const typename Elem<TYPE>::raw* row, int64_t at, int64_t len, float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    if (at + 8 <= len) {
        raw r[8];
        if constexpr (TYPE == OZIMMU_F32) {
            *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u_any*>(row + at);
            *reinterpret_cast<v4u*>(r + 4) = *reinterpret_cast<const v4u_any*>(row + at + 4);
        } else {
            *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u_any*>(row + at);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Elem<TYPE>::load(r[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < len ? Elem<TYPE>::load(row[at + e]) : 0.f;
    }
}
template <int TYPE>
__device__ __forceinline__ void store8(typename Elem<TYPE>::raw* row, int64_t at, int64_t len, const float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    raw r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = Elem<TYPE>::store(x[e]);
    if (at + 8 <= len) {
        *reinterpret_cast<v4u_any*>(row + at) = *reinterpret_cast<const v4u*>(r);
        if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u_any*>(row + at + 4) = *reinterpret_cast<const v4u*>(r + 4);
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

// The largest magnitude of eight values, as bits: those of |w| order like the values, NaN last, so that one that is there stays visible in
// the scale. As integers the largest is the largest positive value, as unsigned ones the largest negative one.
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

// The codes of eight weights as a word. w * (1/s), with a reciprocal that is off by a unit, is off the quotient by less than 2e-6; adding
// 1.5 * 2^23 rounds it to an integer, ties to even, whose low bits then stand in the low bits of the sum. That is the nearest integer to
// the quotient unless the product lies within 1e-5 of a border and is not the quotient itself (a tie, which weights of 8 bits often are):
// then the remainders decide, as they do where a scale that underflowed lets codes leave their range. (Both tests are asked of the
// wavefront: lane by lane, everyone would pay for them. 8192 x 8192 bf16: with the remainders always 62 us.)
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

// max |w| / 7, correctly rounded: the product with the rounded reciprocal, corrected by its remainder; very small ones, whose remainder
// would underflow, and infinities divided.
__device__ __forceinline__ float seventh(float top) {
    constexpr float r = 1.0f / 7.0f;
    const float q = top * r;
    const float exact = fmaf(fmaf(-7.0f, q, top), r, q);
    const bool plain = top > 1e-30f && top <= 3.4028234664e38f;
    if (__builtin_amdgcn_ballot_w64(!plain)) return plain ? exact : top / 7.0f;
    return exact;
}

// A thread cuts eight weights of two rows; the lanes of a group (GROUP / 8 of them, side by side) share its maximum. tx threads along a
// row. Memory-bound: the weights are read once, 16 or 32 bytes a lane, two rows on their way at a time.
template <int TYPE, int STYPE, int GROUP>
__launch_bounds__(kThreads)
__global__ void q4_split_kernel(int64_t n, int64_t k, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, void* scales,
                                int64_t lds, int tx, unsigned across, unsigned first) {
    typedef Elem<TYPE> E;
    typedef Elem<STYPE> S;
    constexpr int ROWS = 2;
    const int ty = kThreads / tx;
    const unsigned block = first + blockIdx.x;
    const int64_t row0 = (int64_t)(block / across) * (ROWS * ty) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(block % across) * tx + threadIdx.x % tx) * 8;
    float w[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) load8<TYPE>(reinterpret_cast<const typename E::raw*>(W) + min(row0 + i * ty, n - 1) * ldw, at, k, w[i]);
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
                                 void* W, int64_t ldw, int tx, unsigned across, unsigned first) {
    typedef Elem<TYPE> E;
    const unsigned block = first + blockIdx.x;
    const int64_t row = (int64_t)(block / across) * (kThreads / tx) + threadIdx.x / tx;
    const int64_t at = ((int64_t)(block % across) * tx + threadIdx.x % tx) * 8;
    if (row >= n || at >= k) return;
    const unsigned word = *reinterpret_cast<const unsigned*>(codes + row * ldq + at / 2);
    const float s = E::load(reinterpret_cast<const typename E::raw*>(scales)[row * lds + (at >> group_log2)]);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s * code_value(word, e);
    store8<TYPE>(reinterpret_cast<typename E::raw*>(W) + row * ldw, at, k, x);
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

// What the operands of a product are made of: weights (n x k) and rows of tokens (t x inner).
struct OperandArgs {
    int64_t n, k, ldq, lds;
    int group_log2;
    const uint8_t* codes;
    const void* scales;
    unsigned short* w_out;
    int* w_exps;
    int w_tx;
    unsigned w_across, w_blocks;
    int64_t t, inner, ldv, ld;   // ld: of both operands
    const void* V;
    unsigned short* v_out;
    int* v_exps;
    int v_tx;
    unsigned v_across;
    unsigned first;             // workgroup of the launch
};

// Rows of 32-bit values in two slices of fp16 under a power-of-two exponent per row; a workgroup per row, which it reads twice
// (the second time from the caches). NaN does not raise the maximum and stays in its place; so does an infinity.
__device__ __forceinline__ void row_slices(const OperandArgs& a, unsigned block, float* shared) {
    const int64_t row = block, k = a.inner;
    const float* x = reinterpret_cast<const float*>(a.V) + row * a.ldv;
    float top = 0.f;
    for (int64_t at = threadIdx.x * 8; at < k; at += kThreads * 8) {
        float v[8];
        load8<OZIMMU_F32>(x, at, k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
    }
    const int e0 = exponent_of(block_max(top, shared)) - kRowShift;
    if (threadIdx.x == 0) a.v_exps[row] = e0;
    const int64_t len = pad_to(k, 32);
    for (int64_t at = threadIdx.x * 8; at < len; at += kThreads * 8) {
        float v[8];
        load8<OZIMMU_F32>(x, at, k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ldexpf(v[e], -e0);
        store_slices8(a.v_out + row * a.ld, at, v);
    }
}

// A padded copy of rows of 16-bit values.
__device__ __forceinline__ void pad_rows(const OperandArgs& a, unsigned block) {
    const int64_t row = (int64_t)(block / a.v_across) * (kThreads / a.v_tx) + threadIdx.x / a.v_tx;
    const int64_t at = ((int64_t)(block % a.v_across) * a.v_tx + threadIdx.x % a.v_tx) * 8;
    if (row >= a.t || at >= a.ld) return;
    const unsigned short* x = reinterpret_cast<const unsigned short*>(a.V) + row * a.ldv;
    unsigned short r[8] = {};
    if (at + 8 <= a.inner)
        *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u_any*>(x + at);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < a.inner) r[e] = x[at + e];
    *reinterpret_cast<v4u*>(a.v_out + row * a.ld + at) = *reinterpret_cast<const v4u*>(r);
}

// The exponent of the largest of `len` scales, `step` apart: |s c| <= 8 s.
__device__ __forceinline__ int scale_exponent(const float* s, int64_t len, int64_t step, float* shared) {
    float top = 0.f;
    for (int64_t i = threadIdx.x; i < len; i += kThreads) top = fmaxf(top, fabsf(s[i * step]));
    return exponent_of(block_max(top, shared)) + 3 - kRowShift;
}

// Rows of W in two slices under an exponent per row, which every workgroup finds for itself: alone on a row its threads share the row's
// scales, else (rows of less than 2048 positions, at most 64 scales) sixteen lanes do.
__device__ __forceinline__ void q4_slices(const OperandArgs& a, unsigned block, float* shared) {
    const int64_t row = (int64_t)(block / a.w_across) * (kThreads / a.w_tx) + threadIdx.x / a.w_tx;
    const int64_t at = ((int64_t)(block % a.w_across) * a.w_tx + threadIdx.x % a.w_tx) * 8;
    const int64_t groups = (a.k + (1 << a.group_log2) - 1) >> a.group_log2;
    const float* scales = reinterpret_cast<const float*>(a.scales) + min(row, a.n - 1) * a.lds;
    int e0;
    if (a.w_tx == kThreads) {
        e0 = scale_exponent(scales, groups, 1, shared);
    } else {
        unsigned top = 0;
        for (int64_t i = threadIdx.x % 16; i < groups; i += 16) top = max(top, __float_as_uint(scales[i]) & 0x7fffffffu);
        e0 = exponent_of(__uint_as_float(max_of_lanes<16>(top))) + 3 - kRowShift;
    }
    if (row >= a.n || at >= pad_to(a.k, 32)) return;
    if (at == 0) a.w_exps[row] = e0;
    float x[8] = {};
    if (at < a.k) {
        const unsigned word = *reinterpret_cast<const unsigned*>(a.codes + row * a.ldq + at / 2);
        const float s = ldexpf(scales[at >> a.group_log2], -e0);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < a.k ? s * code_value(word, e) : 0.f;
    }
    store_slices8(a.w_out + row * a.ld, at, x);
}

// Rows of W rounded to 16 bits: what the matrix cores take of a weight at their full rate, and what an expanded weight is. (Scales on the
// sums instead, as the passes have them, take a second set of sums, which the product's tiles have no registers for; a second slice of
// every weight takes twice the products. Against results of exact weights, rounded: bf16 0.0021 and 0.0017 in the norm, fp16 0.00028 and
// 0.00021.)
template <int TYPE>
__device__ __forceinline__ void q4_rows(const OperandArgs& a, unsigned block) {
    typedef Elem<TYPE> E;
    const int64_t row = (int64_t)(block / a.w_across) * (kThreads / a.w_tx) + threadIdx.x / a.w_tx;
    const int64_t at = ((int64_t)(block % a.w_across) * a.w_tx + threadIdx.x % a.w_tx) * 8;
    if (row >= a.n || at >= a.ld) return;
    float x[8] = {};
    if (at < a.k) {
        const unsigned word = *reinterpret_cast<const unsigned*>(a.codes + row * a.ldq + at / 2);
        const float s = E::load(reinterpret_cast<const typename E::raw*>(a.scales)[row * a.lds + (at >> a.group_log2)]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < a.k ? s * code_value(word, e) : 0.f;
    }
    store8<TYPE>(a.w_out + row * a.ld, at, at + 8, x);
}

// Columns of W as rows along n, rounded to 16 bits or (OZIMMU_F32) in two slices under the exponent of the column's group: a tile of 64
// rows and WIDTH positions through LDS, where eight values of position l lie at place (their eighth) ^ (l / 8 % 8). A thread takes pairs of
// rows.
template <int TYPE, int WIDTH>
__device__ __forceinline__ void q4_columns(const OperandArgs& a, unsigned block, unsigned short* tile) {
    typedef Elem<TYPE> E;
    constexpr int kWords = WIDTH / 8, kPairs = kThreads / kWords, kTimes = 32 / kPairs;
    const int64_t n0 = (int64_t)(block / a.w_across) * 64, k0 = (int64_t)(block % a.w_across) * WIDTH;
    const int word_at = threadIdx.x % kWords;
    const int64_t at = k0 + 8 * word_at;
    unsigned words[kTimes][2];
    float scale[kTimes][2];
    const int lift = TYPE == OZIMMU_F32 && at < a.k ? -a.w_exps[at >> a.group_log2] : 0;
#pragma unroll
    for (int u = 0; u < kTimes; ++u)   // all requests before the first use; rows and positions that are not there repeat the last
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t row = min(n0 + 2 * (threadIdx.x / kWords + u * kPairs) + h, a.n - 1), l = min(at, (a.k - 1) & ~(int64_t)7);
            words[u][h] = *reinterpret_cast<const unsigned*>(a.codes + row * a.ldq + l / 2);
            scale[u][h] = E::load(reinterpret_cast<const typename E::raw*>(a.scales)[row * a.lds + (l >> a.group_log2)]);
        }
#pragma unroll
    for (int u = 0; u < kTimes; ++u) {
        const int i = 2 * (threadIdx.x / kWords + u * kPairs);
        unsigned word[2];
        float s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool here = n0 + i + h < a.n && at < a.k;
            word[h] = here ? words[u][h] : 0x88888888u;
            s[h] = !here ? 0.f : TYPE == OZIMMU_F32 ? ldexpf(scale[u][h], lift) : scale[u][h];
        }
        unsigned* to = reinterpret_cast<unsigned*>(tile + 8 * word_at * 64 + ((i >> 3) ^ (word_at & 7)) * 8 + (i & 7));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = s[0] * code_value(word[0], e), y = s[1] * code_value(word[1], e);
            if constexpr (TYPE == OZIMMU_F32) {
                unsigned short xh, xl, yh, yl;
                two_slices(x, xh, xl);
                two_slices(y, yh, yl);
                to[e * 32] = (unsigned)xh | (unsigned)yh << 16;
                to[e * 32 + WIDTH * 32] = (unsigned)xl | (unsigned)yl << 16;
            } else {
                to[e * 32] = (unsigned)E::store(x) | (unsigned)E::store(y) << 16;
            }
        }
    }
    __syncthreads();
    const int eighth = threadIdx.x % 8;
    const int64_t row = n0 + 8 * eighth;
    if (row >= pad_to(a.n, TYPE == OZIMMU_F32 ? 32 : 64)) return;
#pragma unroll
    for (int l = threadIdx.x / 8; l < WIDTH; l += kThreads / 8) {
        if (k0 + l >= a.k) break;
        const unsigned short* from = tile + l * 64 + (eighth ^ (l >> 3 & 7)) * 8;
        unsigned short* to = a.w_out + (k0 + l) * a.ld;
        if constexpr (TYPE == OZIMMU_F32) {
            to += (row >> 5) * 64 + (row & 31);
            *reinterpret_cast<v4u*>(to) = *reinterpret_cast<const v4u*>(from);
            *reinterpret_cast<v4u*>(to + 32) = *reinterpret_cast<const v4u*>(from + WIDTH * 64);
        } else {
            *reinterpret_cast<v4u*>(to + row) = *reinterpret_cast<const v4u*>(from);
        }
    }
}

// Both operands in one launch: the first workgroups make the weights', the others the tokens'.
// COLUMNS: the width of a tile of columns, 0: rows.
template <int TYPE, int COLUMNS>
__launch_bounds__(kThreads)
__global__ void operands_kernel(OperandArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned short tile[COLUMNS ? COLUMNS * 64 * (TYPE == OZIMMU_F32 ? 2 : 1) : 8];
    __shared__ float shared[kThreads / 64];
    const unsigned block = a.first + blockIdx.x;
    if (block < a.w_blocks) {
        if constexpr (COLUMNS != 0)
            q4_columns<TYPE, COLUMNS>(a, block, tile);
        else if constexpr (TYPE == OZIMMU_F32)
            q4_slices(a, block, shared);
        else
            q4_rows<TYPE>(a, block);
    } else if constexpr (TYPE == OZIMMU_F32) {
        row_slices(a, block - a.w_blocks, shared);
    } else {
        pad_rows(a, block - a.w_blocks);
    }
}

// The exponents of groups of columns, a workgroup per group (they stand before the columns' slices), beside the slices of the tokens.
__launch_bounds__(kThreads)
__global__ void group_exponents_kernel(OperandArgs a, unsigned groups) {
    __shared__ float shared[kThreads / 64];
    if (blockIdx.x < groups) {
        const int e0 = scale_exponent(reinterpret_cast<const float*>(a.scales) + blockIdx.x, a.n, a.lds, shared);
        if (threadIdx.x == 0) a.w_exps[blockIdx.x] = e0;
    } else {
        row_slices(a, blockIdx.x - groups, shared);
    }
}

// Zeros (a product over an empty inner dimension).
template <typename T>
__launch_bounds__(kThreads)
__global__ void zero_rows_kernel(int64_t rows, int64_t cols, T* R, int64_t ld) {
    const int64_t row = blockIdx.x, at = (int64_t)blockIdx.y * kThreads + threadIdx.x;
    if (at < cols) R[row * ld + at] = T(0);
}

// Threads along a row of `chunks` pieces: a power of two of at least 16 (the lanes of the largest group), so that short rows share a
// workgroup.
int threads_along(int64_t chunks) {
    int tx = 16;
    while (tx < kThreads && tx < chunks) tx *= 2;
    return tx;
}
// Workgroups over `rows` rows of `chunks` pieces, tx threads along a row: numbered along the rows, so that those that run together read
// memory in order (by columns first: 8192 x 8192 bf16 cut in 62 us).
unsigned across_of(int64_t chunks, int tx) { return (unsigned)((chunks + tx - 1) / tx); }
int64_t blocks_for(int64_t rows, int64_t chunks, int tx) { return (rows + kThreads / tx - 1) / (kThreads / tx) * (int64_t)across_of(chunks, tx); }
// A launch has fewer than 2^32 threads along its first dimension (of more the runtime starts a part, without an error), which 2^35 weights
// are beyond (4194304 x 8192, 16 GiB of codes): workgroups go out in launches of at most kMostBlocks, of a millisecond each.
// launch(workgroups, the first one's number).
constexpr int64_t kMostBlocks = 1 << 21;
template <class F>
hipError_t in_launches(int64_t blocks, F launch) {
    if (blocks > UINT32_MAX) return hipErrorInvalidValue;   // (2^43 weights)
    for (int64_t first = 0; first < blocks; first += kMostBlocks) launch(dim3((unsigned)std::min(kMostBlocks, blocks - first)), (unsigned)first);
    return hipGetLastError();
}
int log2_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

template <int TYPE, int STYPE>
hipError_t split_typed(int64_t n, int64_t k, int group, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, void* scales, int64_t lds, hipStream_t st) {
    const int64_t chunks = pad_to(k, group) / 8;
    const int tx = threads_along(chunks);
    const unsigned across = across_of(chunks, tx);
    return in_launches(blocks_for((n + 1) / 2, chunks, tx), [&](dim3 grid, unsigned first) {
        if (group == 32)
            q4_split_kernel<TYPE, STYPE, 32><<<grid, kThreads, 0, st>>>(n, k, W, ldw, codes, ldq, scales, lds, tx, across, first);
        else if (group == 64)
            q4_split_kernel<TYPE, STYPE, 64><<<grid, kThreads, 0, st>>>(n, k, W, ldw, codes, ldq, scales, lds, tx, across, first);
        else
            q4_split_kernel<TYPE, STYPE, 128><<<grid, kThreads, 0, st>>>(n, k, W, ldw, codes, ldq, scales, lds, tx, across, first);
    });
}
template <int TYPE>
hipError_t split_from(int64_t n, int64_t k, int group, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, void* scales, int stype, int64_t lds, hipStream_t st) {
    if (stype == OZIMMU_F32) return split_typed<TYPE, OZIMMU_F32>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
    if (stype == OZIMMU_BF16) return split_typed<TYPE, OZIMMU_BF16>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
    return split_typed<TYPE, OZIMMU_F16>(n, k, group, W, ldw, codes, ldq, scales, lds, st);
}

template <int TYPE>
hipError_t expand_typed(int64_t n, int64_t k, int group, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds, void* W, int64_t ldw,
                        hipStream_t st) {
    const int64_t chunks = pad_to(k, 8) / 8;
    const int tx = threads_along(chunks);
    return in_launches(blocks_for(n, chunks, tx), [&](dim3 grid, unsigned first) {
        q4_expand_kernel<TYPE><<<grid, kThreads, 0, st>>>(n, k, log2_of(group), codes, ldq, scales, lds, W, ldw, tx, across_of(chunks, tx), first);
    });
}

template <int TYPE>
void launch_operands_typed(const OperandArgs& a, dim3 grid, int width, hipStream_t st) {
    if (width == 0)
        operands_kernel<TYPE, 0><<<grid, kThreads, 0, st>>>(a);
    else if (width == 64)
        operands_kernel<TYPE, 64><<<grid, kThreads, 0, st>>>(a);
    else
        operands_kernel<TYPE, TYPE == OZIMMU_F32 ? 128 : 256><<<grid, kThreads, 0, st>>>(a);
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
    if (type == OZIMMU_F32) return expand_typed<OZIMMU_F32>(n, k, group, codes, ldq, scales, lds, W, ldw, st);
    if (type == OZIMMU_BF16) return expand_typed<OZIMMU_BF16>(n, k, group, codes, ldq, scales, lds, W, ldw, st);
    return expand_typed<OZIMMU_F16>(n, k, group, codes, ldq, scales, lds, W, ldw, st);
}

hipError_t launch_operands(int64_t t, int64_t n, int64_t k, int group, int type, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds, bool columns,
                           unsigned short* w_out, int* w_exps, const void* V, int64_t ldv, unsigned short* v_out, int* v_exps, int64_t ld, hipStream_t st) {
    OperandArgs a{};
    a.n = n;
    a.k = k;
    a.ldq = ldq;
    a.lds = lds;
    a.group_log2 = log2_of(group);
    a.codes = codes;
    a.scales = scales;
    a.w_out = w_out;
    a.w_exps = w_exps;
    a.t = t;
    a.inner = columns ? n : k;
    a.ldv = ldv;
    a.ld = ld;
    a.V = V;
    a.v_out = v_out;
    a.v_exps = v_exps;
    const bool f32 = type == OZIMMU_F32;
    // Wide tiles read and write whole lines (8192 x 4096 in 16 bits 24 us with 64 positions, 18 with 256); narrow ones are more workgroups
    // where there are few.
    const int most = f32 ? 128 : 256;
    const int width = (n + 63) / 64 * ((k + most - 1) / most) >= 1024 ? most : 64;
    int64_t w_blocks, v_blocks = 0;
    if (columns) {
        a.w_across = (unsigned)((k + width - 1) / width);
        w_blocks = (n + 63) / 64 * (int64_t)a.w_across;
    } else {
        const int64_t chunks = pad_to(k, f32 ? 32 : 64) / 8;
        a.w_tx = threads_along(chunks);
        a.w_across = across_of(chunks, a.w_tx);
        w_blocks = blocks_for(n, chunks, a.w_tx);
    }
    a.w_blocks = (unsigned)w_blocks;
    if (v_out && f32) {
        v_blocks = t;
    } else if (v_out) {
        a.v_tx = threads_along(ld / 8);
        a.v_across = across_of(ld / 8, a.v_tx);
        v_blocks = blocks_for(t, ld / 8, a.v_tx);
    }
    if (columns && f32) {
        const unsigned groups = (unsigned)((k + group - 1) / group);
        group_exponents_kernel<<<dim3(groups + (unsigned)v_blocks), kThreads, 0, st>>>(a, groups);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        v_blocks = 0;
    }
    return in_launches(w_blocks + v_blocks, [&](dim3 grid, unsigned first) {
        a.first = first;
        if (f32)
            launch_operands_typed<OZIMMU_F32>(a, grid, columns ? width : 0, st);
        else if (type == OZIMMU_BF16)
            launch_operands_typed<OZIMMU_BF16>(a, grid, columns ? width : 0, st);
        else
            launch_operands_typed<OZIMMU_F16>(a, grid, columns ? width : 0, st);
    });
}

}  // namespace ozimmu
