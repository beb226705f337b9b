// Y = X W^T for few tokens and weights in four bits: one pass over the codes, no workspace (gfx950).
//
// What bounds it is reading the codes; the sums go to the matrix cores (v_mfma_f32_16x16x32) although most of their rows stay empty with
// one token, because the vector units have their hands full making 16-bit operands of the codes. A wavefront takes 16 NT rows of
// W and a part of k; the wavefronts of a workgroup share the rows and add their parts up in LDS.
//
// A step is 128 positions. A lane holds rows lane % 16 of each 16 x 128 block of codes and quarter lane / 16 of every group (so that an
// MFMA adds up positions of one group only); its word j is MFMA j's operand, and the tokens' operand is loaded from the same positions.
//
// Codes to 16-bit values: the four bits of c + 8 go into the mantissa of 16.0 (one shift, one and-or for two codes), which
// gives 16 + (c + 8) exactly. The 24 too much is taken out by the matrix cores: the sums start from the tokens' product with a
// constant operand of -24, formed once for all rows of the wavefront. So a group's sum is that of x (c + 24) and x (-24) in 32 bits:
// against the terms alone it loses three bits of 24, which results of 8 or 11 bits do not see. 32-bit tokens are
// cut into three bf16 (exactly) and multiplied by exact codes, without the detour.
// The scale of a group is applied to its sum in 32 bits.
#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kWaves = 8;

// The operand of eight tokens' values is paired (0, 4), (1, 5), (2, 6), (3, 7) to match the codes' pairs.
__device__ __forceinline__ v4u pair_by_four(const v4u& x) {
    v4u r;
    r[0] = __builtin_amdgcn_perm(x[2], x[0], 0x05040100u);
    r[1] = __builtin_amdgcn_perm(x[2], x[0], 0x07060302u);
    r[2] = __builtin_amdgcn_perm(x[3], x[1], 0x05040100u);
    r[3] = __builtin_amdgcn_perm(x[3], x[1], 0x07060302u);
    return r;
}

// 16 + (c + 8) of the codes (0, 4), (1, 5), (2, 6), (3, 7) of a word
template <bool BF16>
__device__ __forceinline__ v4u offset_codes(unsigned w) {
    v4u r;
    if constexpr (BF16) {
        constexpr unsigned mask = 0x00780078u, one = 0x41804180u;
        r[0] = ((w << 3) & mask) | one;
        r[1] = ((w >> 1) & mask) | one;
        r[2] = ((w >> 5) & mask) | one;
        r[3] = ((w >> 9) & mask) | one;
    } else {
        constexpr unsigned mask = 0x03c003c0u, one = 0x4c004c00u;
        r[0] = ((w << 6) & mask) | one;
        r[1] = ((w << 2) & mask) | one;
        r[2] = ((w >> 2) & mask) | one;
        r[3] = ((w >> 6) & mask) | one;
    }
    return r;
}
// the codes themselves as bf16
__device__ __forceinline__ v4u exact_codes(unsigned w) {
    v4u r = offset_codes<true>(w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(r[i] << 16) - 24.f, hi = __uint_as_float(r[i] & 0xffff0000u) - 24.f;
        r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
    return r;
}

template <int TYPE>
struct Tokens {
    static constexpr int kPieces = TYPE == OZIMMU_F32 ? 3 : 1;
    v4u piece[kPieces];
};

template <int TYPE>
__device__ __forceinline__ Tokens<TYPE> load_tokens(const typename Elem<TYPE>::raw* x, int64_t at, int64_t k, bool here, bool vec) {
    typedef typename Elem<TYPE>::raw raw;
    raw r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = raw(0);
    if (here) {
        if (vec && at + 8 <= k) {
            *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u*>(x + at);
            if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u*>(r + 4) = *reinterpret_cast<const v4u*>(x + at + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < k) r[e] = x[at + e];
        }
    }
    Tokens<TYPE> t;
    if constexpr (TYPE == OZIMMU_F32) {
        unsigned a[8], b[8], c[8];   // the upper 8 bits of the significand, the next 8, and what is left
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] = __float_as_uint(r[e]) & 0xffff0000u;
            const float rest = r[e] - __uint_as_float(a[e]);
            b[e] = __float_as_uint(rest) & 0xffff0000u;
            c[e] = __float_as_uint(rest - __uint_as_float(b[e]));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t.piece[0][i] = __builtin_amdgcn_perm(a[i + 4], a[i], 0x07060302u);
            t.piece[1][i] = __builtin_amdgcn_perm(b[i + 4], b[i], 0x07060302u);
            t.piece[2][i] = __builtin_amdgcn_perm(c[i + 4], c[i], 0x07060302u);
        }
    } else {
        t.piece[0] = pair_by_four(*reinterpret_cast<const v4u*>(r));
    }
    return t;
}

template <int TYPE, int GROUP, int NT>
__launch_bounds__(kWaves * 64)
__global__ void q4_few_kernel(int t, int64_t n, int64_t k, const void* X, int64_t ldx, bool vec, const uint8_t* codes, int64_t ldq, const void* scales,
                              int64_t lds, void* Y, int64_t ldy) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    constexpr bool BF16 = TYPE != OZIMMU_F16;
    constexpr int GW = GROUP / 32, GROUPS = 128 / GROUP;   // words of a lane per group, groups of a step
    constexpr int DEPTH = 4;                               // steps whose codes are on their way at a time
    __shared__ float part[kWaves][16][16 * NT + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
    const int steps = (int)((k + 127) / 128);
    const int begin = (int)((int64_t)steps * wave / kWaves), end = (int)((int64_t)steps * (wave + 1) / kWaves);
    const int quarter = lane >> 4, token = lane & 15;
    const bool here = token < t;
    const raw* x = reinterpret_cast<const raw*>(X) + (int64_t)(here ? token : 0) * ldx;
    const uint8_t* q[NT];
    const raw* s[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t row = min(n0 + 16 * i + (lane & 15), n - 1);
        q[i] = codes + row * ldq;
        s[i] = reinterpret_cast<const raw*>(scales) + row * lds;
    }
    const int64_t row_bytes = pad_to(k, 32) / 2;
    const int groups = (int)((k + GROUP - 1) / GROUP);

    auto load_codes = [&](int step, unsigned (&w)[NT][4], raw (&sc)[NT][GROUPS]) {
#pragma unroll
        for (int h = 0; h < GROUPS; ++h) {
            const int64_t at = (int64_t)step * 64 + h * (GROUP / 2) + quarter * (GROUP / 8);   // bytes
            const bool in = at < row_bytes;
            const int g = min(step * GROUPS + h, groups - 1);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                // (where a quarter lies beyond the row its tokens are zeros, and any finite code will do)
                if constexpr (GW == 4) {
                    // a row's last 16 bytes can be this quarter's only in full: rows take a multiple of 16 bytes
                    const v4u v = in ? *reinterpret_cast<const v4u*>(q[i] + at) : v4u{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[i][j] = v[j];
                } else if constexpr (GW == 2) {
                    const v2u v = in ? *reinterpret_cast<const v2u*>(q[i] + at) : v2u{0, 0};
                    w[i][2 * h] = v[0];
                    w[i][2 * h + 1] = v[1];
                } else {
                    w[i][h] = in ? *reinterpret_cast<const unsigned*>(q[i] + at) : 0u;
                }
                sc[i][h] = s[i][g];
            }
        }
    };

    v4f total[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) total[i] = v4f{0.f, 0.f, 0.f, 0.f};
    const unsigned minus = BF16 ? 0xc1c0c1c0u : 0xce00ce00u;   // -24, twice
    const v4u minus24 = {minus, minus, minus, minus};

    auto multiply = [&](int step, const unsigned (&w)[NT][4], const raw (&sc)[NT][GROUPS]) {
#pragma unroll
        for (int h = 0; h < GROUPS; ++h) {
            v4f sum[NT];
            v4f start = v4f{0.f, 0.f, 0.f, 0.f};
            Tokens<TYPE> xs[GW];
#pragma unroll
            for (int j = 0; j < GW; ++j) {
                const int64_t at = (int64_t)step * 128 + h * GROUP + quarter * (GROUP / 4) + 8 * j;
                xs[j] = load_tokens<TYPE>(x, at, k, here, vec);
                if constexpr (TYPE != OZIMMU_F32) start = mfma_half<BF16>(xs[j].piece[0], minus24, start);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                sum[i] = start;
#pragma unroll
                for (int j = 0; j < GW; ++j) {
                    const unsigned word = w[i][GW * h + j];
                    if constexpr (TYPE == OZIMMU_F32) {
                        const v4u c = exact_codes(word);
#pragma unroll
                        for (int p = 2; p >= 0; --p) sum[i] = mfma_half<true>(xs[j].piece[p], c, sum[i]);
                    } else {
                        sum[i] = mfma_half<BF16>(xs[j].piece[0], offset_codes<BF16>(word), sum[i]);
                    }
                }
                const float f = E::load(sc[i][h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) total[i][e] = fmaf(f, sum[i][e], total[i][e]);
            }
        }
    };

    unsigned w[DEPTH][NT][4];
    raw sc[DEPTH][NT][GROUPS];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (begin + d < end) load_codes(begin + d, w[d], sc[d]);
    for (int step = begin; step < end; step += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (step + d < end) multiply(step + d, w[d], sc[d]);
            if (step + d + DEPTH < end) load_codes(step + d + DEPTH, w[d], sc[d]);
        }
    }

    // lane: tokens 4 quarter .. + 3, rows lane % 16
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][4 * quarter + e][16 * i + (lane & 15)] = total[i][e];
    __syncthreads();
    for (int at = threadIdx.x; at < t * 16 * NT; at += kWaves * 64) {
        const int tok = at / (16 * NT), col = at % (16 * NT);
        if (n0 + col >= n) continue;
        float sum = part[0][tok][col];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += part[i][tok][col];
        reinterpret_cast<raw*>(Y)[(int64_t)tok * ldy + n0 + col] = E::store(sum);
    }
}

template <int TYPE, int GROUP>
hipError_t launch_typed(int64_t t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    const bool vec = rows_aligned16(X, ldx, sizeof(typename Elem<TYPE>::raw));
    if (n >= 32 * 256)
        q4_few_kernel<TYPE, GROUP, 2><<<dim3((unsigned)((n + 31) / 32)), kWaves * 64, 0, st>>>((int)t, n, k, X, ldx, vec, codes, ldq, scales, lds, Y, ldy);
    else
        q4_few_kernel<TYPE, GROUP, 1><<<dim3((unsigned)((n + 15) / 16)), kWaves * 64, 0, st>>>((int)t, n, k, X, ldx, vec, codes, ldq, scales, lds, Y, ldy);
    return hipGetLastError();
}
template <int TYPE>
hipError_t launch_grouped(int64_t t, int64_t n, int64_t k, int group, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales,
                          int64_t lds, void* Y, int64_t ldy, hipStream_t st) {
    if (group == 32) return launch_typed<TYPE, 32>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    if (group == 64) return launch_typed<TYPE, 64>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    return launch_typed<TYPE, 128>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
}

}  // namespace

hipError_t launch_q4_few(int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes,
                         int64_t ldq, const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st) {
    if (type == OZIMMU_F32) return launch_grouped<OZIMMU_F32>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    if (type == OZIMMU_BF16) return launch_grouped<OZIMMU_BF16>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    return launch_grouped<OZIMMU_F16>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
}

}  // namespace ozimmu
