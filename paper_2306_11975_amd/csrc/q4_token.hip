// Y = X W^T for one token or two and weights in four bits: one pass over the codes on the vector units, no workspace (gfx950).
//
// What bounds it is reading the codes, half a byte for 2 T operations, so the loads come first: a row's codes are read along the row, 16
// bytes a lane, 16 lanes side by side, and four rows a load. (The matrix cores want neighbouring lanes in different rows, and such a load
// looks up a line for every lane: q4_few.hip.) A lane's 32 positions lie in one group; it multiplies them itself, and lanes add up at the
// end, within rows of sixteen. The tokens' piece of 512 positions is loaded once a wavefront, eight values a lane, and goes through LDS to
// the lanes that need it. A wavefront takes 4 R rows and every W-th piece; the W of a workgroup add their parts up in LDS.
//
// A code's sixteenth is one conversion (v_cvt_off_f32_i4, exact), a product one fma in 32 bits; the scale goes on a lane's sum of 32
// products. Two and a quarter instructions a code with one token: 4 us of the vector units for 16384 x 8192, beside the 17.3 us that its 71
// MB take (4.1 TB/s). Measured (us; on the matrix cores -> here, one token, bf16): 2048 x 2048 3.9 -> 2.9, 1024 x 8192 7.7 -> 3.6, 2048 x
// 16384 14.5 -> 6.8, 8192 x 4096 7.4 -> 5.4, 11008 x 4096 12.2 -> 6.8, 16384 x 8192 20.6 -> 17.3, 8 x 65536 34.3 -> 10.4; 32 bits 2048 x
// 2048 5.4 -> 2.9, 16384 x 8192 36.4 -> 15.8.
#include <type_traits>

#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kPiece = 512;   // positions: 16 lanes of 32

template <int CTRL>
__device__ __forceinline__ float plus_lane(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// the sum over 16 neighbouring lanes
__device__ __forceinline__ float sum16(float x) {
    x = plus_lane<0xb1>(x);    // lane ^ 1
    x = plus_lane<0x4e>(x);    // lane ^ 2
    x = plus_lane<0x141>(x);   // the other four of eight
    return plus_lane<0x140>(x);   // the other eight of sixteen
}

template <int TYPE, int T, int R, int W>
__launch_bounds__(W * 64)
__global__ void q4_token_kernel(int t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                                int group_log2, void* Y, int64_t ldy) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    constexpr int XV = TYPE == OZIMMU_F32 ? 2 : 1;   // 16-byte loads of eight values
    __shared__ __attribute__((aligned(16))) v4u tokens[W][T][XV][64];
    __shared__ float part[W][T][4 * R];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (4 * R);
    const int64_t pieces = (k + kPiece - 1) / kPiece;
    const int mine = wave < pieces ? (int)((pieces - wave + W - 1) / W) : 0;
    const int in_piece = lane % 16 * 32;
    // scalar bases, 32-bit offsets (rows are at most OZIMMU_MAX_LD apart); rows that are not there repeat the last one
    const uint8_t* qb = codes + n0 * ldq;
    const raw* sb = reinterpret_cast<const raw*>(scales) + n0 * lds;
    unsigned qo[R], so[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const unsigned row = (unsigned)min((int64_t)(4 * i + lane / 16), n - 1 - n0);
        qo[i] = row * (unsigned)ldq;
        so[i] = row * (unsigned)lds;
    }
    struct Step {
        v4u x[T][XV];   // eight values of the piece's 512: 8 lane .. + 7
        v4u w[R];
        raw s[R];
    };
    auto load = [&](int step, Step& to) {
        const int64_t piece = ((int64_t)step * W + wave) * kPiece, at = piece + in_piece, xat = piece + 8 * lane;
        const bool here = at < k;   // what codes a lane beyond the row reads does not matter: its tokens and its scale are zeros
        const int64_t from = here ? at : 0;
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const raw* xb = reinterpret_cast<const raw*>(X) + min(i, t - 1) * ldx;
            if (xat + 8 <= k) {
#pragma unroll
                for (int v = 0; v < XV; ++v) to.x[i][v] = reinterpret_cast<const v4u_any*>(xb + xat)[v];
            } else {
                raw r[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const raw y = xb[min(xat + e, k - 1)];
                    r[e] = xat + e < k ? y : raw(0);
                }
#pragma unroll
                for (int v = 0; v < XV; ++v) to.x[i][v] = reinterpret_cast<const v4u*>(r)[v];
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            to.w[i] = *reinterpret_cast<const v4u*>(qb + from / 2 + qo[i]);
            const raw s = sb[(from >> group_log2) + so[i]];
            to.s[i] = here ? s : raw(0);
        }
    };
    float total[T][R];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) total[i][r] = 0.f;
    auto multiply = [&](const Step& s) {
        // the tokens to the lanes that multiply them: chunk c of eight values, from lane c, is word c % 4 of lane c / 4 (of sixteen), at
        // place 16 (c % 4) + c / 4
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int v = 0; v < XV; ++v) tokens[wave][i][v][lane % 4 * 16 + lane / 4] = s.x[i][v];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float sum[T][R];
#pragma unroll
        for (int j = 0; j < 4; ++j) {   // a word of eight codes
            float x[T][8];
#pragma unroll
            for (int i = 0; i < T; ++i) {
                v4u y[XV];
#pragma unroll
                for (int v = 0; v < XV; ++v) y[v] = tokens[wave][i][v][16 * j + lane % 16];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (TYPE == OZIMMU_F32)
                        x[i][e] = __uint_as_float(y[e / 4][e % 4]);
                    else
                        x[i][e] = E::load((raw)(y[0][e / 2] >> (16 * (e % 2))));
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const unsigned word = s.w[r][j] ^ 0x88888888u, high = word >> 4;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float c = __builtin_amdgcn_cvt_off_f32_i4((int)((e % 2 ? high : word) >> (8 * (e / 2))));
#pragma unroll
                    for (int i = 0; i < T; ++i) sum[i][r] = j == 0 && e == 0 ? c * x[i][e] : fmaf(c, x[i][e], sum[i][r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float f = E::load(s.s[r]);
#pragma unroll
            for (int i = 0; i < T; ++i) total[i][r] = fmaf(f, sum[i][r], total[i][r]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // (the places are written again)
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    Step s[2];
    if (mine > 0) load(0, s[0]);
    for (int step0 = 0; step0 < mine; step0 += 2) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int step = step0 + d;
            if (step >= mine) break;
            if (step + 1 < mine) load(step + 1, s[d ^ 1]);
            multiply(s[d]);
        }
    }
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float sum = sum16(total[i][r]);
            if (lane % 16 == 0) part[wave][i][4 * r + lane / 16] = sum;
        }
    __syncthreads();
    for (int at = threadIdx.x; at < T * 4 * R; at += W * 64) {
        const int i = at / (4 * R), r = at % (4 * R);
        if (i >= t || n0 + r >= n) continue;
        float sum = part[0][i][r];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += part[w][i][r];
        reinterpret_cast<raw*>(Y)[(int64_t)i * ldy + n0 + r] = E::store(16.f * sum);   // (the codes' sixteenths)
    }
}

template <int TYPE, int T, int R, int W>
hipError_t launch_rows(int64_t t, int64_t n, int64_t k, int group, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                       void* Y, int64_t ldy, hipStream_t st) {
    q4_token_kernel<TYPE, T, R, W><<<dim3((unsigned)((n + 4 * R - 1) / (4 * R))), W * 64, 0, st>>>((int)t, n, k, X, ldx, codes, ldq, scales, lds,
                                                                                                    group == 32 ? 5 : group == 64 ? 6 : 7, Y, ldy);
    return hipGetLastError();
}
// More rows to a wavefront: the tokens go through LDS less often; more workgroups and wavefronts along k: more codes on their way. (One
// token, bf16, R and W 1 and 8, 2 and 8, 2 and 4: 1024 x 8192 3.6, 4.0, 4.7 us; 4096 x 4096 4.4, 3.8, 4.1; 11008 x 4096 7.9, 6.9, 6.8;
// 16384 x 8192 in 32 bits 20.0, 18.0, 15.8.)
template <int TYPE, int T>
hipError_t launch_typed(int64_t t, int64_t n, int64_t k, int group, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    if (n >= 8192) return launch_rows<TYPE, T, 2, 4>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    if (n >= 2048) return launch_rows<TYPE, T, 2, 8>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    return launch_rows<TYPE, T, 1, 8>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
}

}  // namespace

hipError_t launch_q4_token(int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes, int64_t ldq,
                           const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st) {
    auto go = [&](auto two) {
        constexpr int T = decltype(two)::value;
        if (type == OZIMMU_F32) return launch_typed<OZIMMU_F32, T>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
        if (type == OZIMMU_BF16) return launch_typed<OZIMMU_BF16, T>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
        return launch_typed<OZIMMU_F16, T>(t, n, k, group, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    };
    return t == 1 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 2>{});
}

}  // namespace ozimmu
