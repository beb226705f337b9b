// Y = X W^T for few tokens and weights in four bits: a pass over the codes for every 16 or 32 tokens, no workspace (gfx950).
//
// What bounds it is reading the codes, and the tokens again for every 16 NT rows of them; the sums go to the matrix cores
// (v_mfma_f32_16x16x32) although most of their rows stay empty with few tokens, because the vector units have their hands full making
// 16-bit operands of the codes. A wavefront takes 16 NT rows of W, 16 TT tokens and every W-th step of k; the W wavefronts of a
// workgroup share the rows and add their parts up in LDS.
//
// A step is 128 positions. Memory is read along the rows, 16 lanes to 256 bytes of a token's row, four lanes to 64 of a row's codes, and
// goes through LDS (a region for every wavefront, no barrier) into the operands' order; loads in that order, neighbouring lanes in
// different rows, look up a line for every lane (16 tokens, bf16, 16384 x 8192 26.8 us where these take 19.6; 32 tokens 51.8 and 30.5;
// rows of tokens at odd places, 387 x 10575, 58 and 12). A lane's operand of the codes is 16 bytes, 32 positions, of row lane % 16. An
// MFMA adds up positions of one group only: in groups of 64 and 32 the quarters of a wavefront (lane / 16) first exchange words
// (v_permlane32_swap, v_permlane16_swap), so that word j of every lane belongs to one group, and is MFMA j's operand. The tokens' operand
// is read from the same positions.
//
// Codes become 16-bit values exactly, so that products are exact and a sum's error goes by its terms: a value far above the others under
// a code of zero adds nothing to it. bf16: the conversion from four signed bits gives a code's sixteenth in 32 bits, whose upper half is
// all of it; two halves make a word of the operand, and the result is multiplied by 16. fp16: the four bits of c + 8 go into the mantissa
// of 1024, and a packed addition takes 1032 away. (With the offset left in and the tokens' product with it taken off the sums, an MFMA
// more, the roundings of both sums stay behind: fp16 tokens with a value of 6e4 over a code of zero were off by several roundings of the
// result. 64 tokens, 16384 x 8192, groups of 32, 65.5 us so, 60.9 here.)
// 32-bit tokens are cut into three bf16 (exactly), three MFMAs. The scale of a group is applied to its sum in 32 bits.
#include "half_common.h"

namespace ozimmu {
namespace {

// Eight fp16 tokens paired (0, 4), (1, 5), (2, 6), (3, 7) to match the codes' pairs.
__device__ __forceinline__ v4u pair_by_four(const v4u& x) {
    v4u r;
    r[0] = __builtin_amdgcn_perm(x[2], x[0], 0x05040100u);
    r[1] = __builtin_amdgcn_perm(x[2], x[0], 0x07060302u);
    r[2] = __builtin_amdgcn_perm(x[3], x[1], 0x05040100u);
    r[3] = __builtin_amdgcn_perm(x[3], x[1], 0x07060302u);
    return r;
}

// The two constants of fp16 codes in registers of their own (v_and_or_b32 takes one scalar and no two literals), hidden from the
// optimiser, which would turn them back into literals and take two instructions.
struct CodeBits {
    unsigned mask, one;
    static __device__ __forceinline__ CodeBits of() {
        CodeBits c;
        asm("s_mov_b32 %0, 0x000f000f\n\tv_mov_b32 %1, 0x64006400" : "=s"(c.mask), "=v"(c.one));
        return c;
    }
};
// The codes of a word in fp16, (0, 4), (1, 5), (2, 6), (3, 7), exactly: 1024 + (c + 8) less 1032.
__device__ __forceinline__ v4u codes_f16(unsigned w, const CodeBits& b) {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h less = {(_Float16)-1032.f, (_Float16)-1032.f};
    v4u r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(unsigned, __builtin_bit_cast(v2h, ((w >> (4 * i)) & b.mask) | b.one) + less);
    return r;
}
// The sixteenth of the code in the low half of byte BYTE. (In assembly for the choice of a byte: the compiler shifts ahead of most
// conversions instead, up to five instructions a word; 16 tokens, 16384 x 8192, 21.0 us against 19.6.)
template <int BYTE>
__device__ __forceinline__ float sixteenth(unsigned w) {
    float x;
    if constexpr (BYTE == 0)
        x = __builtin_amdgcn_cvt_off_f32_i4((int)w);
    else if constexpr (BYTE == 1)
        asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(x) : "v"(w));
    else if constexpr (BYTE == 2)
        asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(x) : "v"(w));
    else
        asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(x) : "v"(w));
    return x;
}
// The codes' sixteenths in bf16, in order, exactly: the conversion from four signed bits gives them in 32 bits, and they fit the upper
// half.
__device__ __forceinline__ v4u sixteenths_bf16(unsigned w) {
    w ^= 0x88888888u;
    const unsigned high = w >> 4;
    v4u r;
    static_for<0, 4>([&](auto byte) {
        constexpr int i = decltype(byte)::value;
        r[i] = __builtin_amdgcn_perm(__float_as_uint(sixteenth<i>(high)), __float_as_uint(sixteenth<i>(w)), 0x07060302u);
    });
    return r;
}

// Eight tokens' values as loaded, and as operands: one piece, or three bf16 pieces of 32-bit values.
template <int TYPE>
struct Raw {
    v4u v[TYPE == OZIMMU_F32 ? 2 : 1];
};
template <int TYPE>
struct Operand {
    static constexpr int kPieces = TYPE == OZIMMU_F32 ? 3 : 1;
    v4u piece[kPieces];
};
template <int TYPE>
__device__ __forceinline__ Operand<TYPE> operand(const Raw<TYPE>& r) {
    Operand<TYPE> t;
    if constexpr (TYPE == OZIMMU_F32) {
        unsigned a[8], b[8], c[8];   // the upper 8 bits of the significand, the next 8, and what is left
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned bits = r.v[e >> 2][e & 3];
            a[e] = bits & 0xffff0000u;
            const float rest = __uint_as_float(bits) - __uint_as_float(a[e]);
            b[e] = __float_as_uint(rest) & 0xffff0000u;
            c[e] = __float_as_uint(rest - __uint_as_float(b[e]));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t.piece[0][i] = __builtin_amdgcn_perm(a[2 * i + 1], a[2 * i], 0x07060302u);
            t.piece[1][i] = __builtin_amdgcn_perm(b[2 * i + 1], b[2 * i], 0x07060302u);
            t.piece[2][i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
        }
    } else if constexpr (TYPE == OZIMMU_BF16) {
        t.piece[0] = r.v[0];
    } else {
        t.piece[0] = pair_by_four(r.v[0]);
    }
    return t;
}

template <int TYPE, int GROUP, int NT, int TT, int W>
__launch_bounds__(W * 64)
__global__ void q4_few_kernel(int t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales,
                              int64_t lds, void* Y, int64_t ldy) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    constexpr bool BF16 = TYPE != OZIMMU_F16;
    constexpr int GW = GROUP / 32, GROUPS = 128 / GROUP;   // words of a lane per group, groups of a step
    constexpr int DEPTH = 2;                 // steps whose codes are on their way at a time
    constexpr int kRow = 16 * NT + 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_bytes[];
    float* const part = reinterpret_cast<float*>(lds_bytes);   // [wave][token][row], when the walk is over
    constexpr int kTokenRow = 128 * sizeof(raw), kCodes = NT * 1024;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
    const int t0 = blockIdx.y * (16 * TT);
    // Whole steps are dealt to the wavefronts in turn (together they read lines in full); the last wavefront takes what is left of the row
    // beyond them too.
    const int full = (int)(k / 128);
    const int mine = (full - wave + W - 1) / W;
    const int quarter = lane >> 4;
    // position of word j of group h in a step, for this lane (the exchange between quarters below)
    const int at_quarter = GROUP == 128 ? 32 * quarter : GROUP == 64 ? 32 * (quarter & 1) + 16 * (quarter >> 1) : 8 * quarter;
    // In LDS 16-byte piece p of row r lies at place p ^ r % 16 (codes: p ^ r / 4 % 4), so that the 16 rows of a fragment meet different
    // banks. Addresses are a scalar base and a lane's 32-bit offset (rows are at most OZIMMU_MAX_LD apart). Rows of weights that are not
    // there repeat the last one: their results go nowhere. Tokens that are not there are not loaded: neither do theirs.
    const raw* xb = reinterpret_cast<const raw*>(X) + (int64_t)min(t0, t - 1) * ldx;
    const uint8_t* qb = codes + n0 * ldq;
    const raw* sb = reinterpret_cast<const raw*>(scales) + n0 * lds;
    constexpr int kLanes = kTokenRow / 16, kRows = 64 / kLanes, kLoads = 16 * TT / kRows;   // of a token's row, rows of a load, loads of a step
    constexpr int kPer = 16 / sizeof(raw);
    const int tokens_here = min(16 * TT, t - t0);
    unsigned char* const x_lds = lds_bytes + wave * (16 * TT * kTokenRow + kCodes);
    unsigned char* const q_lds = x_lds + 16 * TT * kTokenRow;
    unsigned xo[kLoads], qo[NT], so[NT];   // bytes
#pragma unroll
    for (int i = 0; i < kLoads; ++i) xo[i] = ((unsigned)max(min(kRows * i + lane / kLanes, t - 1 - t0), 0) * (unsigned)ldx + lane % kLanes * kPer) * sizeof(raw);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        qo[i] = (unsigned)min((int64_t)(16 * i + lane / 4), n - 1 - n0) * (unsigned)ldq + lane % 4 * 16;
        so[i] = (unsigned)min((int64_t)(16 * i + (lane & 15)), n - 1 - n0) * (unsigned)lds * sizeof(raw);
    }
    auto from = [](const void* base, int64_t at, unsigned offset) { return reinterpret_cast<const uint8_t*>(base) + at + offset; };

    // 16 bytes of every row and quarter: positions 32 quarter .. + 31 of the step
    auto load_codes = [&](int step, v4u (&w)[NT], raw (&sc)[NT][GROUPS]) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            w[i] = *reinterpret_cast<const v4u*>(from(qb, (int64_t)step * 64, qo[i]));
            const uint8_t* at = from(sb, (int64_t)step * GROUPS * sizeof(raw), so[i]);
            if constexpr (GROUPS * sizeof(raw) == 16)
                *reinterpret_cast<v4u*>(sc[i]) = *reinterpret_cast<const v4u_any*>(at);
            else if constexpr (GROUPS * sizeof(raw) == 8)
                *reinterpret_cast<v2u*>(sc[i]) = *reinterpret_cast<const v2u_any*>(at);
            else if constexpr (GROUPS * sizeof(raw) == 4)
                *reinterpret_cast<unsigned*>(sc[i]) = *reinterpret_cast<const u32_any*>(at);
            else
                sc[i][0] = *reinterpret_cast<const raw*>(at);
        }
    };
    auto load_tokens = [&](int step, v4u (&to)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (kRows * i < tokens_here) to[i] = *reinterpret_cast<const v4u_any*>(from(xb, (int64_t)step * kTokenRow, xo[i]));
    };
    // The same where a row ends inside the step: tokens beyond k are zeros, so any finite code will do there (rows take a multiple of 16
    // bytes).
    auto load_last_codes = [&](v4u (&w)[NT], raw (&sc)[NT][GROUPS]) {
        const int64_t last = pad_to(k, 32) / 2 - 16;
        const int groups = (int)((k + GROUP - 1) / GROUP);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            w[i] = *reinterpret_cast<const v4u*>(from(qb, min((int64_t)full * 64 + lane % 4 * 16, last) - lane % 4 * 16, qo[i]));
#pragma unroll
            for (int h = 0; h < GROUPS; ++h) sc[i][h] = *reinterpret_cast<const raw*>(from(sb, (int64_t)min(full * GROUPS + h, groups - 1) * sizeof(raw), so[i]));
        }
    };
    auto load_last_tokens = [&](v4u (&to)[kLoads]) {
        const int64_t at = (int64_t)full * 128 + lane % kLanes * kPer;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            raw r[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int64_t beyond = max(at + e - (k - 1), (int64_t)0);
                const raw y = *reinterpret_cast<const raw*>(from(xb, ((int64_t)full * 128 + e - beyond) * (int64_t)sizeof(raw), xo[i]));
                r[e] = beyond ? raw(0) : y;
            }
            to[i] = *reinterpret_cast<const v4u*>(r);
        }
    };

    v4f total[NT][TT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) total[i][tt] = v4f{0.f, 0.f, 0.f, 0.f};
    const CodeBits bits = CodeBits::of();

    auto in_order = [] {   // of the wavefront's own accesses to LDS
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    auto multiply = [&](const v4u (&w_read)[NT], const raw (&sc)[NT][GROUPS], const v4u (&x_read)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = kRows * i + lane / kLanes;
            *reinterpret_cast<v4u*>(x_lds + row * kTokenRow + (lane % kLanes ^ (row & 15)) * 16) = x_read[i];
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) *reinterpret_cast<v4u*>(q_lds + i * 1024 + lane / 4 * 64 + (lane % 4 ^ (lane / 16)) * 16) = w_read[i];
        in_order();
        v4u w[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) w[i] = *reinterpret_cast<const v4u*>(q_lds + i * 1024 + (lane & 15) * 64 + (quarter ^ ((lane & 15) / 4)) * 16);
        // words by group: the quarters of a group of 64 or 32 hold positions of two or four groups each and exchange them
        unsigned words[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            v4u v = w[i];
            if constexpr (GROUP < 128) {
                const auto a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
                const auto b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
                v = v4u{a[0], b[0], a[1], b[1]};
                if constexpr (GROUP == 32) {
                    const auto c = __builtin_amdgcn_permlane16_swap(v[0], v[1], false, false);
                    const auto e = __builtin_amdgcn_permlane16_swap(v[2], v[3], false, false);
                    v = v4u{c[0], c[1], e[0], e[1]};
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) words[i][j] = v[j];
        }
#pragma unroll
        for (int h = 0; h < GROUPS; ++h) {
            v4f sum[NT][TT];
#pragma unroll
            for (int j = 0; j < GW; ++j) {
                Operand<TYPE> o[TT];
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    Raw<TYPE> x;
                    const int piece = (at_quarter + GROUP * h + 8 * j) / kPer;
#pragma unroll
                    for (int v = 0; v < 8 / kPer; ++v)
                        x.v[v] = *reinterpret_cast<const v4u*>(x_lds + (16 * tt + (lane & 15)) * kTokenRow + ((piece + v) ^ (lane & 15)) * 16);
                    o[tt] = operand<TYPE>(x);
                }
                const v4f zero = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const unsigned word = words[i][GW * h + j];
                    const v4u c = BF16 ? sixteenths_bf16(word) : codes_f16(word, bits);
#pragma unroll
                    for (int p = Operand<TYPE>::kPieces - 1; p >= 0; --p)   // (of 32-bit tokens the smallest first)
#pragma unroll
                        for (int tt = 0; tt < TT; ++tt) sum[i][tt] = mfma_half<BF16>(o[tt].piece[p], c, j || p + 1 < Operand<TYPE>::kPieces ? sum[i][tt] : zero);
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float f = E::load(sc[i][h]);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) total[i][tt][e] = fmaf(f, sum[i][tt][e], total[i][tt][e]);
            }
        }
    };
    if (mine > 0) {
        v4u w[DEPTH][NT];
        raw sc[DEPTH][NT][GROUPS] __attribute__((aligned(16)));
        v4u xs[2][kLoads] = {};   // this step's tokens and the next one's
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < mine) load_codes(d * W + wave, w[d], sc[d]);
        load_tokens(wave, xs[0]);
        for (int step0 = 0; step0 < mine; step0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int step = step0 + d;
                if (step >= mine) break;
                if (step + 1 < mine) load_tokens((step + 1) * W + wave, xs[(d + 1) & 1]);
                multiply(w[d], sc[d], xs[d & 1]);
                in_order();
                if (step + DEPTH < mine) load_codes((step + DEPTH) * W + wave, w[d], sc[d]);
            }
        }
    }
    if (wave == W - 1 && k > (int64_t)full * 128) {
        v4u w[NT];
        raw sc[NT][GROUPS];
        v4u xs[kLoads];
        load_last_codes(w, sc);
        load_last_tokens(xs);
        multiply(w, sc, xs);
    }
    __syncthreads();   // the parts take the place of the tokens and codes

    // lane: tokens 4 quarter .. + 3 of a tile, rows lane % 16
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part[(wave * 16 * TT + 16 * tt + 4 * quarter + e) * kRow + 16 * i + (lane & 15)] = total[i][tt][e];
    __syncthreads();
    const int here = min(16 * TT, t - t0);
    for (int at = threadIdx.x; at < here * 16 * NT; at += W * 64) {
        const int tok = at / (16 * NT), col = at % (16 * NT);
        if (n0 + col >= n) continue;
        float sum = part[tok * kRow + col];
#pragma unroll
        for (int i = 1; i < W; ++i) sum += part[(i * 16 * TT + tok) * kRow + col];
        reinterpret_cast<raw*>(Y)[(int64_t)(t0 + tok) * ldy + n0 + col] = E::store(BF16 ? 16.f * sum : sum);   // (the codes' sixteenths)
    }
}

template <int TYPE, int GROUP, int NT, int TT, int W>
hipError_t launch_tiles(int64_t t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    constexpr auto kernel = q4_few_kernel<TYPE, GROUP, NT, TT, W>;
    constexpr int kPart = 16 * TT * (16 * NT + 1) * sizeof(float), kWalk = 16 * TT * 128 * sizeof(typename Elem<TYPE>::raw) + NT * 1024;
    constexpr int bytes = W * (kPart > kWalk ? kPart : kWalk);
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
    const dim3 grid((unsigned)((n + 16 * NT - 1) / (16 * NT)), (unsigned)((t + 16 * TT - 1) / (16 * TT)));
    kernel<<<grid, W * 64, bytes, st>>>((int)t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy);
    return hipGetLastError();
}
template <int TYPE, int GROUP>
hipError_t launch_typed(int64_t t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    // The smallest tile with which a workgroup has a compute unit to itself: more rows of W or tokens to a wavefront share operands and
    // loads, fewer keep more compute units busy. (bf16, us, rows x tokens 16 x 16, 32 x 16, 64 x 16, 32 x 32: 16 tokens, 4096 x 11008 13.0,
    // 15.6, 21.2, 17.7; 16384 x 8192 27.1, 21.4, 20.3, 28.8; 64 tokens, 2048 x 16384 22.5, 21.5, 30.9, 25.8; 8192 x 4096 25.7, 21.8, 21.5,
    // 18.0.) Two tiles of tokens take registers that 32-bit tokens do not leave. The smallest has sixteen wavefronts along a long k (2048 x
    // 16384, 16 tokens: 12.7 against 16.4).
    const auto fits = [&](int64_t rows, int64_t tokens) { return ((n + rows - 1) / rows) * ((t + tokens - 1) / tokens) <= kComputeUnits; };
    if constexpr (TYPE != OZIMMU_F32) {
        if (fits(16, 16) && k >= 16 * 128) return launch_tiles<TYPE, GROUP, 1, 1, 16>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    }
    if (fits(16, 16)) return launch_tiles<TYPE, GROUP, 1, 1, 8>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    // (32-bit types in groups of 32 hold four scales a step and row: with four tiles of rows the registers do not suffice. 16 tokens, 16384
    // x 8192 42.8 and 45.5 us, 8192 x 4096 13.0 and 24.4.)
    if constexpr (TYPE == OZIMMU_F32 && GROUP == 32) {
        return launch_tiles<TYPE, GROUP, 2, 1, 8>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    } else {
        if (fits(32, 16)) return launch_tiles<TYPE, GROUP, 2, 1, 8>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
        if constexpr (TYPE != OZIMMU_F32) {
            if (t > 16) return launch_tiles<TYPE, GROUP, 2, 2, 8>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
        }
        return launch_tiles<TYPE, GROUP, 4, 1, 8>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    }
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
