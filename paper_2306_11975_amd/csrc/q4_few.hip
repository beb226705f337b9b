// Y = X W^T for few tokens and weights in four bits: one pass over the codes, no workspace (gfx950).
//
// What bounds it is reading the codes; the sums go to the matrix cores (v_mfma_f32_16x16x32) although most of their rows stay empty with
// one token, because the vector units have their hands full making 16-bit operands of the codes. A wavefront takes 16 NT rows of
// W, 16 TT tokens and every eighth step of k (every second, with TW = 4 wavefronts along the tokens); the wavefronts of a workgroup share the rows and
// add their parts up in LDS.
//
// A step is 128 positions. A lane loads 16 bytes, 32 positions, of row lane % 16 of each 16 x 128 block of codes. An MFMA adds up positions of one
// group only: in groups of 64 and 32 the quarters of a wavefront (lane / 16) first exchange words (v_permlane32_swap, v_permlane16_swap), so that
// word j of every lane belongs to one group, and is MFMA j's operand. (Loads of 8 and 4 bytes instead: 78 us where these take 31.) The tokens' operand
// is loaded from the same positions.
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

// The two constants of offset_codes in registers of their own (v_and_or_b32 takes one scalar and no two literals), hidden from the optimiser, which would turn them back
// into literals and take two instructions.
struct CodeBits {
    unsigned mask, one;
    template <bool BF16>
    static __device__ __forceinline__ CodeBits of() {
        CodeBits c;
        if constexpr (BF16)
            asm("s_mov_b32 %0, 0x00780078\n\tv_mov_b32 %1, 0x41804180" : "=s"(c.mask), "=v"(c.one));
        else
            asm("s_mov_b32 %0, 0x03c003c0\n\tv_mov_b32 %1, 0x4c004c00" : "=s"(c.mask), "=v"(c.one));
        return c;
    }
};
// 16 + (c + 8) of the codes (0, 4), (1, 5), (2, 6), (3, 7) of a word
template <bool BF16>
__device__ __forceinline__ v4u offset_codes(unsigned w, const CodeBits& b) {
    v4u r;
    if constexpr (BF16) {
        r[0] = ((w << 3) & b.mask) | b.one;
        r[1] = ((w >> 1) & b.mask) | b.one;
        r[2] = ((w >> 5) & b.mask) | b.one;
        r[3] = ((w >> 9) & b.mask) | b.one;
    } else {
        r[0] = ((w << 6) & b.mask) | b.one;
        r[1] = ((w << 2) & b.mask) | b.one;
        r[2] = ((w >> 2) & b.mask) | b.one;
        r[3] = ((w >> 6) & b.mask) | b.one;
    }
    return r;
}
// the codes' sixteenths as bf16, exactly: the conversion from four signed bits gives them, and four bits fit the upper half of a 32-bit value
__device__ __forceinline__ v4u exact_codes(unsigned w) {
    w ^= 0x88888888u;
    v4u r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (4 * i))), hi = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (4 * i + 16)));
        r[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
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
            t.piece[0][i] = __builtin_amdgcn_perm(a[i + 4], a[i], 0x07060302u);
            t.piece[1][i] = __builtin_amdgcn_perm(b[i + 4], b[i], 0x07060302u);
            t.piece[2][i] = __builtin_amdgcn_perm(c[i + 4], c[i], 0x07060302u);
        }
    } else {
        t.piece[0] = pair_by_four(r.v[0]);
    }
    return t;
}

template <int TYPE, int GROUP, int NT, int TT, int TW>
__launch_bounds__(kWaves * 64)
__global__ void q4_few_kernel(int t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales,
                              int64_t lds, void* Y, int64_t ldy) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    constexpr bool BF16 = TYPE != OZIMMU_F16;
    constexpr int GW = GROUP / 32, GROUPS = 128 / GROUP;   // words of a lane per group, groups of a step
    constexpr int DEPTH = 2;                 // steps whose codes are on their way at a time
    extern __shared__ float part[];                        // [wave][token][row]
    constexpr int kRow = 16 * NT + 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
    constexpr int KW = kWaves / TW;                        // TW wavefronts along the tokens, KW share the steps
    const int part_k = wave % KW, part_t = wave / KW;
    const int t0 = (blockIdx.y * TW + part_t) * (16 * TT);
    // Whole steps are dealt to the wavefronts in turn (together they read lines in full); the last wavefront takes what is left of the row beyond them too.
    const int full = (int)(k / 128);
    const int mine = t0 < t ? (full - part_k + KW - 1) / KW : 0;
    const int quarter = lane >> 4;
    // position of word j of group h in a step, for this lane (the exchange between quarters below)
    const int at_quarter = GROUP == 128 ? 32 * quarter : GROUP == 64 ? 32 * (quarter & 1) + 16 * (quarter >> 1) : 8 * quarter;
    // Addresses are a scalar base and a lane's 32-bit offset (rows are at most OZIMMU_MAX_LD apart). Lanes of tokens and rows that are not there repeat the last one: their
    // results go nowhere.
    const raw* xb = reinterpret_cast<const raw*>(X) + (int64_t)min(t0, t - 1) * ldx;
    const uint8_t* qb = codes + n0 * ldq;
    const raw* sb = reinterpret_cast<const raw*>(scales) + n0 * lds;
    unsigned xo[TT], qo[NT], so[NT];   // bytes
#pragma unroll
    for (int i = 0; i < TT; ++i) xo[i] = ((unsigned)max(min(16 * i + (lane & 15), t - 1 - t0), 0) * (unsigned)ldx + at_quarter) * sizeof(raw);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const unsigned row = (unsigned)min((int64_t)(16 * i + (lane & 15)), n - 1 - n0);
        qo[i] = row * (unsigned)ldq + quarter * 16;
        so[i] = row * (unsigned)lds * sizeof(raw);
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
    constexpr int kParts = TYPE == OZIMMU_F32 ? 2 : 1;
    auto load_word = [&](int step, int j, Raw<TYPE> (&to)[TT]) {
        const int64_t at = ((int64_t)step * 128 + (j / GW) * GROUP + 8 * (j % GW)) * sizeof(raw);
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int v = 0; v < kParts; ++v) to[i].v[v] = *reinterpret_cast<const v4u_any*>(from(xb, at + 16 * v, xo[i]));
    };
    // The same where a row ends inside the step: tokens beyond k are zeros, so any finite code will do there (rows take a multiple of 16 bytes).
    auto load_last_codes = [&](v4u (&w)[NT], raw (&sc)[NT][GROUPS]) {
        const int64_t last = pad_to(k, 32) / 2 - 16;
        const int groups = (int)((k + GROUP - 1) / GROUP);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            w[i] = *reinterpret_cast<const v4u*>(from(qb, min((int64_t)full * 64 + quarter * 16, last) - quarter * 16, qo[i]));
#pragma unroll
            for (int h = 0; h < GROUPS; ++h) sc[i][h] = *reinterpret_cast<const raw*>(from(sb, (int64_t)min(full * GROUPS + h, groups - 1) * sizeof(raw), so[i]));
        }
    };
    auto load_last_word = [&](int j, Raw<TYPE> (&to)[TT]) {
        const int64_t at = (int64_t)full * 128 + (j / GW) * GROUP + 8 * (j % GW);
#pragma unroll
        for (int i = 0; i < TT; ++i) {
            raw r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t beyond = max(at + at_quarter + e - (k - 1), (int64_t)0);
                const raw y = *reinterpret_cast<const raw*>(from(xb, (at + e - beyond) * (int64_t)sizeof(raw), xo[i]));
                r[e] = beyond ? raw(0) : y;
            }
#pragma unroll
            for (int v = 0; v < kParts; ++v) to[i].v[v] = *reinterpret_cast<const v4u*>(r + 4 * v);
        }
    };

    v4f total[NT][TT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) total[i][tt] = v4f{0.f, 0.f, 0.f, 0.f};
    const unsigned minus = BF16 ? 0xc1c0c1c0u : 0xce00ce00u;   // -24, twice
    const v4u minus24 = {minus, minus, minus, minus};
    const CodeBits bits = CodeBits::of<BF16>();

    auto multiply = [&](const v4u (&w)[NT], const raw (&sc)[NT][GROUPS], const Raw<TYPE> (&xs)[4][TT]) {
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
            v4f sum[NT][TT], offset[TT];
#pragma unroll
            for (int j = 0; j < GW; ++j) {
                Operand<TYPE> o[TT];
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) o[tt] = operand<TYPE>(xs[GW * h + j][tt]);
                const v4f zero = v4f{0.f, 0.f, 0.f, 0.f};
                if constexpr (TYPE != OZIMMU_F32)
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) offset[tt] = mfma_half<BF16>(o[tt].piece[0], minus24, j ? offset[tt] : zero);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const unsigned word = words[i][GW * h + j];
                    if constexpr (TYPE == OZIMMU_F32) {
                        const v4u c = exact_codes(word);
#pragma unroll
                        for (int p = 2; p >= 0; --p)
#pragma unroll
                            for (int tt = 0; tt < TT; ++tt) sum[i][tt] = mfma_half<true>(o[tt].piece[p], c, j || p < 2 ? sum[i][tt] : zero);
                    } else {
                        const v4u c = offset_codes<BF16>(word, bits);
#pragma unroll
                        for (int tt = 0; tt < TT; ++tt) sum[i][tt] = mfma_half<BF16>(o[tt].piece[0], c, j ? sum[i][tt] : zero);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float f = E::load(sc[i][h]);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        total[i][tt][e] = fmaf(f, TYPE == OZIMMU_F32 ? sum[i][tt][e] : sum[i][tt][e] + offset[tt][e], total[i][tt][e]);
            }
        }
    };
    if (mine > 0) {
        v4u w[DEPTH][NT];
        raw sc[DEPTH][NT][GROUPS] __attribute__((aligned(16)));
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < mine) load_codes(d * KW + part_k, w[d], sc[d]);
        Raw<TYPE> xs[2][4][TT];   // this step's tokens and the next one's
#pragma unroll
        for (int j = 0; j < 4; ++j) load_word(part_k, j, xs[0][j]);
        for (int step0 = 0; step0 < mine; step0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int step = step0 + d;
                if (step >= mine) break;
                if (step + 1 < mine)
#pragma unroll
                    for (int j = 0; j < 4; ++j) load_word((step + 1) * KW + part_k, j, xs[(d + 1) & 1][j]);
                multiply(w[d], sc[d], xs[d & 1]);
                if (step + DEPTH < mine) load_codes((step + DEPTH) * KW + part_k, w[d], sc[d]);
            }
        }
    }
    if (part_k == KW - 1 && t0 < t && k > (int64_t)full * 128) {
        v4u w[NT];
        raw sc[NT][GROUPS];
        Raw<TYPE> xs[4][TT];
        load_last_codes(w, sc);
#pragma unroll
        for (int j = 0; j < 4; ++j) load_last_word(j, xs[j]);
        multiply(w, sc, xs);
    }

    // lane: tokens 4 quarter .. + 3 of a tile, rows lane % 16
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part[((part_k * TW + part_t) * 16 * TT + 16 * tt + 4 * quarter + e) * kRow + 16 * i + (lane & 15)] = total[i][tt][e];
    __syncthreads();
    const int first = blockIdx.y * (16 * TT * TW), here = min(16 * TT * TW, t - first);
    for (int at = threadIdx.x; at < here * 16 * NT; at += kWaves * 64) {
        const int tok = at / (16 * NT), col = at % (16 * NT);
        if (n0 + col >= n) continue;
        float sum = part[tok * kRow + col];
#pragma unroll
        for (int i = 1; i < KW; ++i) sum += part[(i * 16 * TT * TW + tok) * kRow + col];
        reinterpret_cast<raw*>(Y)[(int64_t)(first + tok) * ldy + n0 + col] = E::store(TYPE == OZIMMU_F32 ? 16.f * sum : sum);   // (the codes' sixteenths)
    }
}

template <int TYPE, int GROUP, int NT, int TT, int TW>
hipError_t launch_tiles(int64_t t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    constexpr auto kernel = q4_few_kernel<TYPE, GROUP, NT, TT, TW>;
    constexpr int bytes = kWaves * 16 * TT * (16 * NT + 1) * sizeof(float);
    if (hipError_t e = allow_dynamic_lds<kernel>(bytes); e != hipSuccess) return e;
    const dim3 grid((unsigned)((n + 16 * NT - 1) / (16 * NT)), (unsigned)((t + 16 * TT * TW - 1) / (16 * TT * TW)));
    kernel<<<grid, kWaves * 64, bytes, st>>>((int)t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy);
    return hipGetLastError();
}
template <int TYPE, int GROUP>
hipError_t launch_typed(int64_t t, int64_t n, int64_t k, const void* X, int64_t ldx, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                        void* Y, int64_t ldy, hipStream_t st) {
    // More rows of W to a wavefront: fewer loads of tokens; more wavefronts: more codes on their way. (t = 16, n = 16384, k = 8192 with 16, 32, 64 rows: 46.9, 32.7, 25.8 us;
    // t = 1: 27.7, 22.5, 20.9; but n = 8192, k = 4096, t = 1: 8.7, 8.0, 12.0.) Two tiles of tokens share the operands made of the codes; with
    // 32-bit tokens the registers do not suffice; those have four wavefronts along the tokens instead of all along k, where that leaves enough workgroups: a part of k is
    // longer and fewer sums meet in LDS (300 tokens, n = 1500, k = 1000: 17.9 -> 15.1 us). (So many 16-bit tokens do not come here.)
    const int64_t rows32 = (n + 31) / 32;
    if constexpr (TYPE != OZIMMU_F32) {
        if (t > 16) return launch_tiles<TYPE, GROUP, 2, 2, 1>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
        if (n >= 64 * 256) return launch_tiles<TYPE, GROUP, 4, 1, 1>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    } else {
        if (t > 32 && rows32 * ((t + 63) / 64) >= 192) return launch_tiles<TYPE, GROUP, 2, 1, 4>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    }
    if (rows32 * ((t + 15) / 16) >= 256) return launch_tiles<TYPE, GROUP, 2, 1, 1>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
    return launch_tiles<TYPE, GROUP, 1, 1, 1>(t, n, k, X, ldx, codes, ldq, scales, lds, Y, ldy, st);
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
