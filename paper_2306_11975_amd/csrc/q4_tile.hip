// Y = X W^T of weights in four bits with 16-bit tokens, tile by tile, the operand of the weights made on the way (gfx950). One launch, no
// workspace.
//
// A workgroup owns BM tokens x BN outputs; a slab is 64 positions of k. What a slab takes from memory is on its way in registers several
// slabs ahead: 16 bytes a lane of the tokens, and codes with their scales. A slab's codes become the weights s c, rounded once to 16 bits
// (as they are where the weights' operand is made by a pass of its own), and go to LDS beside the tokens, in the layout of nt_product.h:
// rows of 128 bytes, 16-byte piece p of row r at place p ^ (r % 8), which the fragments' reads (16 rows, one piece) meet without bank
// conflicts.
//
// Against the passes of q4_few.hip (32 tokens each): the codes are converted once for BM tokens and take one MFMA, not two. Against a pass
// that writes the operand and a product that reads it: four times fewer bytes of the weights come and none go; every tile of tokens
// converts the codes again. So it serves the counts between the two. us in bf16, of the passes, here, of operand and product: 300 tokens
// through 8192 x 4096 83, 60, 65; 128 through 16384 x 8192 119, 88, 156, 256 (128 x 128 tiles from here) 234, 128, 222, 512 439, 198, 238;
// 128 through 5000 x 200 11.2, 6.4, 8.9; 512 through 20000 x 64 109, 12.0, 16.0. What bounds it is a workgroup's walk: 0.5 us a slab of 64
// x 64 (0.95 of 128 x 128), of which the conversion, in the same wavefronts as the MFMAs, takes more than half. (dX = dY W, whose codes lie
// across the inner dimension, gains nothing so: 128 x 8192 x 4096 83 us against 38.)
#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;   // 2 x 2 wavefronts

struct TileArgs {
    int t, n, k;                // tokens, outputs, positions (at least eight)
    const unsigned short* X;    // t x k
    int64_t ldx;
    const uint8_t* codes;
    int64_t ldq;
    const unsigned short* scales;
    int64_t lds;
    int group_log2, groups, last_bytes;   // of a row of codes: bytes less the last 16
    unsigned short* Y;          // t x n
    int64_t ldy;
    int tiles_m, tiles_n;
};

// Code e of a word whose codes have been turned into signed ones (c + 8 with its highest bit changed).
__device__ __forceinline__ float code_of(unsigned word, int e) { return (float)((int)(word << (28 - 4 * e)) >> 28); }

// The eight weights s c of a word, rounded to 16 bits (why: q4_rows of q4.hip). bf16: in order; fp16: paired (0, 4), (1, 5), (2, 6), (3,
// 7).
template <int TYPE>
__device__ __forceinline__ v4u weights_of(unsigned word, unsigned short scale) {
    v4u r;
    if constexpr (TYPE == OZIMMU_BF16) {
        const float s = bf16_to_f32(scale);
        word ^= 0x88888888u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = s * code_of(word, 2 * i), y = s * code_of(word, 2 * i + 1);
            r[i] = (unsigned)f32_to_bf16(x) | (unsigned)f32_to_bf16(y) << 16;
        }
    } else {
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        const _Float16 h = __builtin_bit_cast(_Float16, scale);
        const v2h s = {h, h}, less = {(_Float16)-1032.f, (_Float16)-1032.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // 1024 + (c + 8) in the mantissa; both steps exact but for the product's rounding
            const v2h x = __builtin_bit_cast(v2h, ((word >> (4 * i)) & 0x000f000fu) | 0x64006400u);
            r[i] = __builtin_bit_cast(unsigned, (x + less) * s);
        }
    }
    return r;
}
template <int TYPE, int BM, int BN>
__launch_bounds__(kThreads, BM == 64 ? 4 : 2)
__global__ void q4_tile_kernel(TileArgs a) {
    typedef Elem<TYPE> E;
    constexpr bool BF16 = TYPE == OZIMMU_BF16;
    constexpr int MI = BM / 32, NI = BN / 32;            // 16 x 16 results of a wavefront
    constexpr int XL = BM / 32;                          // 16-byte pieces of the tokens for a thread and slab
    constexpr int WW = BN / 32;                          // words of codes
    constexpr int PER_ROW = kThreads / BN;               // threads of a row of codes
    constexpr int AHEAD = 4;                             // slabs of codes on their way; of tokens two
    constexpr unsigned kStage = (BM + BN) * 128;
    __shared__ __attribute__((aligned(16))) unsigned char lds[2 * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x;
    int tm, tn;
    tile_of_block(blockIdx.x, a.tiles_m, a.tiles_n, tm, tn);
    const int row0 = tm * BM, col0 = tn * BN;
    const int slabs = (a.k + 63) / 64, whole = a.k / 64;

    // ---- memory to registers: scalar bases, 32-bit offsets
    const uint8_t* const xb = reinterpret_cast<const uint8_t*>(a.X + (int64_t)row0 * a.ldx);
    unsigned xo[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) xo[i] = ((unsigned)min(tid / 8 + 32 * i, a.t - 1 - row0) * (unsigned)a.ldx + tid % 8 * 8) * 2;
    auto load_tokens = [&](int slab, v4u (&x)[XL]) {
        if (slab < whole) {
#pragma unroll
            for (int i = 0; i < XL; ++i) x[i] = *reinterpret_cast<const v4u_any*>(xb + (int64_t)slab * 128 + xo[i]);
        } else {   // the slab in which the rows end: a piece that reaches beyond is read from the row's last eight values, moved down, zeros behind them
            const int over = min(max(slab * 64 + tid % 8 * 8 + 8 - a.k, 0), 8);
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                const int back = max(slab * 64 + tid % 8 * 8 + 8 - a.k, 0);
                v4u y = *reinterpret_cast<const v4u_any*>(xb + ((int64_t)slab * 64 - back) * 2 + xo[i]);
                if (over & 4) y = v4u{y[2], y[3], 0u, 0u};
                if (over & 2) y = v4u{y[1], y[2], y[3], 0u};
                if (over & 1) y = v4u{y[0] >> 16 | y[1] << 16, y[1] >> 16 | y[2] << 16, y[2] >> 16 | y[3] << 16, y[3] >> 16};
                if (over & 8) y = v4u{0u, 0u, 0u, 0u};
                x[i] = y;
            }
        }
    };
    struct Codes {   // of one row, with their scale
        unsigned w[WW];
        unsigned short s;
    };
    const uint8_t* const qb = a.codes + (int64_t)col0 * a.ldq;
    const int w_row = min(tid / PER_ROW, a.n - 1 - col0), w_at = tid % PER_ROW * (8 * WW);
    const unsigned short* const sb = a.scales + (int64_t)col0 * a.lds;
    auto load_codes = [&](int slab, Codes& c) {
        // positions beyond the row repeat its end, and are then replaced
        const unsigned at = (unsigned)min(slab * 32 + w_at / 2, a.last_bytes + (w_at / 2 & 15));
        const uint8_t* from = qb + (unsigned)w_row * (unsigned)a.ldq + at;
        if constexpr (WW == 4)
            *reinterpret_cast<v4u*>(c.w) = *reinterpret_cast<const v4u*>(from);
        else
            *reinterpret_cast<v2u*>(c.w) = *reinterpret_cast<const v2u*>(from);
        c.s = sb[(unsigned)w_row * (unsigned)a.lds + min((slab * 64 + w_at) >> a.group_log2, a.groups - 1)];
        // The slab in which the rows end: weights of zero beyond, whatever codes stand there (a large scale makes an infinity of one, and a
        // token's zero times that is NaN). Here, four slabs ahead, and not in the conversion, where a branch costs up to 5 %.
        if (slab >= whole) {
            const int here = a.k - slab * 64 - w_at;   // positions of this thread's
#pragma unroll
            for (int u = 0; u < WW; ++u) {
                const int beyond = 4 * min(max(here - 8 * u, 0), 8);   // from this bit on
                const unsigned keep = beyond < 32 ? (1u << beyond) - 1u : ~0u;
                c.w[u] = (c.w[u] & keep) | (0x88888888u & ~keep);
            }
            if (here <= 0) c.s = 0;
        }
    };

    // ---- registers to LDS
    auto store_tokens = [&](int stage, const v4u (&x)[XL]) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int row = tid / 8 + 32 * i;
            v4u y = x[i];
            if constexpr (!BF16)   // in the order of the weights' pairs
                y = v4u{__builtin_amdgcn_perm(x[i][2], x[i][0], 0x05040100u), __builtin_amdgcn_perm(x[i][2], x[i][0], 0x07060302u),
                        __builtin_amdgcn_perm(x[i][3], x[i][1], 0x05040100u), __builtin_amdgcn_perm(x[i][3], x[i][1], 0x07060302u)};
            *reinterpret_cast<v4u*>(lds + stage * kStage + row * 128 + ((tid % 8 ^ (row & 7)) * 16)) = y;
        }
    };
    auto store_codes = [&](int stage, const Codes& c) {
        unsigned char* const base = lds + stage * kStage + BM * 128;
        const int row = tid / PER_ROW;
#pragma unroll
        for (int u = 0; u < WW; ++u)
            *reinterpret_cast<v4u*>(base + row * 128 + (((tid % PER_ROW * WW + u) ^ (row & 7)) * 16)) = weights_of<TYPE>(c.w[u], c.s);
    };

    const int wm = wave >> 1, wn = wave & 1;
    v4f acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    const int fr = lane & 15, fq = lane >> 4;
    struct Frags {
        v4u p[MI], q[NI];
    };
    auto read = [&](int stage, int h, Frags& f) {
        const unsigned char* at_p = lds + stage * kStage + (wm * (BM / 2) + fr) * 128;
        const unsigned char* at_q = lds + stage * kStage + BM * 128 + (wn * (BN / 2) + fr) * 128;
#pragma unroll
        for (int i = 0; i < MI; ++i) f.p[i] = *reinterpret_cast<const v4u*>(at_p + i * 2048 + (((fq + 4 * h) ^ (fr & 7)) * 16));
#pragma unroll
        for (int j = 0; j < NI; ++j) f.q[j] = *reinterpret_cast<const v4u*>(at_q + j * 2048 + (((fq + 4 * h) ^ (fr & 7)) * 16));
    };
    auto multiply = [&](const Frags& f) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mfma_half<BF16>(f.q[j], f.p[i], acc[i][j]);
    };

    // (the compiler's own barrier would wait for the loads that are on their way too)
    auto meet = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    // ---- the walk: in slab s, s + 1 goes from registers to LDS, s + 3 of the tokens and s + 5 of the codes are asked for
    v4u x[2][XL] = {};
    Codes c[AHEAD] = {};
    load_tokens(0, x[0]);
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (d < slabs) load_codes(d, c[d]);
    if (1 < slabs) load_tokens(1, x[1]);
    store_tokens(0, x[0]);
    store_codes(0, c[0]);
    if (2 < slabs) load_tokens(2, x[0]);
    if (AHEAD < slabs) load_codes(AHEAD, c[0]);
    meet();
    for (int slab0 = 0; slab0 < slabs; slab0 += AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int slab = slab0 + d;
            if (slab >= slabs) break;
            Frags f;
            read(d & 1, 0, f);
            multiply(f);
            read(d & 1, 1, f);
            multiply(f);
            if (slab + 1 < slabs) {
                store_tokens((d + 1) & 1, x[(d + 1) & 1]);
                store_codes((d + 1) & 1, c[(d + 1) % AHEAD]);
                if (slab + 3 < slabs) load_tokens(slab + 3, x[(d + 1) & 1]);
                if (slab + 1 + AHEAD < slabs) load_codes(slab + 1 + AHEAD, c[(d + 1) % AHEAD]);
            }
            meet();
        }
    }

    // lane: row (token) lane % 16, columns 4 (lane / 16) .. + 3
    const bool wide = (a.ldy & 3) == 0 && (reinterpret_cast<uintptr_t>(a.Y) & 7) == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int r = row0 + wm * (BM / 2) + 16 * i + fr;
        if (r >= a.t) continue;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int col = col0 + wn * (BN / 2) + 16 * j + 4 * fq;
            if (col >= a.n) continue;
            unsigned short v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = E::store(acc[i][j][e]);
            unsigned short* at = a.Y + (int64_t)r * a.ldy + col;
            if (wide && col + 4 <= a.n)
                *reinterpret_cast<v2u*>(at) = *reinterpret_cast<const v2u*>(v);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < a.n) at[e] = v[e];
        }
    }
}

template <int TYPE, int BM, int BN>
hipError_t launch_tile(TileArgs& a, hipStream_t st) {
    a.tiles_m = (a.t + BM - 1) / BM;
    a.tiles_n = (a.n + BN - 1) / BN;
    q4_tile_kernel<TYPE, BM, BN><<<dim3((unsigned)a.tiles_m * a.tiles_n), kThreads, 0, st>>>(a);
    return hipGetLastError();
}
template <int TYPE>
hipError_t launch_shape(TileArgs& a, bool large, hipStream_t st) {
    return large ? launch_tile<TYPE, 128, 128>(a, st) : launch_tile<TYPE, 64, 64>(a, st);
}

}  // namespace

hipError_t launch_q4_tiles(bool large, int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes, int64_t ldq,
                           const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st) {
    TileArgs a{};
    a.t = (int)t;
    a.k = (int)k;
    a.n = (int)n;
    a.X = static_cast<const unsigned short*>(X);
    a.ldx = ldx;
    a.codes = codes;
    a.ldq = ldq;
    a.scales = static_cast<const unsigned short*>(scales);
    a.lds = lds;
    a.group_log2 = group == 32 ? 5 : group == 64 ? 6 : 7;
    a.groups = (int)((k + group - 1) / group);
    a.last_bytes = (int)(pad_to(k, 32) / 2 - 16);
    a.Y = static_cast<unsigned short*>(Y);
    a.ldy = ldy;
    return type == OZIMMU_BF16 ? launch_shape<OZIMMU_BF16>(a, large, st) : launch_shape<OZIMMU_F16>(a, large, st);
}

}  // namespace ozimmu
