// C ABI of the operators on weight matrices: argument checks, workspace layout, choice and sequencing of kernels. What computes is in
// q4.hip, q4_token.hip, q4_few.hip, q4_tile.hip, orthogonalize.hip, orthogonalize_small.hip and nt_product.h.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "weights_internal.h"

using namespace ozimmu;

namespace {

constexpr int64_t kMaxDim = OZIMMU_MAX_DIM;
constexpr int64_t kMaxInPlaceLd = 1 << 23;   // the product kernel's row offsets inside a tile are 32-bit byte counts

bool dim_ok(int64_t x) { return x >= 0 && x <= kMaxDim; }
bool type_ok(int type) { return type == OZIMMU_F32 || type == OZIMMU_BF16 || type == OZIMMU_F16; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
size_t size_of(int type) { return type == OZIMMU_F32 ? 4 : 2; }
size_t align_up(size_t x) { return (x + OZIMMU_WORKSPACE_ALIGN - 1) / OZIMMU_WORKSPACE_ALIGN * OZIMMU_WORKSPACE_ALIGN; }
int64_t row_bytes(int64_t k) { return pad_to(k, 32) / 2; }
int64_t groups_of(int64_t k, int group) { return (k + group - 1) / group; }
ozimmu_status_t hip_status(hipError_t e) { return e == hipSuccess ? OZIMMU_OK : OZIMMU_ERR_HIP; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// What every call on weights in four bits checks of them (n, k > 0).
ozimmu_status_t check_q4(int64_t k, int group, const void* codes, int64_t ldq, const void* scales, int scale_type, int64_t lds) {
    if (ldq < row_bytes(k) || ldq % 16 != 0 || lds < groups_of(k, group) || ldq > OZIMMU_MAX_LD || lds > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!codes || !scales) return OZIMMU_ERR_NULL;
    if (misaligned(codes, 16) || misaligned(scales, size_of(scale_type))) return OZIMMU_ERR_MISALIGNED;
    return OZIMMU_OK;
}

// Room for the sums of shared tiles (nt_choose): at most 32 workgroups share one, four slabs at least to each, and no product takes more
// than kPartialBytes.
size_t partial_room(int64_t batch, int64_t m, int64_t n, int64_t slabs) {
    const int64_t parts = std::min<int64_t>(32, slabs / 4);
    if (parts < 2) return 0;
    const double bytes = (double)batch * (double)pad_to(m, 256) * (double)pad_to(n, 256) * (double)parts * sizeof(float);
    return bytes < (double)kPartialBytes ? (size_t)bytes : kPartialBytes;
}

// The operands of a product with many tokens in the workspace: V (t rows of `inner` values) and the weights (`outer` rows). 32-bit types
// take two slices.
struct Operands {
    int64_t inner, outer, ld;
    size_t off_v, off_w, off_ev, off_ew, off_partial, partial, total;
};
Operands operands(int64_t t, int64_t n, int64_t k, int group, int type, bool gradient) {
    Operands o{};
    o.inner = gradient ? n : k;
    o.outer = gradient ? k : n;
    o.ld = type == OZIMMU_F32 ? 2 * pad_to(o.inner, 32) : pad_to(o.inner, 64);
    size_t off = 0;
    o.off_w = off;
    off = align_up(off + (size_t)o.outer * o.ld * 2);
    o.off_v = off;
    off = align_up(off + (size_t)t * o.ld * 2);
    o.off_ew = off;
    if (type == OZIMMU_F32) off = align_up(off + sizeof(int) * (size_t)(gradient ? groups_of(k, group) : n));
    o.off_ev = off;
    if (type == OZIMMU_F32) off = align_up(off + sizeof(int) * (size_t)t);
    o.off_partial = off;
    o.partial = partial_room(1, t, o.outer, o.ld / kSlabValues);
    off = align_up(off + o.partial);
    o.total = off;
    return o;
}
// How Y = X W^T is computed: for one token or two on the vector units (q4_token.hip); by passes over the codes on the matrix cores, 16 or
// 32 tokens each (q4_few.hip); tile by tile, the weights' operand made on the way (q4_tile.hip, 16-bit types); or as an operand of the
// weights and the tiled product (nt_product.h), which gradients take always.
//
// One token through rows of 512 positions and more is faster on the vector units everywhere, two tokens but for wide layers in bf16 (two,
// passes and vector units, us: 2048 x 2048 4.5, 3.4; 4096 x 11008 bf16 8.7, 12.1, 32 bits 18.5, 12.0; 16384 x 8192 bf16 18.3, 22.7; one
// through 512 x 256 2.5, 2.9). From there on the choice is by an estimate of each, in us. 256 workgroups of the passes (32 rows of weights
// and 32 tokens; 64 and 16 in 32 bits, 32 and 16 with groups of 32) are a round, whose time grows with k. A tile's walk takes half a
// microsecond a slab of 64 positions (twice that the large ones) until the chip has more than one workgroup for a compute unit. The product
// takes a walk along k, the operand's bytes, dearer once no cache holds them, and its own operations. Fitted to 24 to 2048 tokens through
// fifteen layers from 20000 x 64 and 1000 x 333 to 16384 x 8192, where the choices take 0.9 % more than the best ones do on average, 21 %
// at most (1024 tokens, 16384 x 8192: large tiles 382, product 317), and 28 % with groups of 32 in 32 bits. Times of passes, tiles, large
// tiles, product: bf16 2048 x 2048, 64 tokens 7.0, 19.4, 33.7, 17.3, 512 23.4, 20.2, 34.2, 20.4; 8192 x 4096, 64 19.4, 35.3, 62.8, 39.2,
// 256 67.7, 47.3, 64.4, 49.6, 1024 254, 147, 103, 84; 16384 x 8192, 128 119, 88, 123, 156, 512 439, 295, 198, 238; 32 bits 16384 x 8192,
// 128 226, -, -, 319; 8192 x 4096, 384 191, -, -, 116.
//
// With more tokens the answer turns to the product once and stays, so that a workspace serves fewer tokens too: every estimate rises with
// the tokens at least as the product's does. (The passes are held against the product of their round's first tokens; `more` is added to the
// tiles' flat part.)
enum class Way { token, passes, tiles, large_tiles, product };
Way way_of(int64_t t, int64_t n, int64_t k, int group, int type, bool gradient) {
    if (gradient) return Way::product;
    if (k >= 512 && (t == 1 || (t == 2 && (type != OZIMMU_BF16 || n < 4096)))) return Way::token;
    if (t <= 16) return Way::passes;
    const bool wide = type == OZIMMU_F32, narrow = wide && group == 32;   // 64 rows a workgroup of the passes, or 32
    const double nk = (double)n * (double)k, beyond = std::max(0.0, nk - 4.0e7);
    const int64_t passes = wide ? (t + 15) / 16 : (t + 31) / 32, rows = wide && !narrow ? (n + 63) / 64 : (n + 31) / 32;
    const double rounds = std::ceil((double)rows * (double)passes / 256.0), first = (rounds - 1.0) * 256.0 / (double)rows;   // tokens (passes) ahead of this round
    const double product = wide ? 10.7 + 0.0051 * k + 8.75e-7 * nk + 5.3e-7 * beyond : 18.9 + 0.0013 * k + 5.7e-7 * nk + 3.9e-7 * beyond;
    const double more = (wide ? 1.0e-7 : 5.0e-8) * nk;   // of a pass
    const double few = passes > 65535 ? 1.0e300 : narrow ? 0.24 + rounds * (1.6 + 0.0024 * k) : wide ? 0.24 + rounds * (2.25 + 0.0039 * k) : 5.0 + rounds * (0.27 + 0.00184 * k);   // (the launch's second dimension)
    const bool few_lose = few > product + more * first;
    if (wide || k < 8) return few_lose ? Way::product : Way::passes;
    const double slabs = (double)((k + 63) / 64), grown = more * (double)passes;
    const double fill = (double)((n + 63) / 64) * (double)passes / 512.0, fill_large = (double)((n + 127) / 128) * (double)passes / 1024.0;   // workgroups by compute unit
    const double held = 3.2 + 0.54 * fill, held_large = 3.8 + 2.2 * fill_large, slope = (0.23 + 0.225 * fill) * slabs, slope_large = (0.2 + 0.62 * fill_large) * slabs;
    const double surely = std::min(held + std::max(0.51 * slabs + grown, slope), held_large + std::max(slabs + grown, slope_large));
    if (few_lose && surely > product + grown) return Way::product;
    const double tiles = held + std::max(0.51 * slabs, slope), large = held_large + std::max(slabs, slope_large);
    if (few <= std::min(tiles, large)) return Way::passes;
    return large < tiles ? Way::large_tiles : Way::tiles;
}

ozimmu_status_t q4_product(bool gradient, int64_t t, int64_t n, int64_t k, int group, int type, const void* V, int64_t ldv, const uint8_t* codes,
                           int64_t ldq, const void* scales, int64_t lds, void* R, int64_t ldr, void* ws, size_t ws_bytes, void* stream) {
    if (!dim_ok(t) || !dim_ok(n) || !dim_ok(k) || !group_ok(group)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    const int64_t inner = gradient ? n : k, outer = gradient ? k : n;
    if (t == 0 || outer == 0) return OZIMMU_OK;
    if (ldv < inner || ldr < outer || ldv > OZIMMU_MAX_LD || ldr > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!R) return OZIMMU_ERR_NULL;
    if (misaligned(R, size_of(type))) return OZIMMU_ERR_MISALIGNED;
    if (inner > 0) {
        if (!V) return OZIMMU_ERR_NULL;
        if (misaligned(V, size_of(type))) return OZIMMU_ERR_MISALIGNED;
        if (ozimmu_status_t rc = check_q4(k, group, codes, ldq, scales, type, lds); rc != OZIMMU_OK) return rc;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (inner == 0) return hip_status(launch_zero_rows(t, outer, R, type, ldr, st));
    const Way way = way_of(t, n, k, group, type, gradient);
    if (way == Way::token) return hip_status(launch_q4_token(t, n, k, group, V, type, ldv, codes, ldq, scales, lds, R, ldr, st));
    if (way == Way::passes) return hip_status(launch_q4_few(t, n, k, group, V, type, ldv, codes, ldq, scales, lds, R, ldr, st));
    if (way == Way::tiles || way == Way::large_tiles)
        return hip_status(launch_q4_tiles(way == Way::large_tiles, t, n, k, group, V, type, ldv, codes, ldq, scales, lds, R, ldr, st));
    const Operands o = operands(t, n, k, group, type, gradient);
    if (!ws || misaligned(ws, OZIMMU_WORKSPACE_ALIGN) || ws_bytes < o.total) return OZIMMU_ERR_WORKSPACE;
    unsigned char* base = static_cast<unsigned char*>(ws);
    unsigned short* w = reinterpret_cast<unsigned short*>(base + o.off_w);
    int* ew = reinterpret_cast<int*>(base + o.off_ew);
    int* ev = reinterpret_cast<int*>(base + o.off_ev);
    unsigned short* v = reinterpret_cast<unsigned short*>(base + o.off_v);
    // rows of 16-bit values that the kernel can read as they lie need no copy
    const bool in_place = type != OZIMMU_F32 && inner % kSlabValues == 0 && ldv < kMaxInPlaceLd && rows_aligned16(V, ldv, 2);
    hipError_t e = launch_operands(t, n, k, group, type, codes, ldq, scales, lds, gradient, w, ew, V, ldv, in_place ? nullptr : v, ev, o.ld, st);
    NtArgs a{};
    a.P = in_place ? static_cast<const unsigned short*>(V) : v;
    a.ldp = in_place ? ldv : o.ld;
    a.Q = w;
    a.ldq = o.ld;
    a.slabs = (int)(o.ld / kSlabValues);
    a.m = (int)t;
    a.n = (int)outer;
    a.batch = 1;
    a.factor = 1.0f;
    a.partial = reinterpret_cast<float*>(base + o.off_partial);
    a.partial_bytes = o.partial;
    a.out = R;
    a.ldo = ldr;
    if (type == OZIMMU_F32) {
        a.exp_p = ev;
        a.exp_q = ew;
        a.q_run = gradient ? group : 1;
    }
    if (e == hipSuccess)
        e = launch_nt_product(a, type == OZIMMU_F32 ? 2 : 1, type == OZIMMU_BF16, type == OZIMMU_F32 ? kOutF32 : type == OZIMMU_BF16 ? kOutBf16 : kOutF16, st);
    return hip_status(e);
}

// Buffers of the orthogonal update, all in two slices: X as rows along the longer side, its transpose twice (one is read while the next is
// written), A and the polynomial.
struct OrthLayout {
    int64_t r, l;              // shorter and longer side
    int64_t ld_x, ld_t;        // values per row: along the longer side, along the shorter one
    int64_t size_x, size_t_, size_a;
    size_t off_x, off_t[2], off_a, off_q, off_norm, off_partial, partial, total;
};
OrthLayout orth_layout(int64_t batch, int64_t m, int64_t n) {
    OrthLayout o{};
    o.r = std::min(m, n);
    o.l = std::max(m, n);
    o.ld_x = 2 * pad_to(o.l, 32);
    o.ld_t = 2 * pad_to(o.r, 32);
    o.size_x = o.r * o.ld_x;
    o.size_t_ = o.l * o.ld_t;
    o.size_a = o.r * o.ld_t;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes); return at; };
    o.off_x = take(2 * (size_t)batch * o.size_x);
    o.off_t[0] = take(2 * (size_t)batch * o.size_t_);
    o.off_t[1] = take(2 * (size_t)batch * o.size_t_);
    o.off_a = take(2 * (size_t)batch * o.size_a);
    o.off_q = take(2 * (size_t)batch * o.size_a);
    o.off_norm = take(sizeof(double) * (size_t)batch * norm_parts(m, n));
    o.partial = std::max(partial_room(batch, o.r, o.r, std::max(o.ld_x, o.ld_t) / kSlabValues), partial_room(batch, o.r, o.l, o.ld_t / kSlabValues));
    o.off_partial = take(o.partial);
    o.total = off;
    return o;
}

struct NarrowLayout {
    size_t off_norm, off_images, off_factors, off_sums, total;
};
NarrowLayout narrow_layout(int64_t batch, int64_t m, int64_t n) {
    NarrowLayout o{};
    const size_t panels = (size_t)batch * ((std::max(m, n) + kNarrowPanel - 1) / kNarrowPanel);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes); return at; };
    o.off_norm = take(sizeof(double) * (size_t)batch * norm_parts(m, n));
    o.off_images = take(panels * kNarrowPanel * 256);
    o.off_factors = take((size_t)batch * 64 * 64 * 4);
    o.off_sums = take(panels * 64 * 64 * sizeof(float));
    o.total = off;
    return o;
}
// A shorter side of up to 64: panels, two launches a step, up to the length where one workgroup's sum of their parts takes what that saves
// (us, products and panels: 64 x 257 82 and 48, 64 x 1024 90 and 56, 64 x 4096 125 and 75, 32 x 8192 122 and 99, 64 x 16384 151 and 157; 64
// of 64 x 1024 157 and 100).
bool narrow_update(int64_t m, int64_t n) { return std::min(m, n) <= kSmallShorter && std::max(m, n) <= kNarrowLonger; }

bool small_update(int64_t m, int64_t n) { return std::min(m, n) <= kSmallShorter && std::max(m, n) <= kSmallLonger; }

// The power of two that slices of fp16 hold the iterates under: the largest up to 2^14 with which nothing overflows. The singular values
// start at most at one, p(x) = a x + b x^3 + c x^5 takes [0, r] into [0, max |p|], and no element of X, A = X X^T or a + b A + c A^2 is
// larger than its matrix's norm. -1: there is none, or a < 1: small values would shrink towards the 2^-25 that the slices leave of it.
int slice_shift(int steps, double a, double b, double c) {
    if (!(a >= 1.0)) return -1;
    double r = 1.0, top = 1.0;
    for (int i = 0; i < steps; ++i) {
        auto p = [&](double y) { return std::fabs(std::sqrt(y) * (a + y * (b + y * c))); };
        auto q = [&](double y) { return std::fabs(a + y * (b + y * c)); };
        const double y1 = r * r;
        double next = std::max(p(0.0), p(y1)), poly = std::max(q(0.0), q(y1));
        auto try_at = [&](double y) {
            if (y > 0.0 && y < y1) {
                next = std::max(next, p(y));
                poly = std::max(poly, q(y));
            }
        };
        // p' = a + 3 b y + 5 c y^2 and q' = b + 2 c y vanish
        const double d = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0) {
            if (d >= 0.0) {
                try_at((-3.0 * b + std::sqrt(d)) / (10.0 * c));
                try_at((-3.0 * b - std::sqrt(d)) / (10.0 * c));
            }
            try_at(-b / (2.0 * c));
        } else if (b != 0.0) {
            try_at(-a / (3.0 * b));
        }
        r = 1.01 * next;   // (room for roundings)
        top = std::max({top, r, r * r, poly});
        if (!(top < 4096.0)) return -1;
    }
    int shift = 14;
    while (shift > 0 && top * 1.05 * (double)(1 << shift) > 65504.0) --shift;
    return shift;
}

}  // namespace

extern "C" {

ozimmu_status_t ozimmu_q4_geometry(int64_t k, int group, int64_t* bytes, int64_t* groups) {
    if (!dim_ok(k) || !group_ok(group)) return OZIMMU_ERR_BAD_DIM;
    if (!bytes || !groups) return OZIMMU_ERR_NULL;
    *bytes = row_bytes(k);
    *groups = groups_of(k, group);
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_q4_split(int64_t n, int64_t k, int group, ozimmu_type_t type, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq,
                                ozimmu_type_t scale_type, void* scales, int64_t lds, void* stream) {
    if (!dim_ok(n) || !dim_ok(k) || !group_ok(group)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type) || !type_ok(scale_type)) return OZIMMU_ERR_BAD_TYPE;
    if (n == 0 || k == 0) return OZIMMU_OK;
    if (ldw < k || ldw > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!W) return OZIMMU_ERR_NULL;
    if (misaligned(W, size_of(type))) return OZIMMU_ERR_MISALIGNED;
    if (ozimmu_status_t rc = check_q4(k, group, codes, ldq, scales, scale_type, lds); rc != OZIMMU_OK) return rc;
    return hip_status(launch_q4_split(n, k, group, W, type, ldw, codes, ldq, scales, scale_type, lds, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_q4_expand(int64_t n, int64_t k, int group, ozimmu_type_t type, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds,
                                 void* W, int64_t ldw, void* stream) {
    if (!dim_ok(n) || !dim_ok(k) || !group_ok(group)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (n == 0 || k == 0) return OZIMMU_OK;
    if (ldw < k || ldw > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!W) return OZIMMU_ERR_NULL;
    if (misaligned(W, size_of(type))) return OZIMMU_ERR_MISALIGNED;
    if (ozimmu_status_t rc = check_q4(k, group, codes, ldq, scales, type, lds); rc != OZIMMU_OK) return rc;
    return hip_status(launch_q4_expand(n, k, group, codes, ldq, scales, type, lds, W, ldw, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_q4_workspace_bytes(int64_t t, int64_t n, int64_t k, int group, ozimmu_type_t type, int gradient, size_t* bytes) {
    if (!dim_ok(t) || !dim_ok(n) || !dim_ok(k) || !group_ok(group)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (!bytes) return OZIMMU_ERR_NULL;
    *bytes = t == 0 || n == 0 || k == 0 || way_of(t, n, k, group, type, gradient != 0) != Way::product ? 0 : operands(t, n, k, group, type, gradient != 0).total;
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_q4_gemm(int64_t t, int64_t n, int64_t k, int group, ozimmu_type_t type, const void* X, int64_t ldx, const uint8_t* codes,
                               int64_t ldq, const void* scales, int64_t lds, void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    return q4_product(false, t, n, k, group, type, X, ldx, codes, ldq, scales, lds, Y, ldy, workspace, workspace_bytes, stream);
}

ozimmu_status_t ozimmu_q4_gemm_grad(int64_t t, int64_t n, int64_t k, int group, ozimmu_type_t type, const void* dY, int64_t lddy, const uint8_t* codes,
                                    int64_t ldq, const void* scales, int64_t lds, void* dX, int64_t lddx, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    return q4_product(true, t, n, k, group, type, dY, lddy, codes, ldq, scales, lds, dX, lddx, workspace, workspace_bytes, stream);
}

ozimmu_status_t ozimmu_orthogonalize_workspace_bytes(int64_t batch, int64_t m, int64_t n, size_t* bytes) {
    if (!dim_ok(m) || !dim_ok(n) || batch < 0 || batch > OZIMMU_MAX_BATCH) return OZIMMU_ERR_BAD_DIM;
    if (!bytes) return OZIMMU_ERR_NULL;
    *bytes = batch == 0 || m == 0 || n == 0 || small_update(m, n) ? 0 : narrow_update(m, n) ? narrow_layout(batch, m, n).total : orth_layout(batch, m, n).total;
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_orthogonalize(int64_t batch, int64_t m, int64_t n, ozimmu_type_t type, const void* G, int64_t ldg, int64_t stride_g, void* X,
                                     int64_t ldx, int64_t stride_x, int steps, double a, double b, double c, double eps, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    if (!dim_ok(m) || !dim_ok(n) || batch < 0 || batch > OZIMMU_MAX_BATCH) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (steps < 1 || steps > OZIMMU_MAX_STEPS || !std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !(eps >= 0.0) || !std::isfinite(eps))
        return OZIMMU_ERR_BAD_POLYNOMIAL;
    const int shift = slice_shift(steps, a, b, c);
    if (shift < 0) return OZIMMU_ERR_BAD_POLYNOMIAL;
    if (batch == 0 || m == 0 || n == 0) return OZIMMU_OK;
    if (ldg < n || ldx < n || (batch > 1 && (stride_g < 0 || stride_x < (m - 1) * ldx + n))) return OZIMMU_ERR_BAD_LD;
    if (!G || !X) return OZIMMU_ERR_NULL;
    if (misaligned(G, size_of(type)) || misaligned(X, size_of(type))) return OZIMMU_ERR_MISALIGNED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (small_update(m, n)) return hip_status(launch_orthogonalize_small(batch, m, n, G, type, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st));
    if (narrow_update(m, n)) {
        const NarrowLayout o = narrow_layout(batch, m, n);
        if (!workspace || misaligned(workspace, OZIMMU_WORKSPACE_ALIGN) || workspace_bytes < o.total) return OZIMMU_ERR_WORKSPACE;
        unsigned char* base = static_cast<unsigned char*>(workspace);
        double* norms = reinterpret_cast<double*>(base + o.off_norm);
        hipError_t e = launch_norm_partials(batch, m, n, G, type, ldg, stride_g, norms, st);
        if (e == hipSuccess)
            e = launch_orthogonalize_narrow(batch, m, n, G, type, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, norms, base + o.off_images, base + o.off_factors,
                                            reinterpret_cast<float*>(base + o.off_sums), st);
        return hip_status(e);
    }
    const OrthLayout o = orth_layout(batch, m, n);
    if (!workspace || misaligned(workspace, OZIMMU_WORKSPACE_ALIGN) || workspace_bytes < o.total) return OZIMMU_ERR_WORKSPACE;
    unsigned char* base = static_cast<unsigned char*>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<unsigned short*>(base + off); };
    double* partials = reinterpret_cast<double*>(base + o.off_norm);
    const bool tall = m > n;

    hipError_t e = launch_norm_partials(batch, m, n, G, type, ldg, stride_g, partials, st);
    unsigned short *x = at(o.off_x), *xt = at(o.off_t[0]);
    if (e == hipSuccess)
        e = tall ? launch_normalised_slices(batch, m, n, G, type, ldg, stride_g, partials, eps, shift, xt, o.ld_t, o.size_t_, x, o.ld_x, o.size_x, st)
                 : launch_normalised_slices(batch, m, n, G, type, ldg, stride_g, partials, eps, shift, x, o.ld_x, o.size_x, xt, o.ld_t, o.size_t_, st);
    const float down = (float)std::ldexp(1.0, -shift);   // a sum of products of two scaled values is scaled twice
    for (int i = 0; i < steps && e == hipSuccess; ++i) {
        unsigned short *now = at(o.off_t[i & 1]), *next = at(o.off_t[(i & 1) ^ 1]);
        NtArgs g{};
        g.batch = (int)batch;
        g.partial = reinterpret_cast<float*>(base + o.off_partial);
        g.partial_bytes = o.partial;
        g.m = g.n = (int)o.r;
        g.symmetric = true;
        g.factor = down;
        // A = X X^T
        g.P = g.Q = x;
        g.ldp = g.ldq = o.ld_x;
        g.batch_p = g.batch_q = o.size_x;
        g.slabs = (int)(o.ld_x / kSlabValues);
        g.C = g.CT = at(o.off_a);
        g.ldc = g.ldct = o.ld_t;
        g.batch_c = g.batch_ct = o.size_a;
        e = launch_nt_product(g, 2, false, kOutSlices, st);
        if (e != hipSuccess) break;
        // a + b A + c A^2
        g.P = g.Q = g.in = at(o.off_a);
        g.ldp = g.ldq = o.ld_t;
        g.batch_p = g.batch_q = o.size_a;
        g.slabs = (int)(o.ld_t / kSlabValues);
        g.C = g.CT = at(o.off_q);
        g.factor = (float)(c * (double)down);
        g.beta = (float)b;
        g.diagonal = (float)std::ldexp(a, shift);
        e = launch_nt_product(g, 2, false, kOutSlices, st);
        if (e != hipSuccess) break;
        // times X
        const bool last = i + 1 == steps;
        NtArgs u{};
        u.batch = (int)batch;
        u.partial = g.partial;
        u.partial_bytes = o.partial;
        u.slabs = (int)(o.ld_t / kSlabValues);
        u.ldp = u.ldq = o.ld_t;
        if (last && tall) {   // X^T (a + b A + c A^2), as it lies in the result
            u.P = now;
            u.batch_p = o.size_t_;
            u.Q = at(o.off_q);
            u.batch_q = o.size_a;
            u.m = (int)o.l;
            u.n = (int)o.r;
        } else {
            u.P = at(o.off_q);
            u.batch_p = o.size_a;
            u.Q = now;
            u.batch_q = o.size_t_;
            u.m = (int)o.r;
            u.n = (int)o.l;
        }
        if (last) {
            u.factor = down * down;
            u.out = X;
            u.ldo = ldx;
            u.batch_o = stride_x;
            e = launch_nt_product(u, 2, false, type == OZIMMU_F32 ? kOutF32 : type == OZIMMU_BF16 ? kOutBf16 : kOutF16, st);
        } else {
            u.factor = down;
            u.C = x;
            u.ldc = o.ld_x;
            u.batch_c = o.size_x;
            u.CT = next;
            u.ldct = o.ld_t;
            u.batch_ct = o.size_t_;
            e = launch_nt_product(u, 2, false, kOutSlices, st);
        }
    }
    return hip_status(e);
}

}  // extern "C"
