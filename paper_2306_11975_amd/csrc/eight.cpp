// C ABI of the products in 8-bit floating point and of the operators for mixtures of experts: argument checks, workspace layout, choice and
// sequencing of kernels. What computes is in f8_cut.hip, f8_few.hip, f8_product.h, route.hip and experts.hip.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "eight_internal.h"

using namespace ozimmu;

namespace {

constexpr int64_t kMaxDim = OZIMMU_MAX_DIM;

bool dim_ok(int64_t x) { return x >= 0 && x <= kMaxDim; }
bool type_ok(int type) { return type == OZIMMU_F32 || type == OZIMMU_BF16 || type == OZIMMU_F16; }
bool scale_ok(int type) { return type == OZIMMU_F32 || type == OZIMMU_E8M0; }
size_t size_of(int type) { return type == OZIMMU_F32 ? 4 : type == OZIMMU_E4M3 || type == OZIMMU_E8M0 ? 1 : 2; }
size_t align_up(size_t x) { return (x + OZIMMU_WORKSPACE_ALIGN - 1) / OZIMMU_WORKSPACE_ALIGN * OZIMMU_WORKSPACE_ALIGN; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
ozimmu_status_t hip_status(hipError_t e) { return e == hipSuccess ? OZIMMU_OK : OZIMMU_ERR_HIP; }

ozimmu_status_t check_codes(int64_t k, const void* codes, int64_t ldq) {
    if (ldq < f8_row_bytes(k) || ldq % 16 != 0 || ldq > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!codes) return OZIMMU_ERR_NULL;
    return misaligned(codes, 16) ? OZIMMU_ERR_MISALIGNED : OZIMMU_OK;
}
ozimmu_status_t check_scales(int64_t k, int scale_type, const void* scales, int64_t lds) {
    if (lds > OZIMMU_MAX_LD || (scale_type == OZIMMU_F32 ? lds < f8_groups(k) : lds < f8_scale_bytes(k) || lds % 4 != 0)) return OZIMMU_ERR_BAD_LD;
    if (!scales) return OZIMMU_ERR_NULL;
    return misaligned(scales, 4) ? OZIMMU_ERR_MISALIGNED : OZIMMU_OK;
}
ozimmu_status_t check_matrix(const void* M, int type, int64_t ld, int64_t cols) {
    if (ld < cols || ld > OZIMMU_MAX_LD) return OZIMMU_ERR_BAD_LD;
    if (!M) return OZIMMU_ERR_NULL;
    return misaligned(M, size_of(type)) ? OZIMMU_ERR_MISALIGNED : OZIMMU_OK;
}

bool ws_ok(const void* ws, size_t bytes, size_t needed) { return needed == 0 || (ws && !misaligned(ws, OZIMMU_WORKSPACE_ALIGN) && bytes >= needed); }

enum { kGemm = 0, kGemmGrad = 1, kWeightGrad = 2 };

// Few rows: straight from memory, 16 rows of tokens at a time, without a cut of its own (f8_few.hip). Cut and tiles take two launches, but stream the
// weights through LDS by whole lines and read the tokens once for every 64 columns. us, few rows against tiles, tokens and results of bf16:
// 2048 x 2048 1 row 5.6, 9.5, 64 rows 8.5, 11.2, 128 13.6, 13.6; 4096 x 4096 16 rows 9.8, 13.3, 32 12.6, 13.4, 64 22, 15; 8192 x 4096 1 row 10.4,
// 13.6, 16 rows 12.6, 14.6, 32 22, 15; 16 experts of 2048 x 1024 8 rows 7.4, 10.2, 64 rows 12.5, 11.4. 32 bits: 2048 x 2048 64 rows 10.0, 11.4, 128 17,
// 13; 8192 x 4096 16 rows 15.9, 15.6; 2048 x 8192 1 row 11.7, 13.3, 16 rows 21, 14. Given codes: 2048 x 2048 64 rows 7.1, 7.6; 8192 x 4096 16
// rows 11.0, 11.3. The limit is where they meet, in weights read. (The answer turns once as rows grow, so that a workspace serves fewer.)
bool few_rows(int op, int64_t rows, int64_t n, int64_t k, int64_t experts, int type) {
    if (op == kGemm && type == OZIMMU_E4M3) k = f8_row_bytes(k);      // (a caller may know codes' length by whole runs alone, when sizing the workspace or when calling)
    const double runs = experts ? (double)(rows / 16 + std::min(experts, rows)) : rows <= 16 ? 0.5 : (double)((rows + 15) / 16);
    return runs * (double)n * (double)k <= 16777216.0;
}

// What a call keeps in its workspace: the cut rows (P), for gradients the transposed weights or the cut columns of X (Q).
struct Layout {
    int64_t ldp, ldsp, ldq, ldsq;
    size_t off_p, off_sp, off_q, off_sq, off_partial, partial, total;
};
Layout layout(int op, int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts, int type) {
    Layout o{};
    size_t off = 0;
    auto take = [&](int64_t bytes) { const size_t at = off; off = align_up(off + (size_t)bytes); return at; };
    const int64_t e = std::max<int64_t>(experts, 1);
    if (op == kWeightGrad) {
        o.ldsp = o.ldsq = most_token_runs(rows, experts);
        o.ldp = o.ldq = o.ldsp * kRun;
        o.off_p = take(n * o.ldp);
        o.off_sp = take(n * o.ldsp);
        o.off_q = take(k * o.ldq);
        o.off_sq = take(k * o.ldsq);
    } else {
        const int64_t inner = op == kGemm ? k : n;
        o.ldp = f8_row_bytes(inner);
        o.ldsp = f8_scale_bytes(inner);
        if (type != OZIMMU_E4M3 && (op == kGemmGrad || !few_rows(op, rows, n, k, experts, type))) {
            o.off_p = take((op == kGemm ? t : rows) * o.ldp);
            o.off_sp = take((op == kGemm ? t : rows) * o.ldsp);
        }
        if (op == kGemmGrad) {
            o.ldq = f8_row_bytes(n);
            o.ldsq = f8_scale_bytes(n);
            o.off_q = take(e * k * o.ldq);
            o.off_sq = take(e * f8_groups(k) * o.ldsq * 4);
        }
    }
    if (experts == 0 && !(op != kWeightGrad && few_rows(op, rows, n, k, experts, type)))
        o.partial = op == kWeightGrad ? f8_partial_room(n, k, f8_groups(rows)) : f8_partial_room(rows, op == kGemm ? n : k, f8_groups(op == kGemm ? k : n));
    o.off_partial = take((int64_t)o.partial);
    o.total = off;
    return o;
}

ozimmu_status_t check_sizes(int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts) {
    if (!dim_ok(t) || !dim_ok(rows) || !dim_ok(n) || !dim_ok(k) || experts < 0 || experts > OZIMMU_MAX_EXPERTS) return OZIMMU_ERR_BAD_DIM;
    return experts == 0 && t != rows ? OZIMMU_ERR_BAD_DIM : OZIMMU_OK;
}
ozimmu_status_t check_experts(int64_t t, int64_t rows, int64_t experts, const int* offsets, const int* source) {
    if (experts == 0) return offsets || source ? OZIMMU_ERR_BAD_DIM : OZIMMU_OK;
    if (!offsets) return OZIMMU_ERR_NULL;
    if (!source && t != rows) return OZIMMU_ERR_BAD_DIM;
    return misaligned(offsets, 4) || (source && misaligned(source, 4)) ? OZIMMU_ERR_MISALIGNED : OZIMMU_OK;
}

// `few`: as few_rows has it (never for weights' gradients, whose codes lie in the workspace)
hipError_t product(const F8Args& a, bool few, hipStream_t st) {
    if (few) return launch_f8_few(a, st);
    const F8Choice c = choose_f8_tile(a);
    if (c.shape == kF8Shapes) return hipErrorInvalidConfiguration;
    if (a.out_type == OZIMMU_F32) return launch_f8_tiles_exact(a, c, st);
    return c.shape == kF8Tile256 ? launch_f8_large(a, st) : launch_f8_tiles(a, c, st);
}

ozimmu_status_t f8_product(int op, int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts, int type, const void* V, int64_t ldv, const uint8_t* v_scales, int64_t ldvs,
                           const uint8_t* codes, int64_t ldq, int scale_type, const void* scales, int64_t lds, const int* offsets, const int* source, int out_type, void* R, int64_t ldr, void* ws,
                           size_t ws_bytes, void* stream) {
    if (ozimmu_status_t rc = check_sizes(t, rows, n, k, experts); rc != OZIMMU_OK) return rc;
    if (!(type_ok(type) || type == OZIMMU_E4M3) || !scale_ok(scale_type) || !type_ok(out_type)) return OZIMMU_ERR_BAD_TYPE;
    const int64_t inner = op == kGemm ? k : n, outer = op == kGemm ? n : k;
    if (rows == 0 || outer == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_experts(t, rows, experts, offsets, source); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_matrix(R, out_type, ldr, outer); rc != OZIMMU_OK) return rc;
    const Layout o = layout(op, t, rows, n, k, experts, type);
    if (inner > 0 && t > 0) {
        if (type == OZIMMU_E4M3) {
            if (ozimmu_status_t rc = check_codes(inner, V, ldv); rc != OZIMMU_OK) return rc;
            if (ozimmu_status_t rc = check_scales(inner, OZIMMU_E8M0, v_scales, ldvs); rc != OZIMMU_OK) return rc;
        } else if (ozimmu_status_t rc = check_matrix(V, type, ldv, inner); rc != OZIMMU_OK) {
            return rc;
        }
        if (ozimmu_status_t rc = check_codes(k, codes, ldq); rc != OZIMMU_OK) return rc;
        if (ozimmu_status_t rc = check_scales(k, scale_type, scales, lds); rc != OZIMMU_OK) return rc;
        const int64_t ldp = type == OZIMMU_E4M3 ? ldv : o.ldp, ldsp = type == OZIMMU_E4M3 ? ldvs : o.ldsp;
        if (source && (t * ldp >= int64_t(1) << 32 || t * ldsp >= int64_t(1) << 32)) return OZIMMU_ERR_BAD_LD;
        if (!ws_ok(ws, ws_bytes, o.total)) return OZIMMU_ERR_WORKSPACE;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* base = static_cast<unsigned char*>(ws);
    F8Args a{};
    a.rows = (int)rows;
    a.t = (int)t;
    a.n = (int)outer;
    a.experts = (int)experts;
    a.offsets = offsets;
    a.source = source;
    a.scale_type = scale_type;
    a.out = R;
    a.out_type = out_type;
    a.ldo = ldr;
    a.V = V;
    a.v_type = type;
    a.ldv = ldv;
    a.k = inner;
    const bool few = few_rows(op, rows, n, k, experts, type);
    if (inner == 0 || t == 0) return hip_status(launch_f8_few(a, st));   // zeros
    a.slabs = (int)f8_groups(inner);
    hipError_t e = hipSuccess;
    if (type == OZIMMU_E4M3) {
        a.P = static_cast<const uint8_t*>(V);
        a.ldp = ldv;
        a.sp = v_scales;
        a.ldsp = ldvs;
    } else if (op == kGemmGrad || !few) {      // (gradients: the cut goes with the turn of the weights)
        a.P = base + o.off_p;
        a.ldp = o.ldp;
        a.sp = base + o.off_sp;
        a.ldsp = o.ldsp;
        if (op == kGemm) e = launch_f8_split(t, inner, 1, V, type, ldv, base + o.off_p, o.ldp, base + o.off_sp, o.ldsp, st);
    }
    if (op == kGemm) {
        a.Q = codes;
        a.ldq = ldq;
        a.sq = scales;
        a.ldsq = lds;
    } else {
        a.Q = base + o.off_q;
        a.ldq = o.ldq;
        a.sq = base + o.off_sq;
        a.ldsq = o.ldsq;
        const bool cut = type != OZIMMU_E4M3;
        if (cut) {
            a.V = a.P;
            a.v_type = OZIMMU_E4M3;
            a.ldv = a.ldp;
        }
        e = launch_f8_gradient_operands(std::max<int64_t>(experts, 1), n, k, codes, ldq, scale_type, scales, lds, base + o.off_q, base + o.off_sq, rows, V, type, ldv,
                                        cut ? base + o.off_p : nullptr, base + o.off_sp, st);
    }
    if (o.partial) a.partial = reinterpret_cast<float*>(base + o.off_partial);
    a.partial_bytes = o.partial;
    if (e == hipSuccess) e = product(a, few, st);
    return hip_status(e);
}

ozimmu_status_t check_route(int64_t t, int64_t experts, int top, int type, int score, double scale) {
    if (!dim_ok(t) || experts < 1 || experts > OZIMMU_MAX_EXPERTS || top < 1 || top > OZIMMU_MAX_CHOICES || top > experts || !std::isfinite((float)scale)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type) || (score != OZIMMU_SOFTMAX && score != OZIMMU_SIGMOID)) return OZIMMU_ERR_BAD_TYPE;
    return OZIMMU_OK;
}
ozimmu_status_t check_pairs(int64_t t, int top) {
    return !dim_ok(t) || top < 1 || top > OZIMMU_MAX_CHOICES ? OZIMMU_ERR_BAD_DIM : OZIMMU_OK;
}

}  // namespace

namespace ozimmu {

// Room for the sums of shared tiles: at most eight workgroups to a tile, four slabs at least to each.
size_t f8_partial_room(int64_t rows, int64_t n, int64_t slabs) {
    const int64_t parts = std::min<int64_t>(8, slabs / 4);
    if (parts < 2) return 0;
    const double bytes = (double)pad_to(rows, 128) * (double)pad_to(n, 128) * (double)parts * sizeof(float);
    return bytes < (double)kPartialBytes ? (size_t)bytes : kPartialBytes;
}

// By an estimate, in us: of a round of tiles, what the fullest compute unit takes for a slab, from `alone` (one workgroup) to `full` (`slots` / 256),
// and what a round takes beside its slabs. Fitted to 35 products with 16-bit results and 14 with 32-bit ones, 64 to 16384 rows, 16 to 64 slabs, dense
// and over 8 to 128 experts. 4096 x 4096 x 4096 by tiles of 256, 128, 64 x 128, 64, 32 x 64: 60, 76, 88, 119, 147; 1024 x 4096 x 4096: 42, 31, 26, 33,
// 44; 512 x 2048 x 2048: 24, 16, 11, 9.1, 8.8; 8192 rows of 64 experts, 1024 x 1024: 25, 30, 28, 30, -. Over experts a tile's rows end with the
// expert's: half a tile is counted for each.
F8Choice choose_f8_tile(const F8Args& a) {
    struct Shape {
        int rows, cols, slots;
        double alone, full, round, call;
    };
    static const Shape half[kF8Shapes] = {{256, 256, 256, 0.95, 1.5, 10.0, 5.0}, {128, 128, 512, 0.80, 1.10, 3.5, 3.0}, {64, 128, 768, 0.62, 0.87, 3.2, 2.5}, {64, 64, 1280, 0.38, 1.13, 1.3, 2.0},
                                          {32, 64, 1536, 0.38, 0.83, 1.0, 2.0}};
    static const Shape wide[kF8Shapes] = {{256, 256, 0, 0.0, 0.0, 0.0, 0.0}, {128, 128, 512, 1.5, 2.3, 4.0, 3.0}, {64, 128, 768, 0.9, 1.95, 3.0, 2.5}, {64, 64, 1024, 0.58, 1.43, 1.3, 2.0},
                                          {32, 64, 1536, 0.50, 1.25, 1.0, 2.0}};
    F8Choice best{kF8Shapes, 0, 1, a.slabs};      // (none: more tiles than a launch has)
    double best_us = 1e30;
    for (int i = 0; i < kF8Shapes; ++i) {
        const Shape& s = a.out_type == OZIMMU_F32 ? wide[i] : half[i];
        if (s.slots == 0 || (i == kF8Tile256 && a.scale_type == OZIMMU_F32)) continue;
        const double columns = (double)((a.n + s.cols - 1) / s.cols), tiles_m = (double)((a.rows + s.rows - 1) / s.rows), used = (double)std::min(a.experts, a.along_rows ? a.t : a.rows);
        double all = tiles_m * columns, slabs = (double)a.slabs;
        if (a.experts && a.along_rows) {
            all *= used;
            slabs = used > 0.0 ? (double)a.t / 128.0 / used + 0.5 : 0.0;
        } else if (a.experts) {
            all = std::max((double)a.rows / s.rows + 0.5 * used, used) * columns;
        }
        if (all > (double)(INT32_MAX / 64)) continue;
        auto round_us = [&](double workgroups, double walk) {
            if (workgroups <= 0.0) return 0.0;
            const double most = (double)(s.slots / 256), deepest = std::ceil(workgroups / 256.0);
            const double share = most > 1.0 ? (deepest - 1.0) / (most - 1.0) : workgroups / 256.0;
            return s.round + walk * (s.alone + (s.full - s.alone) * share);
        };
        const double rounds = std::floor(all / s.slots), rest = all - rounds * s.slots;
        const double whole_us = s.call + rounds * round_us(s.slots, slabs) + round_us(rest, slabs);
        if (whole_us < best_us) {
            best_us = whole_us;
            best = F8Choice{i, (int)(a.experts ? 0.0 : all), 1, a.slabs};
        }
        if (a.experts || !a.partial || rest <= 0.0 || i == kF8Tile256) continue;
        // the tiles of a last round that is not full may be shared, at the price of their sums' way through memory and of a launch
        for (int parts = 2; parts <= 8 && rest * parts <= s.slots; ++parts) {
            const int walk = (int)pad_to((a.slabs + parts - 1) / parts, 4), taken = (a.slabs + walk - 1) / walk;
            const double bytes = rest * parts * s.rows * s.cols * sizeof(float);
            if (taken != parts || bytes > (double)a.partial_bytes) continue;
            const double us = s.call + rounds * round_us(s.slots, slabs) + round_us(rest * parts, walk) + 2.5 + 2.0 * bytes / 4.0e6;
            if (us < best_us) {
                best_us = us;
                best = F8Choice{i, (int)(rounds * s.slots), parts, walk};
            }
        }
    }
    return best;
}

}  // namespace ozimmu

extern "C" {

ozimmu_status_t ozimmu_f8_geometry(int64_t k, int64_t* row_bytes, int64_t* scale_bytes) {
    if (!dim_ok(k)) return OZIMMU_ERR_BAD_DIM;
    if (!row_bytes || !scale_bytes) return OZIMMU_ERR_NULL;
    *row_bytes = f8_row_bytes(k);
    *scale_bytes = f8_scale_bytes(k);
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_f8_split(int64_t n, int64_t k, int block_rows, ozimmu_type_t type, const void* W, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds, void* stream) {
    if (!dim_ok(n) || !dim_ok(k) || (block_rows != 1 && block_rows != 128)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (n == 0 || k == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_matrix(W, type, ldw, k); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_codes(k, codes, ldq); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_scales(k, OZIMMU_E8M0, scales, lds); rc != OZIMMU_OK) return rc;
    return hip_status(launch_f8_split(n, k, block_rows, W, type, ldw, codes, ldq, scales, lds, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_f8_expand(int64_t n, int64_t k, int block_rows, const uint8_t* codes, int64_t ldq, ozimmu_type_t scale_type, const void* scales, int64_t lds, ozimmu_type_t type, void* W,
                                 int64_t ldw, void* stream) {
    if (!dim_ok(n) || !dim_ok(k) || (block_rows != 1 && block_rows != 128)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type) || !scale_ok(scale_type)) return OZIMMU_ERR_BAD_TYPE;
    if (n == 0 || k == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_matrix(W, type, ldw, k); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_codes(k, codes, ldq); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_scales(k, scale_type, scales, lds); rc != OZIMMU_OK) return rc;
    return hip_status(launch_f8_expand(n, k, block_rows, codes, ldq, scale_type, scales, lds, W, type, ldw, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_f8_workspace_bytes(int op, int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts, ozimmu_type_t type, size_t* bytes) {
    if (op < kGemm || op > kWeightGrad) return OZIMMU_ERR_BAD_DIM;
    if (ozimmu_status_t rc = check_sizes(t, rows, n, k, experts); rc != OZIMMU_OK) return rc;
    if (!type_ok(type) && !(type == OZIMMU_E4M3 && op != kWeightGrad)) return OZIMMU_ERR_BAD_TYPE;
    if (!bytes) return OZIMMU_ERR_NULL;
    *bytes = t == 0 || rows == 0 || n == 0 || k == 0 ? 0 : layout(op, t, rows, n, k, experts, type).total;
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_f8_gemm(int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts, ozimmu_type_t type, const void* X, int64_t ldx, const uint8_t* x_scales, int64_t ldxs,
                               const uint8_t* codes, int64_t ldq, ozimmu_type_t scale_type, const void* scales, int64_t lds, const int* offsets, const int* source, ozimmu_type_t out_type, void* Y,
                               int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    return f8_product(kGemm, t, rows, n, k, experts, type, X, ldx, x_scales, ldxs, codes, ldq, scale_type, scales, lds, offsets, source, out_type, Y, ldy, workspace, workspace_bytes, stream);
}

ozimmu_status_t ozimmu_f8_gemm_grad(int64_t rows, int64_t n, int64_t k, int64_t experts, ozimmu_type_t type, const void* dY, int64_t lddy, const uint8_t* dy_scales, int64_t lddys,
                                    const uint8_t* codes, int64_t ldq, ozimmu_type_t scale_type, const void* scales, int64_t lds, const int* offsets, ozimmu_type_t out_type, void* dX, int64_t lddx,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    return f8_product(kGemmGrad, rows, rows, n, k, experts, type, dY, lddy, dy_scales, lddys, codes, ldq, scale_type, scales, lds, offsets, nullptr, out_type, dX, lddx, workspace, workspace_bytes,
                      stream);
}

ozimmu_status_t ozimmu_f8_weight_grad(int64_t t, int64_t rows, int64_t n, int64_t k, int64_t experts, ozimmu_type_t type, const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                      const int* offsets, const int* source, ozimmu_type_t out_type, void* dW, int64_t lddw, void* workspace, size_t workspace_bytes, void* stream) {
    if (ozimmu_status_t rc = check_sizes(t, rows, n, k, experts); rc != OZIMMU_OK) return rc;
    if (!type_ok(type) || !type_ok(out_type)) return OZIMMU_ERR_BAD_TYPE;
    if (n == 0 || k == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_experts(t, rows, experts, offsets, source); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_matrix(dW, out_type, lddw, k); rc != OZIMMU_OK) return rc;
    const Layout o = layout(kWeightGrad, t, rows, n, k, experts, type);
    const bool empty = rows == 0 || t == 0;
    if (!empty) {
        if (ozimmu_status_t rc = check_matrix(dY, type, lddy, n); rc != OZIMMU_OK) return rc;
        if (ozimmu_status_t rc = check_matrix(X, type, ldx, k); rc != OZIMMU_OK) return rc;
        if (!ws_ok(workspace, workspace_bytes, o.total)) return OZIMMU_ERR_WORKSPACE;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* base = static_cast<unsigned char*>(workspace);
    F8Args a{};
    a.along_rows = true;
    a.rows = (int)n;
    a.t = (int)rows;
    a.n = (int)k;
    a.experts = (int)experts;
    a.offsets = offsets;
    a.scale_type = OZIMMU_E8M0;
    a.out = dW;
    a.out_type = out_type;
    a.ldo = lddw;
    if (empty) {
        a.t = 0;   // no rows, so no slabs
        return hip_status(product(a, false, st));
    }
    if (o.partial) a.partial = reinterpret_cast<float*>(base + o.off_partial);
    a.partial_bytes = o.partial;
    a.slabs = (int)f8_groups(rows);
    a.P = base + o.off_p;
    a.sp = base + o.off_sp;
    a.ldp = o.ldp;
    a.ldsp = o.ldsp;
    a.Q = base + o.off_q;
    a.sq = base + o.off_sq;
    a.ldq = o.ldq;
    a.ldsq = o.ldsq;
    const F8Columns dy{dY, lddy, n, (int)rows, nullptr, base + o.off_p, base + o.off_sp}, x{X, ldx, k, (int)t, source, base + o.off_q, base + o.off_sq};
    hipError_t e = launch_f8_cut_tokens(rows, experts, offsets, type, dy, x, o.ldsp, st);
    if (e == hipSuccess) e = product(a, false, st);
    return hip_status(e);
}

ozimmu_status_t ozimmu_route(int64_t t, int64_t experts, int top, ozimmu_type_t type, const void* logits, int64_t ldl, const float* bias, ozimmu_score_t score, int groups, int top_groups,
                             int renormalize, double scale, int* indices, float* weights, void* stream) {
    if (ozimmu_status_t rc = check_route(t, experts, top, type, score, scale); rc != OZIMMU_OK) return rc;
    if (groups < 1 || groups > experts || experts % groups != 0 || top_groups < 1 || top_groups > groups) return OZIMMU_ERR_BAD_DIM;
    if (t == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_matrix(logits, type, ldl, experts); rc != OZIMMU_OK) return rc;
    if (!indices || !weights) return OZIMMU_ERR_NULL;
    if (misaligned(indices, 4) || misaligned(weights, 4) || (bias && misaligned(bias, 4))) return OZIMMU_ERR_MISALIGNED;
    const RouteArgs a{(int)t, (int)experts, top, logits, type, ldl, bias, score == OZIMMU_SIGMOID, groups, top_groups, renormalize != 0, (float)scale};
    return hip_status(launch_route(a, indices, weights, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_route_grad(int64_t t, int64_t experts, int top, ozimmu_type_t type, const void* logits, int64_t ldl, const int* indices, const float* dweights, ozimmu_score_t score,
                                  int renormalize, double scale, void* dlogits, int64_t lddl, void* stream) {
    if (ozimmu_status_t rc = check_route(t, experts, top, type, score, scale); rc != OZIMMU_OK) return rc;
    if (t == 0) return OZIMMU_OK;
    if (ozimmu_status_t rc = check_matrix(logits, type, ldl, experts); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_matrix(dlogits, type, lddl, experts); rc != OZIMMU_OK) return rc;
    if (!indices || !dweights) return OZIMMU_ERR_NULL;
    if (misaligned(indices, 4) || misaligned(dweights, 4)) return OZIMMU_ERR_MISALIGNED;
    const RouteArgs a{(int)t, (int)experts, top, logits, type, ldl, nullptr, score == OZIMMU_SIGMOID, 1, 1, renormalize != 0, (float)scale};
    return hip_status(launch_route_grad(a, indices, dweights, dlogits, lddl, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_expert_order_workspace_bytes(int64_t t, int top, int64_t experts, size_t* bytes) {
    if (ozimmu_status_t rc = check_pairs(t, top); rc != OZIMMU_OK) return rc;
    if (experts < 1 || experts > OZIMMU_MAX_EXPERTS) return OZIMMU_ERR_BAD_DIM;
    if (!bytes) return OZIMMU_ERR_NULL;
    *bytes = expert_order_bytes(t * top, (int)experts);
    return OZIMMU_OK;
}

ozimmu_status_t ozimmu_expert_order(int64_t t, int top, int64_t experts, const int* indices, int* offsets, int* source, int* place, void* workspace, size_t workspace_bytes, void* stream) {
    if (ozimmu_status_t rc = check_pairs(t, top); rc != OZIMMU_OK) return rc;
    if (experts < 1 || experts > OZIMMU_MAX_EXPERTS) return OZIMMU_ERR_BAD_DIM;
    if (!offsets || (t > 0 && (!indices || !source || !place))) return OZIMMU_ERR_NULL;
    if (misaligned(indices, 4) || misaligned(offsets, 4) || misaligned(source, 4) || misaligned(place, 4)) return OZIMMU_ERR_MISALIGNED;
    if (!ws_ok(workspace, workspace_bytes, expert_order_bytes(t * top, (int)experts))) return OZIMMU_ERR_WORKSPACE;
    return hip_status(launch_expert_order((int)t, top, (int)experts, indices, offsets, source, place, static_cast<int*>(workspace), static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_expert_combine(int64_t t, int top, int64_t rows, int64_t n, ozimmu_type_t type, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy,
                                      void* stream) {
    if (ozimmu_status_t rc = check_pairs(t, top); rc != OZIMMU_OK) return rc;
    if (rows < 0 || rows > INT32_MAX || !dim_ok(n)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (t == 0 || n == 0) return OZIMMU_OK;
    if (rows > 0)
        if (ozimmu_status_t rc = check_matrix(O, type, ldo, n); rc != OZIMMU_OK) return rc;
    if (ozimmu_status_t rc = check_matrix(Y, type, ldy, n); rc != OZIMMU_OK) return rc;
    if (!place) return OZIMMU_ERR_NULL;
    if (misaligned(place, 4) || (weights && misaligned(weights, 4))) return OZIMMU_ERR_MISALIGNED;
    return hip_status(launch_expert_combine((int)t, top, (int)rows, n, type, O, ldo, place, weights, Y, ldy, static_cast<hipStream_t>(stream)));
}

ozimmu_status_t ozimmu_expert_combine_grad(int64_t t, int top, int64_t rows, int64_t n, ozimmu_type_t type, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place,
                                           const float* weights, void* dO, int64_t lddo, float* dweights, void* stream) {
    if (ozimmu_status_t rc = check_pairs(t, top); rc != OZIMMU_OK) return rc;
    if (rows < 0 || rows > INT32_MAX || !dim_ok(n)) return OZIMMU_ERR_BAD_DIM;
    if (!type_ok(type)) return OZIMMU_ERR_BAD_TYPE;
    if (t == 0) return OZIMMU_OK;
    if (n > 0) {
        if (ozimmu_status_t rc = check_matrix(dY, type, lddy, n); rc != OZIMMU_OK) return rc;
        if (rows > 0) {
            if (ozimmu_status_t rc = check_matrix(O, type, ldo, n); rc != OZIMMU_OK) return rc;
            if (ozimmu_status_t rc = check_matrix(dO, type, lddo, n); rc != OZIMMU_OK) return rc;
        }
    }
    if (!place || !weights || !dweights) return OZIMMU_ERR_NULL;
    if (misaligned(place, 4) || misaligned(weights, 4) || misaligned(dweights, 4)) return OZIMMU_ERR_MISALIGNED;
    return hip_status(launch_expert_combine_grad((int)t, top, (int)rows, n, type, dY, lddy, O, ldo, place, weights, dO, lddo, dweights, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
