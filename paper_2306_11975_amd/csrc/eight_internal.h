// What the operators in 8-bit floating point (f8_cut.hip, f8_few.hip, f8_product*.hip) and those of mixtures of experts (route.hip,
// experts.hip) share with their entry points (eight.cpp).
#pragma once

#include "weights_internal.h"

namespace ozimmu {

constexpr int kRun = 128;   // positions that share a scale
inline int64_t f8_row_bytes(int64_t k) { return pad_to(k, kRun); }
inline int64_t f8_groups(int64_t k) { return (k + kRun - 1) / kRun; }
inline int64_t f8_scale_bytes(int64_t k) { return pad_to(f8_groups(k), 4); }

// Rows along the tokens (the transposed operands of a weights' gradient): every expert's runs begin at a multiple of four, so that their scales
// can be read four at a time. At most so many runs.
inline int64_t most_token_runs(int64_t rows, int64_t experts) { return pad_to(f8_groups(rows), 4) + 4 * (experts < rows ? experts : rows); }

// f8_cut.hip
// Blocks of block_rows (1 or 128) x 128 of W.
hipError_t launch_f8_split(int64_t n, int64_t k, int block_rows, const void* W, int type, int64_t ldw, uint8_t* codes, int64_t ldq, uint8_t* scales, int64_t lds, hipStream_t st);
hipError_t launch_f8_expand(int64_t n, int64_t k, int block_rows, const uint8_t* codes, int64_t ldq, int scale_type, const void* scales, int64_t lds, void* W, int type, int64_t ldw, hipStream_t st);
// The operands of a gradient dY W: codes and scales of the transposed weights (blocks of 128 x 128), expert by expert, in rows of pad_to(n, 128)
// bytes, and scales (of the type that they have) in rows of f8_scale_bytes(n) values; and, where v_codes is not null, V (rows x n) cut by 1 x 128.
hipError_t launch_f8_gradient_operands(int64_t experts, int64_t n, int64_t k, const uint8_t* codes, int64_t ldq, int scale_type, const void* scales, int64_t lds, uint8_t* codes_t,
                                       void* scales_t, int64_t rows, const void* V, int type, int64_t ldv, uint8_t* v_codes, uint8_t* v_scales, hipStream_t st);
// The operands of a weights' gradient: rows of V (by source, of t) cut along their direction, in runs of 128 that begin with every expert (experts
// 0: one), transposed: codes n x 128 runs, scales n x runs.
struct F8Columns {
    const void* V;
    int64_t ldv, n;
    int t;
    const int* source;
    uint8_t *codes, *scales;
};
hipError_t launch_f8_cut_tokens(int64_t rows, int64_t experts, const int* offsets, int type, const F8Columns& dy, const F8Columns& x, int64_t runs, hipStream_t st);

// R = P Q^T for codes under scales. P: rows (tokens), Q: rows (outputs), both along the inner dimension in slabs of 128 bytes.
struct F8Args {
    const void* V;            // launch_f8_few: the rows (v_type, ldv values apart, k of them: cut on the way; OZIMMU_E4M3: codes, with sp)
    int v_type;
    int64_t ldv, k;
    const uint8_t* P;         // the others: their codes
    const uint8_t* sp;        // a byte for each row and slab
    const uint8_t* Q;
    const void* sq;           // bytes or 32-bit values for 128 rows and a slab (q_rows: bytes for each row)
    int64_t ldp, ldsp, ldq, ldsq;
    int slabs;                // of a row
    int rows, t, n;           // rows of R, rows of P, columns of R
    int experts;              // 0: one product
    const int* offsets;       // rows offsets[e] .. offsets[e + 1] of R meet the rows e n .. (e + 1) n of Q
    const int* source;        // row r of R comes from row source[r] of P
    bool along_rows;          // weights' gradients: P has `rows` rows and Q n, both along t tokens; a product for each expert, over its runs' slabs
    int scale_type;           // of sq
    void* out;
    int out_type;
    int64_t ldo;
    float* partial;           // room for the sums of shared tiles
    size_t partial_bytes;
};
// f8_few.hip: few rows to an expert, codes straight from memory
hipError_t launch_f8_few(const F8Args& a, hipStream_t st);
// Which tile a product takes, and how its last round of tiles is shared along the inner dimension (the first `whole` tiles are not).
enum F8Shape { kF8Tile256, kF8Tile128, kF8Tile64x128, kF8Tile64, kF8Tile32x64, kF8Shapes };
struct F8Choice {
    int shape, whole, parts, part_slabs;
};
F8Choice choose_f8_tile(const F8Args& a);
size_t f8_partial_room(int64_t rows, int64_t n, int64_t slabs);
// f8_large.hip: tiles of 256 x 256, 16-bit results, scales of a byte
hipError_t launch_f8_large(const F8Args& a, hipStream_t st);
// f8_product.hip, f8_product_exact.hip: smaller tiles; results of 16 bits, of 32
hipError_t launch_f8_tiles(const F8Args& a, const F8Choice& c, hipStream_t st);
hipError_t launch_f8_tiles_exact(const F8Args& a, const F8Choice& c, hipStream_t st);

// route.hip
struct RouteArgs {
    int t, experts, top;
    const void* logits;
    int type;
    int64_t ldl;
    const float* bias;
    int sigmoid, groups, top_groups, renormalize;
    float scale;
};
hipError_t launch_route(const RouteArgs& a, int* indices, float* weights, hipStream_t st);
hipError_t launch_route_grad(const RouteArgs& a, const int* indices, const float* dweights, void* dlogits, int64_t lddl, hipStream_t st);

// experts.hip
size_t expert_order_bytes(int64_t pairs, int experts);
hipError_t launch_expert_order(int t, int top, int experts, const int* indices, int* offsets, int* source, int* place, int* counts, hipStream_t st);
hipError_t launch_expert_combine(int t, int top, int rows, int64_t n, int type, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy, hipStream_t st);
hipError_t launch_expert_combine_grad(int t, int top, int rows, int64_t n, int type, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place, const float* weights, void* dO,
                                      int64_t lddo, float* dweights, hipStream_t st);

}  // namespace ozimmu
