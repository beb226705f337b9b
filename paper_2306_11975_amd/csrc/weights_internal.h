// What the operators on weight matrices share: products of weights in four bits (q4.hip, q4_few.hip), the orthogonal update
// (orthogonalize.hip) and the 16-bit matrix-core product under both (nt_product.h).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ozimmu.h"

namespace ozimmu {

// A matrix of 16-bit values as the product kernel reads it: rows along the inner dimension, in slabs of 64 values (128 bytes). With one
// slice a slab is 64 positions; with two it is 32 positions of the first slice and the same 32 of the second (value = first + second).
constexpr int kSlabValues = 64;

// C = P Q^T on the 16-bit matrix cores (both operands rows along the inner dimension), with what becomes of the sums.
struct NtArgs {
    const unsigned short* P;
    const unsigned short* Q;
    int64_t ldp, ldq;              // values per row
    int64_t batch_p, batch_q;      // values per matrix
    int slabs;                     // of a row
    int m, n, batch;               // rows of P, rows of Q, matrices
    bool symmetric;                // P and Q give a symmetric C: only tiles on and above the diagonal are formed, the rest mirrored
    float factor;                  // of the sums
    float* partial;                // room for the sums of tiles whose inner dimension several workgroups share, and how much there is of it (bytes);
    size_t partial_bytes;          // without it they do not
    // typed result, row-major
    void* out;
    int64_t ldo, batch_o;
    const int* exp_p;              // optional: C is scaled by 2^(exp_p[row] + exp_q[col / q_run])
    const int* exp_q;
    int q_run;
    // result in two slices, and transposed: v = factor * sum + beta * in + diagonal on the diagonal
    unsigned short* C;
    unsigned short* CT;
    const unsigned short* in;      // two slices, laid out like C
    int64_t ldc, ldct, batch_c, batch_ct;
    float beta, diagonal;
};
enum NtResult { kOutF32 = 0, kOutBf16 = 1, kOutF16 = 2, kOutSlices = 3 };
// `slices`: 1 (bf16 where `bf16`, else fp16) or 2 (fp16)
// Room that launch_nt_product can make use of for any product (at most so many workgroups share tiles).
constexpr size_t kPartialBytes = 512 * 128 * 128 * sizeof(float);
hipError_t launch_nt_product(const NtArgs& a, int slices, bool bf16, NtResult result, hipStream_t st);

// 16-byte accesses are possible to every row of an array of rows
inline bool rows_aligned16(const void* p, int64_t ld, size_t size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * (int64_t)size) % 16 == 0;
}

__host__ __device__ inline int64_t pad_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// q4.hip
hipError_t launch_q4_split(int64_t n, int64_t k, int group, const void* W, int type, int64_t ldw, uint8_t* codes, int64_t ldq,
                           void* scales, int scale_type, int64_t lds, hipStream_t st);
// The weights s c as a typed matrix.
hipError_t launch_q4_expand(int64_t n, int64_t k, int group, const uint8_t* codes, int64_t ldq, const void* scales, int type,
                            int64_t lds, void* W, int64_t ldw, hipStream_t st);
// The operands of a product of many tokens, rows of ld values: the weights (`columns`: their columns) and, where v_out is not null, the
// rows of V. 16-bit types: one slice, padded to slabs. OZIMMU_F32: two slices of fp16 scaled by 2^-exponent: one exponent per row, for
// columns of W one per group.
hipError_t launch_operands(int64_t t, int64_t n, int64_t k, int group, int type, const uint8_t* codes, int64_t ldq, const void* scales, int64_t lds, bool columns,
                           unsigned short* w_out, int* w_exps, const void* V, int64_t ldv, unsigned short* v_out, int* v_exps, int64_t ld, hipStream_t st);
// Zeros into a typed matrix.
hipError_t launch_zero_rows(int64_t rows, int64_t cols, void* R, int type, int64_t ld, hipStream_t st);
// q4_token.hip: Y = X W^T for one token or two
hipError_t launch_q4_token(int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes, int64_t ldq,
                           const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st);
// q4_few.hip: Y = X W^T for few tokens, a pass over the codes for every 16 or 32 of them
hipError_t launch_q4_few(int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes,
                         int64_t ldq, const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st);

// q4_tile.hip: Y = X W^T of 16-bit types and k >= 8 for more tokens, the operand of the weights made tile by tile (64 x 64, or `large`: 128
// x 128)
hipError_t launch_q4_tiles(bool large, int64_t t, int64_t n, int64_t k, int group, const void* X, int type, int64_t ldx, const uint8_t* codes, int64_t ldq,
                           const void* scales, int64_t lds, void* Y, int64_t ldy, hipStream_t st);

// orthogonalize.hip
constexpr int kMostNormParts = 1024;   // partial sums of squares per matrix
int norm_parts(int64_t m, int64_t n);
hipError_t launch_norm_partials(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride,
                                double* partials, hipStream_t st);
// G / (|G| + eps) in two slices of fp16 scaled by 2^shift, as it lies (rows of n) and transposed (rows of m)
hipError_t launch_normalised_slices(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride,
                                    const double* partials, double eps, int shift, unsigned short* rows, int64_t ldr,
                                    int64_t batch_r, unsigned short* cols, int64_t ldc, int64_t batch_c, hipStream_t st);

// orthogonalize_small.hip: the whole update by one workgroup per matrix
constexpr int64_t kSmallShorter = 64, kSmallLonger = 256;
hipError_t launch_orthogonalize_small(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride_g, void* X, int64_t ldx,
                                      int64_t stride_x, int steps, double a, double b, double c, double eps, int shift, hipStream_t st);

// The same for longer ones, in panels of kNarrowPanel positions: `images` holds kNarrowPanel * 256 bytes and `sums` 64 * 64 values for
// every panel of every matrix, `factors` 64 * 64 * 4 bytes for every matrix
constexpr int kNarrowPanel = 128;
constexpr int64_t kNarrowLonger = 8192;
hipError_t launch_orthogonalize_narrow(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride_g, void* X, int64_t ldx,
                                       int64_t stride_x, int steps, double a, double b, double c, double eps, int shift, const double* norms, unsigned char* images,
                                       unsigned char* factors, float* sums, hipStream_t st);

}  // namespace ozimmu
