// The orthogonal update's own kernels: the Frobenius norm and the normalised matrix in two slices (gfx950). The products of the
// iteration are nt_product.h's.
#include <algorithm>

#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double block_sum(double x, double* shared) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = shared[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) x += shared[i];
    __syncthreads();
    return x;
}

// Sums of squares in 64 bits (squares of 32-bit values do not overflow there): workgroup b of a matrix takes rows b, b + gridDim.x, ...
// A fixed order: the same sum on every run.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void norm_partials_kernel(int64_t m, int64_t n, const void* G, int64_t ldg, int64_t stride, double* partials) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    constexpr int V = 16 / sizeof(raw);
    __shared__ double shared[kThreads / 64];
    const raw* g = reinterpret_cast<const raw*>(G) + blockIdx.y * stride;
    double sum = 0.0;
    // threads over the 16-byte pieces of as many rows at a time as fill the workgroup
    const int64_t pieces = (n + V - 1) / V;
    int tx = 1;
    while (tx < kThreads && tx < pieces) tx *= 2;
    const int ty = kThreads / tx;
    for (int64_t row = (int64_t)blockIdx.x * ty + threadIdx.x / tx; row < m; row += (int64_t)gridDim.x * ty)
        for (int64_t p = threadIdx.x % tx; p < pieces; p += tx) {
            const raw* at = g + row * ldg + p * V;
            raw r[V];
            if (p * V + V <= n)
                *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u_any*>(at);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) r[e] = p * V + e < n ? at[e] : raw(0);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double x = E::load(r[e]);
                sum = fma(x, x, sum);
            }
        }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) partials[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// A 64 x 64 tile of G, divided by its norm, in two slices: rows as they lie, and through LDS transposed. The padding of rows is written as
// zeros. A thread takes 16 values of a row, then of a column: memory-bound, 16-byte accesses throughout.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void normalised_slices_kernel(int64_t m, int64_t n, const void* G, int64_t ldg, int64_t stride, const double* partials, int parts, double eps,
                                         double scale, unsigned short* rows, int64_t ldr, int64_t batch_r, unsigned short* cols, int64_t ldc,
                                         int64_t batch_c, int tiles_n) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    __shared__ unsigned tile[64][65];   // first slice low, second high
    __shared__ double shared[kThreads / 64];
    const int64_t z = blockIdx.y;
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 64, n0 = (int64_t)(blockIdx.x % tiles_n) * 64;
    const int across = threadIdx.x / 4, along = threadIdx.x % 4 * 16;
    const int64_t row = m0 + across, at = n0 + along;
    const raw* g = reinterpret_cast<const raw*>(G) + z * stride + min(row, m - 1) * ldg + at;
    raw held[16];
    if (at + 16 <= n) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(raw); ++i) reinterpret_cast<v4u*>(held)[i] = reinterpret_cast<const v4u_any*>(g)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) held[e] = at + e < n ? g[e] : raw(0);
    }
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += partials[z * parts + i];
    sum = block_sum(sum, shared);
    const double norm = sqrt(sum) + eps;
    const double inv = norm > 0.0 ? scale / norm : norm;   // (a matrix of zeros stays one; NaN stays NaN)
    unsigned short h[16], l[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        two_slices(row < m && at + e < n ? (float)((double)E::load(held[e]) * inv) : 0.f, h[e], l[e]);
        tile[across][along + e] = (unsigned)h[e] | (unsigned)l[e] << 16;
    }
    auto store = [](unsigned short* to, const unsigned short (&h)[16], const unsigned short (&l)[16]) {
        reinterpret_cast<v4u*>(to)[0] = reinterpret_cast<const v4u*>(h)[0];
        reinterpret_cast<v4u*>(to)[1] = reinterpret_cast<const v4u*>(h)[1];
        reinterpret_cast<v4u*>(to + 32)[0] = reinterpret_cast<const v4u*>(l)[0];
        reinterpret_cast<v4u*>(to + 32)[1] = reinterpret_cast<const v4u*>(l)[1];
    };
    if (row < m && at < pad_to(n, 32)) store(rows + z * batch_r + row * ldr + (at >> 5) * 64 + (at & 31), h, l);
    __syncthreads();
    const int64_t col = n0 + across, down = m0 + along;
    if (col < n && down < pad_to(m, 32)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const unsigned both = tile[along + e][across];
            h[e] = (unsigned short)both;
            l[e] = (unsigned short)(both >> 16);
        }
        store(cols + z * batch_c + col * ldc + (down >> 5) * 64 + (down & 31), h, l);
    }
}

}  // namespace

int norm_parts(int64_t m, int64_t n) { return (int)std::min<int64_t>(kMostNormParts, std::max<int64_t>(1, m * n / 8192)); }

hipError_t launch_norm_partials(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride, double* partials, hipStream_t st) {
    const dim3 grid((unsigned)norm_parts(m, n), (unsigned)batch);
    if (type == OZIMMU_F32)
        norm_partials_kernel<OZIMMU_F32><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials);
    else if (type == OZIMMU_BF16)
        norm_partials_kernel<OZIMMU_BF16><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials);
    else
        norm_partials_kernel<OZIMMU_F16><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials);
    return hipGetLastError();
}

hipError_t launch_normalised_slices(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride, const double* partials,
                                    double eps, int shift, unsigned short* rows, int64_t ldr, int64_t batch_r, unsigned short* cols, int64_t ldc,
                                    int64_t batch_c, hipStream_t st) {
    const int tiles_n = (int)((n + 63) / 64);
    const dim3 grid((unsigned)((m + 63) / 64 * tiles_n), (unsigned)batch);
    const double scale = (double)(1 << shift);
    const int parts = norm_parts(m, n);
    if (type == OZIMMU_F32)
        normalised_slices_kernel<OZIMMU_F32><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials, parts, eps, scale, rows, ldr, batch_r, cols, ldc, batch_c, tiles_n);
    else if (type == OZIMMU_BF16)
        normalised_slices_kernel<OZIMMU_BF16><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials, parts, eps, scale, rows, ldr, batch_r, cols, ldc, batch_c, tiles_n);
    else
        normalised_slices_kernel<OZIMMU_F16><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride, partials, parts, eps, scale, rows, ldr, batch_r, cols, ldc, batch_c, tiles_n);
    return hipGetLastError();
}

}  // namespace ozimmu
