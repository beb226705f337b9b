// The orthogonal update of matrices whose shorter side is at most 64. Up to 256 along the longer one, one workgroup per matrix runs the
// whole iteration out of LDS; up to 8192, panels (below) (gfx950).
//
// As launches of the product kernel the iteration takes 17 of them, about 4 us each whatever the size; here a step is three passes of MFMAs
// between barriers. In LDS lie, in two slices of fp16 as in nt_product.h (rows in slabs of 128 bytes: 32 positions of the first slice and
// of the second, 16-byte piece c of row r at place c ^ (r % 8)): X (64 rows along the longer side), its transpose, and A, which the
// polynomial of A then replaces. Every pass forms its results in registers, waits for everyone's reads, and writes.
#include <algorithm>

#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;

// byte of position `at` in row `row` of an array of `rows` rows, first slice; the second one's piece is 4 places on: bit 6 of the byte
// changed
__device__ __forceinline__ unsigned slot(int rows, int row, int at) {
    return (unsigned)((at >> 5) * rows + row) * 128 + (((at & 31) >> 3) ^ (row & 7)) * 16 + (at & 7) * 2;
}

// Both slices of one value.
__device__ __forceinline__ void put(unsigned char* base, unsigned at, unsigned short h, unsigned short s) {
    *reinterpret_cast<unsigned short*>(base + at) = h;
    *reinterpret_cast<unsigned short*>(base + (at ^ 64)) = s;
}
// A lane's 16 bytes of the fragment of 16 rows from `row` on; `of`: Lane::frag0 or frag1.
__device__ __forceinline__ v4u frag(const unsigned char* base, int rows, int slab, int row, unsigned of) {
    return *reinterpret_cast<const v4u*>(base + (unsigned)(slab * rows + row) * 128 + of);
}
__device__ __forceinline__ v4f three(const v4u& q0, const v4u& q1, const v4u& p0, const v4u& p1, v4f s) {
    s = mfma_half<false>(q1, p0, s);
    s = mfma_half<false>(q0, p1, s);
    return mfma_half<false>(q0, p0, s);
}
// A lane holds element (row, col .. col + 3) of a 16 x 16 result: row lane % 16, col 4 (lane / 16).
__device__ __forceinline__ void put_row(unsigned char* base, int rows, int row, int col, const float (&v)[4], unsigned short (&h)[4], unsigned short (&s)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) two_slices(v[e], h[e], s[e]);
    const unsigned at = slot(rows, row, col);
    *reinterpret_cast<v2u*>(base + at) = *reinterpret_cast<const v2u*>(h);
    *reinterpret_cast<v2u*>(base + (at ^ 64)) = *reinterpret_cast<const v2u*>(s);
}
struct Lane {
    int lane, wave, quarter;
    unsigned frag0, frag1;
    int ai, aj;   // this wavefront's 16 x 32 part of A
    __device__ __forceinline__ Lane() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        quarter = lane >> 4;
        frag0 = (lane & 15) * 128 + ((quarter ^ (lane & 7)) * 16);
        frag1 = (lane & 15) * 128 + (((quarter + 4) ^ (lane & 7)) * 16);
        ai = (wave >> 1) * 16;
        aj = (wave & 1) * 32;
    }
};
// Its part of X X^T, X as 64 rows of `slabs` slabs.
__device__ __forceinline__ void gram(const Lane& me, const unsigned char* x_at, int slabs, v4f (&acc)[2]) {
    for (int slab = 0; slab < slabs; ++slab) {
        const v4u p0 = frag(x_at, 64, slab, me.ai, me.frag0), p1 = frag(x_at, 64, slab, me.ai, me.frag1);
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j] = three(frag(x_at, 64, slab, me.aj + 16 * j, me.frag0), frag(x_at, 64, slab, me.aj + 16 * j, me.frag1), p0, p1, acc[j]);
    }
}
// From sums of X X^T to the polynomial of A in A's place. (Nobody reads that place any more; in the end nobody else has read the polynomial
// yet.)
__device__ __forceinline__ void polynomial(const Lane& me, unsigned char* a_at, const v4f (&acc)[2], float a, float b, float c, int shift) {
    const float down = ldexpf(1.f, -shift);
    float mine[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        unsigned short h[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[j][e] = acc[j][e] * down;
        put_row(a_at, 64, me.ai + (me.lane & 15), me.aj + 16 * j + 4 * me.quarter, mine[j], h, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[j][e] = f16_to_f32(h[e]) + f16_to_f32(s[e]);
    }
    __syncthreads();
    // a + b A + c A^2
    v4f square[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    gram(me, a_at, 2, square);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        unsigned short h[4], s[4];
        const int row = me.ai + (me.lane & 15), col = me.aj + 16 * j + 4 * me.quarter;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            mine[j][e] = fmaf(b, mine[j][e], c * down * square[j][e]);
            if (row == col + e) mine[j][e] += ldexpf(a, shift);
        }
        put_row(a_at, 64, row, col, mine[j], h, s);
    }
    __syncthreads();
}
// The polynomial times the 16 columns of X from `col` on, which lie transposed in rows of t_at.
__device__ __forceinline__ void times_x(const Lane& me, const unsigned char* a_at, const unsigned char* t_at, int l_pad, int col, v4f (&next)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int slab = 0; slab < 2; ++slab) {
        const v4u q0 = frag(t_at, l_pad, slab, col, me.frag0), q1 = frag(t_at, l_pad, slab, col, me.frag1);
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = three(q0, q1, frag(a_at, 64, slab, 16 * i, me.frag0), frag(a_at, 64, slab, 16 * i, me.frag1), next[i]);
    }
}
// Those results as the new X and its transpose ..
__device__ __forceinline__ void put_x(const Lane& me, unsigned char* x_at, unsigned char* t_at, int l_pad, int col, const v4f (&next)[4], float down) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 16 * i + (me.lane & 15), at = col + 4 * me.quarter;
        float v[4];
        unsigned short h[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = next[i][e] * down;
        put_row(x_at, 64, row, at, v, h, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) put(t_at, slot(l_pad, at + e, row), h[e], s[e]);
    }
}
// .. or as the result: columns l0 + col of an r x l matrix, or rows of the transposed one.
template <int TYPE>
__device__ __forceinline__ void store_x(const Lane& me, typename Elem<TYPE>::raw* out, int64_t ldx, bool tall, int r, int64_t l, int64_t col, const v4f (&next)[4], float down) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 16 * i + (me.lane & 15);
        const int64_t at = col + 4 * me.quarter;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (row < r && at + e < l) out[tall ? (at + e) * ldx + row : (int64_t)row * ldx + at + e] = Elem<TYPE>::store(next[i][e] * down * down);
    }
}

template <int TYPE>
__launch_bounds__(kThreads)
__global__ void orthogonalize_small_kernel(int m, int n, const void* G, int64_t ldg, int64_t stride_g, void* X, int64_t ldx, int64_t stride_x, int steps, float a,
                                           float b, float c, double eps, int shift, int l_pad) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __shared__ double shared[kWaves];
    unsigned char* const x_at = lds;                           // 64 rows of l_pad
    unsigned char* const t_at = lds + 64 * l_pad * 4;          // l_pad rows of 64
    unsigned char* const a_at = lds + 2 * 64 * l_pad * 4;      // 64 rows of 64
    const Lane me;
    const int lane = me.lane, wave = me.wave;
    const bool tall = m > n;
    const int r = tall ? n : m, l = tall ? m : n;
    const raw* g = reinterpret_cast<const raw*>(G) + blockIdx.x * stride_g;
    raw* out = reinterpret_cast<raw*>(X) + blockIdx.x * stride_x;

    // the norm, in 64 bits and a fixed order
    double sum = 0.0;
    for (int j = lane; j < n; j += 64) {
        const raw* at = g + j;
#pragma unroll 8
        for (int i = wave; i < m; i += kWaves) {
            const double v = E::load(at[(int64_t)i * ldg]);
            sum = fma(v, v, sum);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) shared[wave] = sum;
    __syncthreads();
    sum = shared[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) sum += shared[i];
    const double norm = sqrt(sum) + eps;
    const double inv = norm > 0.0 ? (double)(1 << shift) / norm : norm;   // (a matrix of zeros stays one; NaN stays NaN)

    // X_0 and its transpose, zeros in the padding (where a norm that is not finite does not reach either); along G's rows, from the caches
    const int rows = tall ? l_pad : 64, cols = tall ? 64 : l_pad;
    for (int j = lane; j < cols; j += 64) {
        const raw* at = g + min(j, n - 1);
#pragma unroll 4
        for (int i = wave; i < rows; i += kWaves) {
            const raw y = at[(int64_t)min(i, m - 1) * ldg];
            unsigned short h, s;
            two_slices((float)((double)E::load(y) * inv), h, s);
            if (i >= m || j >= n) h = s = 0;
            const int xr = tall ? j : i, xc = tall ? i : j;
            put(x_at, slot(64, xr, xc), h, s);
            put(t_at, slot(l_pad, xc, xr), h, s);
        }
    }
    __syncthreads();

    const float down = ldexpf(1.f, -shift);
    constexpr int kMostTiles = 2;                            // of 16 columns of X for a wavefront: l_pad <= 256
    for (int step = 0; step < steps; ++step) {
        const bool last = step + 1 == steps;
        v4f acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        gram(me, x_at, l_pad / 32, acc);
        // (A's place still holds the last step's polynomial, which everyone has read: a barrier stands behind its last use)
        polynomial(me, a_at, acc, a, b, c, shift);
        v4f next[kMostTiles][4];
#pragma unroll
        for (int t = 0; t < kMostTiles; ++t)
            if ((wave + t * kWaves) * 16 < l_pad) times_x(me, a_at, t_at, l_pad, (wave + t * kWaves) * 16, next[t]);
        if (!last) __syncthreads();
#pragma unroll
        for (int t = 0; t < kMostTiles; ++t) {
            const int col = (wave + t * kWaves) * 16;
            if (col >= l_pad) continue;
            if (last)
                store_x<TYPE>(me, out, ldx, tall, r, l, col, next[t], down);
            else
                put_x(me, x_at, t_at, l_pad, col, next[t], down);
        }
        if (!last) __syncthreads();
    }
}

template <int TYPE>
hipError_t launch_typed(int64_t batch, int64_t m, int64_t n, const void* G, int64_t ldg, int64_t stride_g, void* X, int64_t ldx, int64_t stride_x, int steps, double a,
                        double b, double c, double eps, int shift, hipStream_t st) {
    constexpr auto kernel = orthogonalize_small_kernel<TYPE>;
    const int l_pad = (int)pad_to(m > n ? m : n, 32), bytes = (2 * l_pad + 64) * 64 * 4;
    if (hipError_t e = allow_dynamic_lds<kernel>((2 * (int)kSmallLonger + 64) * 64 * 4); e != hipSuccess) return e;
    kernel<<<dim3((unsigned)batch), kThreads, bytes, st>>>((int)m, (int)n, G, ldg, stride_g, X, ldx, stride_x, steps, (float)a, (float)b, (float)c, eps, shift, l_pad);
    return hipGetLastError();
}

// ---- a longer side beyond that: panels of 128 positions along it, a workgroup each, which leave their part of A = X X^T; one workgroup adds the parts up, in order, and makes the
// polynomial, and the next launch multiplies the panels by it: two launches a step, against three or four of the products. X (transposed)
// and the polynomial go through memory as they lie in LDS. What bounds it is latency, 4 to 7 us a launch (64 x 1024: 90 us as products, 56
// here; 64 of them 157 and 100).
enum PanelPart { kFirst, kMiddle, kLast };

template <int TYPE, int PART>
__launch_bounds__(kThreads)
__global__ void panel_kernel(int64_t m, int64_t n, const void* G, int64_t ldg, int64_t stride_g, void* X, int64_t ldx, int64_t stride_x, const double* norms, int parts, double eps,
                             int shift, unsigned char* images, const unsigned char* factors, v4f* sums) {
    typedef Elem<TYPE> E;
    typedef typename E::raw raw;
    __shared__ __attribute__((aligned(16))) unsigned char x_at[kNarrowPanel * 64 * 4], t_at[kNarrowPanel * 64 * 4], a_at[64 * 64 * 4];
    __shared__ double shared[kWaves];
    const Lane me;
    const int64_t z = blockIdx.y, panel = z * gridDim.x + blockIdx.x, l0 = (int64_t)blockIdx.x * kNarrowPanel;
    const bool tall = m > n;
    v4u* const image = reinterpret_cast<v4u*>(images + panel * (int64_t)sizeof(t_at));
    if constexpr (PART == kFirst) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < parts; i += kThreads) sum += norms[z * parts + i];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if (me.lane == 0) shared[me.wave] = sum;
        __syncthreads();
        sum = shared[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += shared[i];
        const double norm = sqrt(sum) + eps;
        const double inv = norm > 0.0 ? (double)(1 << shift) / norm : norm;   // (a matrix of zeros stays one; NaN stays NaN)
        const raw* g = reinterpret_cast<const raw*>(G) + z * stride_g;
        const int rows = tall ? kNarrowPanel : 64, cols = tall ? 64 : kNarrowPanel;
        const int64_t row0 = tall ? l0 : 0, col0 = tall ? 0 : l0;
        for (int j = me.lane; j < cols; j += 64) {
            const raw* at = g + min(col0 + j, n - 1);
#pragma unroll 8
            for (int i = me.wave; i < rows; i += kWaves) {
                const raw y = at[min(row0 + i, m - 1) * ldg];
                unsigned short h, s;
                two_slices((float)((double)E::load(y) * inv), h, s);
                if (row0 + i >= m || col0 + j >= n) h = s = 0;
                const int xr = tall ? j : i, xc = tall ? i : j;
                put(x_at, slot(64, xr, xc), h, s);
                put(t_at, slot(kNarrowPanel, xc, xr), h, s);
            }
        }
    } else {
        const v4u* const factor = reinterpret_cast<const v4u*>(factors + z * (int64_t)sizeof(a_at));
#pragma unroll
        for (int i = 0; i < (int)(sizeof(t_at) / 16 / kThreads); ++i) reinterpret_cast<v4u*>(t_at)[i * kThreads + threadIdx.x] = image[i * kThreads + threadIdx.x];
#pragma unroll
        for (int i = 0; i < (int)(sizeof(a_at) / 16 / kThreads); ++i) reinterpret_cast<v4u*>(a_at)[i * kThreads + threadIdx.x] = factor[i * kThreads + threadIdx.x];
        __syncthreads();
        const float down = ldexpf(1.f, -shift);
        v4f next[4];
        times_x(me, a_at, t_at, kNarrowPanel, me.wave * 16, next);
        if constexpr (PART == kLast) {
            store_x<TYPE>(me, reinterpret_cast<raw*>(X) + z * stride_x, ldx, tall, (int)(tall ? n : m), tall ? m : n, l0 + me.wave * 16, next, down);
            return;
        }
        __syncthreads();
        put_x(me, x_at, t_at, kNarrowPanel, me.wave * 16, next, down);
    }
    if constexpr (PART != kLast) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < (int)(sizeof(t_at) / 16 / kThreads); ++i) image[i * kThreads + threadIdx.x] = reinterpret_cast<const v4u*>(t_at)[i * kThreads + threadIdx.x];
        v4f acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        gram(me, x_at, kNarrowPanel / 32, acc);
#pragma unroll
        for (int j = 0; j < 2; ++j) sums[(panel * 2 + j) * kThreads + threadIdx.x] = acc[j];
    }
}

__launch_bounds__(kThreads)
__global__ void panel_polynomial_kernel(int panels, const v4f* sums, float a, float b, float c, int shift, unsigned char* factors) {
    __shared__ __attribute__((aligned(16))) unsigned char a_at[64 * 64 * 4];
    const Lane me;
    const v4f* from = sums + (int64_t)blockIdx.x * panels * (2 * kThreads) + threadIdx.x;
    v4f acc[2] = {from[0], from[kThreads]};
#pragma unroll 8
    for (int p = 1; p < panels; ++p)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const v4f x = from[(int64_t)(p * 2 + j) * kThreads];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] += x[e];
        }
    polynomial(me, a_at, acc, a, b, c, shift);
    v4u* const factor = reinterpret_cast<v4u*>(factors + blockIdx.x * sizeof(a_at));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(a_at) / 16 / kThreads); ++i) factor[i * kThreads + threadIdx.x] = reinterpret_cast<const v4u*>(a_at)[i * kThreads + threadIdx.x];
}

template <int TYPE>
hipError_t launch_narrow(int64_t batch, int64_t m, int64_t n, const void* G, int64_t ldg, int64_t stride_g, void* X, int64_t ldx, int64_t stride_x, int steps, double a, double b,
                         double c, double eps, int shift, const double* norms, unsigned char* images, unsigned char* factors, float* sums, hipStream_t st) {
    const int panels = (int)((std::max(m, n) + kNarrowPanel - 1) / kNarrowPanel), parts = norm_parts(m, n);
    const dim3 grid((unsigned)panels, (unsigned)batch);
    v4f* const to = reinterpret_cast<v4f*>(sums);
    panel_kernel<TYPE, kFirst><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride_g, X, ldx, stride_x, norms, parts, eps, shift, images, factors, to);
    for (int i = 0; i < steps; ++i) {
        if (i > 0)
            panel_kernel<OZIMMU_F32, kMiddle><<<grid, kThreads, 0, st>>>(m, n, nullptr, 0, 0, nullptr, 0, 0, nullptr, 0, eps, shift, images, factors, to);
        panel_polynomial_kernel<<<dim3((unsigned)batch), kThreads, 0, st>>>(panels, to, (float)a, (float)b, (float)c, shift, factors);
    }
    panel_kernel<TYPE, kLast><<<grid, kThreads, 0, st>>>(m, n, G, ldg, stride_g, X, ldx, stride_x, norms, parts, eps, shift, images, factors, to);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_orthogonalize_small(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride_g, void* X, int64_t ldx,
                                      int64_t stride_x, int steps, double a, double b, double c, double eps, int shift, hipStream_t st) {
    if (type == OZIMMU_F32) return launch_typed<OZIMMU_F32>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
    if (type == OZIMMU_BF16) return launch_typed<OZIMMU_BF16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
    return launch_typed<OZIMMU_F16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
}

hipError_t launch_orthogonalize_narrow(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride_g, void* X, int64_t ldx,
                                       int64_t stride_x, int steps, double a, double b, double c, double eps, int shift, const double* norms, unsigned char* images,
                                       unsigned char* factors, float* sums, hipStream_t st) {
    if (type == OZIMMU_F32)
        return launch_narrow<OZIMMU_F32>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, norms, images, factors, sums, st);
    if (type == OZIMMU_BF16)
        return launch_narrow<OZIMMU_BF16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, norms, images, factors, sums, st);
    return launch_narrow<OZIMMU_F16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, norms, images, factors, sums, st);
}

}  // namespace ozimmu
