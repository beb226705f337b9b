// The orthogonal update of matrices whose shorter side is at most 64 and whose longer one at most 256: one workgroup per matrix
// runs the whole iteration out of LDS (gfx950).
//
// As launches of the product kernel the iteration takes 17 of them, about 4 us each whatever the size; here a step is three
// passes of MFMAs between barriers. In LDS lie, in two slices of fp16 as in nt_product.h (rows in slabs of 128 bytes: 32 positions of the first slice and of the
// second, 16-byte piece c of row r at place c ^ (r % 8)): X (64 rows along the longer side), its transpose, and A, which the
// polynomial of A then replaces. Every pass forms its results in registers, waits for everyone's reads, and writes.
#include "half_common.h"

namespace ozimmu {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;

// byte of position `at` in row `row` of an array of `rows` rows, first slice; the second one's piece is 4 places on: bit 6 of the byte changed
__device__ __forceinline__ unsigned slot(int rows, int row, int at) {
    return (unsigned)((at >> 5) * rows + row) * 128 + (((at & 31) >> 3) ^ (row & 7)) * 16 + (at & 7) * 2;
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
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4;
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

    auto put = [](unsigned char* base, unsigned at, unsigned short h, unsigned short s) {
        *reinterpret_cast<unsigned short*>(base + at) = h;
        *reinterpret_cast<unsigned short*>(base + (at ^ 64)) = s;
    };
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

    // a lane's 16 bytes of a fragment of 16 rows
    const unsigned frag0 = (lane & 15) * 128 + ((quarter ^ (lane & 7)) * 16);
    const unsigned frag1 = (lane & 15) * 128 + (((quarter + 4) ^ (lane & 7)) * 16);
    auto frag = [&](const unsigned char* base, int rows, int slab, int row, unsigned of) {
        return *reinterpret_cast<const v4u*>(base + (unsigned)(slab * rows + row) * 128 + of);
    };
    auto three = [](const v4u& q0, const v4u& q1, const v4u& p0, const v4u& p1, v4f s) {
        s = mfma_half<false>(q1, p0, s);
        s = mfma_half<false>(q0, p1, s);
        return mfma_half<false>(q0, p0, s);
    };
    // a lane holds element (row, col .. col + 3) of a 16 x 16 result: row lane % 16, col 4 quarter
    auto put_row = [&](unsigned char* base, int rows, int row, int col, const float (&v)[4], unsigned short (&h)[4], unsigned short (&s)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) two_slices(v[e], h[e], s[e]);
        const unsigned at = slot(rows, row, col);
        *reinterpret_cast<v2u*>(base + at) = *reinterpret_cast<const v2u*>(h);
        *reinterpret_cast<v2u*>(base + (at ^ 64)) = *reinterpret_cast<const v2u*>(s);
    };
    const float down = ldexpf(1.f, -shift);
    const int ai = (wave >> 1) * 16, aj = (wave & 1) * 32;   // this wavefront's 16 x 32 part of A
    constexpr int kMostTiles = 2;                            // of 16 columns of X for a wavefront: l_pad <= 256
    for (int step = 0; step < steps; ++step) {
        const bool last = step + 1 == steps;
        // A = X X^T
        v4f acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        for (int slab = 0; slab < l_pad / 32; ++slab) {
            const v4u p0 = frag(x_at, 64, slab, ai, frag0), p1 = frag(x_at, 64, slab, ai, frag1);
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[j] = three(frag(x_at, 64, slab, aj + 16 * j, frag0), frag(x_at, 64, slab, aj + 16 * j, frag1), p0, p1, acc[j]);
        }
        // (A's place still holds the last step's polynomial, which everyone has read: a barrier stands behind its last use)
        float mine[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            unsigned short h[4], s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[j][e] = acc[j][e] * down;
            put_row(a_at, 64, ai + (lane & 15), aj + 16 * j + 4 * quarter, mine[j], h, s);
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[j][e] = f16_to_f32(h[e]) + f16_to_f32(s[e]);
        }
        __syncthreads();
        // a + b A + c A^2
        v4f square[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int slab = 0; slab < 2; ++slab) {
            const v4u p0 = frag(a_at, 64, slab, ai, frag0), p1 = frag(a_at, 64, slab, ai, frag1);
#pragma unroll
            for (int j = 0; j < 2; ++j) square[j] = three(frag(a_at, 64, slab, aj + 16 * j, frag0), frag(a_at, 64, slab, aj + 16 * j, frag1), p0, p1, square[j]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            unsigned short h[4], s[4];
            const int row = ai + (lane & 15), col = aj + 16 * j + 4 * quarter;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mine[j][e] = fmaf(b, mine[j][e], c * down * square[j][e]);
                if (row == col + e) mine[j][e] += ldexpf(a, shift);
            }
            put_row(a_at, 64, row, col, mine[j], h, s);
        }
        __syncthreads();
        // times X
        v4f next[kMostTiles][4];
#pragma unroll
        for (int t = 0; t < kMostTiles; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) next[t][i] = v4f{0.f, 0.f, 0.f, 0.f};
            const int tile = wave + t * kWaves;
            if (tile * 16 >= l_pad) continue;
#pragma unroll
            for (int slab = 0; slab < 2; ++slab) {
                const v4u q0 = frag(t_at, l_pad, slab, tile * 16, frag0), q1 = frag(t_at, l_pad, slab, tile * 16, frag1);
#pragma unroll
                for (int i = 0; i < 4; ++i) next[t][i] = three(q0, q1, frag(a_at, 64, slab, 16 * i, frag0), frag(a_at, 64, slab, 16 * i, frag1), next[t][i]);
            }
        }
        if (!last) __syncthreads();
#pragma unroll
        for (int t = 0; t < kMostTiles; ++t) {
            const int tile = wave + t * kWaves;
            if (tile * 16 >= l_pad) continue;
            const int col = tile * 16 + 4 * quarter;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * i + (lane & 15);
                float v[4];
                if (last) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row < r && col + e < l) out[tall ? (int64_t)(col + e) * ldx + row : (int64_t)row * ldx + col + e] = E::store(next[t][i][e] * down * down);
                } else {
                    unsigned short h[4], s[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = next[t][i][e] * down;
                    put_row(x_at, 64, row, col, v, h, s);
#pragma unroll
                    for (int e = 0; e < 4; ++e) put(t_at, slot(l_pad, col + e, row), h[e], s[e]);
                }
            }
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

}  // namespace

hipError_t launch_orthogonalize_small(int64_t batch, int64_t m, int64_t n, const void* G, int type, int64_t ldg, int64_t stride_g, void* X, int64_t ldx,
                                      int64_t stride_x, int steps, double a, double b, double c, double eps, int shift, hipStream_t st) {
    if (type == OZIMMU_F32) return launch_typed<OZIMMU_F32>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
    if (type == OZIMMU_BF16) return launch_typed<OZIMMU_BF16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
    return launch_typed<OZIMMU_F16>(batch, m, n, G, ldg, stride_g, X, ldx, stride_x, steps, a, b, c, eps, shift, st);
}

}  // namespace ozimmu
