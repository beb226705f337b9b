// Rows sorted by expert, and the experts' results brought back to the tokens, with its gradient (gfx950). No atomics: equal calls give equal
// bits.
#include <algorithm>

#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;
constexpr int kOrderWaves = 16;       // of a workgroup of the sort
constexpr int kPairsOfWave = 256;     // pairs that one of its wavefronts takes, 64 at a time
constexpr int kPairsOfBlock = kOrderWaves * kPairsOfWave;

// Stable sort by counting. Pass one: every workgroup counts its pairs by expert. Pass two: the pairs before the workgroup's own, by expert and
// in all, give each expert's first row; within the workgroup wavefronts count again, in order, and within a wavefront a pair's rank is the
// number of lower lanes with its expert, from ten ballots over the bits of the expert's number.
__device__ __forceinline__ int expert_of(const int* indices, int64_t at, int64_t pairs, int experts) {
    const int e = at < pairs ? indices[at] : -1;
    return (unsigned)e < (unsigned)experts ? e : -1;
}
__device__ __forceinline__ unsigned long long lanes_alike(int e) {
    unsigned long long same = __builtin_amdgcn_ballot_w64(e >= 0);
#pragma unroll
    for (int b = 0; b < 10; ++b) {
        const unsigned long long set = __builtin_amdgcn_ballot_w64(e >> b & 1);
        same &= (e >> b & 1) ? set : ~set;
    }
    return same;
}
// counts[wave][expert] of the workgroup's pairs
__device__ __forceinline__ void count_pairs(const int* indices, int64_t pairs, int experts, int* counts) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < experts * kOrderWaves; e += kOrderWaves * 64) counts[e] = 0;
    __syncthreads();
    int* mine = counts + wave * experts;
    for (int p = 0; p < kPairsOfWave; p += 64) {
        const int e = expert_of(indices, (int64_t)blockIdx.x * kPairsOfBlock + wave * kPairsOfWave + p + lane, pairs, experts);
        const unsigned long long same = lanes_alike(e);
        if (e >= 0 && __builtin_ctzll(same) == lane) mine[e] += __builtin_popcountll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

__launch_bounds__(kOrderWaves * 64)
__global__ void expert_count_kernel(int64_t pairs, int experts, const int* indices, int* counts) {
    extern __shared__ int local[];
    count_pairs(indices, pairs, experts, local);
    for (int e = threadIdx.x; e < experts; e += kOrderWaves * 64) {
        int sum = 0;
        for (int w = 0; w < kOrderWaves; ++w) sum += local[w * experts + e];
        counts[(int64_t)blockIdx.x * experts + e] = sum;
    }
}

__launch_bounds__(kOrderWaves * 64)
__global__ void expert_place_kernel(int64_t pairs, int top, int experts, const int* indices, const int* counts, int* offsets, int* source, int* place) {
    extern __shared__ int local[];      // kOrderWaves counts of each expert, and one more row
    __shared__ int wave_sums[kOrderWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = threadIdx.x;
    count_pairs(indices, pairs, experts, local);
    // each expert's pairs in the workgroups before this one, and in all
    int before = 0, total = 0;
    if (e < experts) {
        if (gridDim.x == 1) {
            for (int w = 0; w < kOrderWaves; ++w) total += local[w * experts + e];
        } else {
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int c = counts[(int64_t)b * experts + e];
                before += b < (int)blockIdx.x ? c : 0;
                total += c;
            }
        }
    }
    const int sum = wave_scan(total);
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int first = sum - total, all = 0;
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) {
        first += w < wave ? wave_sums[w] : 0;
        all += wave_sums[w];
    }
    if (e < experts) {
        int at = first + before;
        for (int w = 0; w < kOrderWaves; ++w) {   // counts become the wavefronts' first rows
            const int c = local[w * experts + e];
            local[w * experts + e] = at;
            at += c;
        }
        if (blockIdx.x == 0) {
            offsets[e] = first;
            if (e == 0) offsets[experts] = all;
        }
    }
    __syncthreads();
    int* mine = local + wave * experts;
    for (int p = 0; p < kPairsOfWave; p += 64) {
        const int64_t at = (int64_t)blockIdx.x * kPairsOfBlock + wave * kPairsOfWave + p + lane;
        const int x = expert_of(indices, at, pairs, experts);
        const unsigned long long same = lanes_alike(x);
        int row = -1;
        if (x >= 0) row = mine[x] + __builtin_popcountll(same & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (x >= 0 && __builtin_ctzll(same) == lane) mine[x] += __builtin_popcountll(same);
        __builtin_amdgcn_wave_barrier();
        if (at < pairs) {
            place[at] = row;
            if (row >= 0) source[row] = (int)(at / top);
            if (at >= all) source[at] = -1;   // rows behind the last expert's
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void load8f(const void* M, int64_t row, int64_t ld, int64_t at, int64_t n, float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    const raw* p = static_cast<const raw*>(M) + row * ld + at;
    raw r[8];
    if (at + 8 <= n) {
        *reinterpret_cast<v4u*>(r) = *reinterpret_cast<const v4u_any*>(p);
        if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u*>(r + 4) = *reinterpret_cast<const v4u_any*>(p + 4);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = at + e < n ? p[e] : raw(0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Elem<TYPE>::load(r[e]);
}
template <int TYPE>
__device__ __forceinline__ void store8f(void* M, int64_t row, int64_t ld, int64_t at, int64_t n, const float (&x)[8]) {
    typedef typename Elem<TYPE>::raw raw;
    raw* p = static_cast<raw*>(M) + row * ld + at;
    raw r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = Elem<TYPE>::store(x[e]);
    if (at + 8 <= n) {
        *reinterpret_cast<v4u_any*>(p) = *reinterpret_cast<const v4u*>(r);
        if constexpr (TYPE == OZIMMU_F32) *reinterpret_cast<v4u_any*>(p + 4) = *reinterpret_cast<const v4u*>(r + 4);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < n) p[e] = r[e];
    }
}

// Y[t] = sum over j of w[t][j] O[place[t][j]], in order, in 32 bits. Bound: memory.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void combine_kernel(int top, int rows, int64_t n, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy, int per_row, int64_t items) {
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= items) return;
    const int64_t token = item / per_row, at = (item % per_row) * 8;
    float acc[8] = {};
    for (int j = 0; j < top; ++j) {
        const int row = place[token * top + j];
        const float w = weights ? weights[token * top + j] : 1.f;
        float x[8] = {};
        if ((unsigned)row < (unsigned)rows) load8f<TYPE>(O, row, ldo, at, n, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, x[e], acc[e]);
    }
    store8f<TYPE>(Y, token, ldy, at, n, acc);
}

// dO[place[t][j]] = w[t][j] dY[t] and dw[t][j] = <dY[t], O[place[t][j]]>: a wavefront takes one pair and reads both rows once. Bound: memory.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void combine_grad_kernel(int top, int rows, int64_t n, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place, const float* weights, void* dO, int64_t lddo,
                                    float* dweights, int64_t pairs) {
    const int lane = threadIdx.x & 63;
    const int64_t pair = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (pair >= pairs) return;
    const int64_t token = pair / top;
    const int row = place[pair];
    const bool there = (unsigned)row < (unsigned)rows;
    const float w = weights[pair];
    float dot = 0.f;
    if (there)
        for (int64_t at = lane * 8; at < n; at += 512) {
            float y[8], x[8];
            load8f<TYPE>(dY, token, lddy, at, n, y);
            load8f<TYPE>(O, row, ldo, at, n, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dot = fmaf(x[e], y[e], dot);
                y[e] *= w;
            }
            store8f<TYPE>(dO, row, lddo, at, n, y);
        }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) dot += __shfl_xor(dot, d);
    if (lane == 0) dweights[pair] = dot;
}

template <class F>
hipError_t by_type(int type, F&& f) {
    switch (type) {
        case OZIMMU_F32: f(std::integral_constant<int, OZIMMU_F32>{}); break;
        case OZIMMU_BF16: f(std::integral_constant<int, OZIMMU_BF16>{}); break;
        default: f(std::integral_constant<int, OZIMMU_F16>{}); break;
    }
    return hipGetLastError();
}

}  // namespace

size_t expert_order_bytes(int64_t pairs, int experts) {
    const int64_t blocks = (pairs + kPairsOfBlock - 1) / kPairsOfBlock;
    return blocks <= 1 ? 0 : (size_t)blocks * experts * sizeof(int);
}

hipError_t launch_expert_order(int t, int top, int experts, const int* indices, int* offsets, int* source, int* place, int* counts, hipStream_t st) {
    const int64_t pairs = (int64_t)t * top, blocks = std::max<int64_t>(1, (pairs + kPairsOfBlock - 1) / kPairsOfBlock);
    const int bytes = kOrderWaves * experts * (int)sizeof(int);
    if (hipError_t e = allow_dynamic_lds<expert_count_kernel>(kOrderWaves * OZIMMU_MAX_EXPERTS * (int)sizeof(int)); e != hipSuccess) return e;
    if (hipError_t e = allow_dynamic_lds<expert_place_kernel>(kOrderWaves * OZIMMU_MAX_EXPERTS * (int)sizeof(int)); e != hipSuccess) return e;
    if (blocks > 1) expert_count_kernel<<<dim3((unsigned)blocks), dim3(kOrderWaves * 64), bytes, st>>>(pairs, experts, indices, counts);
    expert_place_kernel<<<dim3((unsigned)blocks), dim3(kOrderWaves * 64), bytes, st>>>(pairs, top, experts, indices, counts, offsets, source, place);
    return hipGetLastError();
}

hipError_t launch_expert_combine(int t, int top, int rows, int64_t n, int type, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy, hipStream_t st) {
    const int64_t per_row = (n + 7) / 8, items = t * per_row, grid = (items + kThreads - 1) / kThreads;
    if (grid <= 0 || grid > INT32_MAX) return hipErrorInvalidConfiguration;
    return by_type(type, [&](auto kind) {
        combine_kernel<decltype(kind)::value><<<dim3((unsigned)grid), dim3(kThreads), 0, st>>>(top, rows, n, O, ldo, place, weights, Y, ldy, (int)per_row, items);
    });
}

hipError_t launch_expert_combine_grad(int t, int top, int rows, int64_t n, int type, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place, const float* weights, void* dO,
                                      int64_t lddo, float* dweights, hipStream_t st) {
    const int64_t pairs = (int64_t)t * top;
    const dim3 grid((unsigned)((pairs + 3) / 4));
    return by_type(type, [&](auto kind) {
        combine_grad_kernel<decltype(kind)::value><<<grid, dim3(kThreads), 0, st>>>(top, rows, n, dY, lddy, O, ldo, place, weights, dO, lddo, dweights, pairs);
    });
}

}  // namespace ozimmu
