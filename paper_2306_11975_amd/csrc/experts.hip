// Rows sorted by expert, and the experts' results brought back to the tokens, with its gradient (gfx950). No atomics: equal calls give equal
// bits.
#include <algorithm>

#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;
// Stable sort by counting. Pass one (where there is more than one workgroup): every workgroup counts its pairs by expert. Pass two: the pairs
// before the workgroup's own, by expert and in all, give each expert's first row; within the workgroup wavefronts count again, in order, and within
// a wavefront a pair's rank is the number of lower lanes with its expert, from ten ballots over the bits of the expert's number. Up to kSumBlocks
// workgroups each adds up the others' counts itself; beyond, a pass between turns them into first rows. Bound: latency, in steps that follow each
// other. 131072 pairs, 256 experts, us: 18.4 with 256 pairs to a wavefront, 11.8 with 64 (12.6 with the pass between).
constexpr int kOrderWaves = 16;       // of a workgroup, at most
constexpr int kOrderThreads = 1024;
constexpr int kSumBlocks = 128;
constexpr int64_t kManyPairs = 262144;
// pairs that a wavefront takes, 64 at a time
int pairs_of_wave(int64_t pairs) { return pairs <= kManyPairs ? 64 : 512; }
int64_t order_blocks(int64_t pairs) { return std::max<int64_t>(1, (pairs + kOrderWaves * pairs_of_wave(pairs) - 1) / (kOrderWaves * pairs_of_wave(pairs))); }

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
// counts[wave][expert] of the workgroup's pairs, `waves` wavefronts with `each`
__device__ __forceinline__ void count_pairs(const int* indices, int64_t pairs, int experts, int waves, int each, int* counts) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < experts * waves; e += blockDim.x) counts[e] = 0;
    __syncthreads();
    if (wave < waves) {
        int* mine = counts + wave * experts;
        const int64_t first = ((int64_t)blockIdx.x * waves + wave) * each;
        for (int p = 0; p < each && first + p < pairs; p += 64) {
            const int e = expert_of(indices, first + p + lane, pairs, experts);
            const unsigned long long same = lanes_alike(e);
            if (e >= 0 && __builtin_ctzll(same) == lane) mine[e] += __builtin_popcountll(same);
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
}

__launch_bounds__(kOrderThreads)
__global__ void expert_count_kernel(int64_t pairs, int experts, int each, const int* indices, int* counts) {
    extern __shared__ int local[];
    count_pairs(indices, pairs, experts, kOrderWaves, each, local);
    for (int e = threadIdx.x; e < experts; e += blockDim.x) {
        int sum = 0;
        for (int w = 0; w < kOrderWaves; ++w) sum += local[w * experts + e];
        counts[(int64_t)blockIdx.x * experts + e] = sum;
    }
}

// Counts become the numbers of pairs before each workgroup's, their sums the last row: a workgroup takes 64 experts, its wavefronts runs of blocks.
__launch_bounds__(kOrderThreads)
__global__ void expert_sum_kernel(int blocks, int experts, int* counts) {
    __shared__ int runs[kOrderWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const int each = (blocks + kOrderWaves - 1) / kOrderWaves, from = wave * each, to = min(blocks, from + each);
    int sum = 0;
    if (e < experts)
#pragma unroll 8
        for (int b = from; b < to; ++b) sum += counts[(int64_t)b * experts + e];
    runs[wave][lane] = sum;
    __syncthreads();
    if (e >= experts) return;
    int before = 0, all = 0;
    for (int w = 0; w < kOrderWaves; ++w) {
        before += w < wave ? runs[w][lane] : 0;
        all += runs[w][lane];
    }
#pragma unroll 8
    for (int b = from; b < to; ++b) {
        const int c = counts[(int64_t)b * experts + e];
        counts[(int64_t)b * experts + e] = before;
        before += c;
    }
    if (wave == 0) counts[(int64_t)blocks * experts + e] = all;
}

__launch_bounds__(kOrderThreads)
__global__ void expert_place_kernel(int64_t pairs, int top, int experts, int waves, int each, const int* indices, const int* counts, int* offsets, int* source, int* place) {
    extern __shared__ int local[];      // counts of each wavefront and expert
    __shared__ int wave_sums[kOrderWaves], others[2][kOrderThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    count_pairs(indices, pairs, experts, waves, each, local);
    // Each expert's pairs in the workgroups before this one, and in all. Several threads share an expert's column where there are threads for it.
    int before = 0, total = 0;
    const int e = threadIdx.x;
    if (gridDim.x == 1) {
        if (e < experts)
            for (int w = 0; w < waves; ++w) total += local[w * experts + e];
    } else if ((int)gridDim.x > kSumBlocks) {
        if (e < experts) {
            before = counts[(int64_t)blockIdx.x * experts + e];
            total = counts[(int64_t)gridDim.x * experts + e];
        }
    } else {
        const int teams = max(1, (int)blockDim.x / experts), team = threadIdx.x / experts, column = threadIdx.x - team * experts;
        if (team < teams) {
#pragma unroll 8
            for (int b = team; b < (int)gridDim.x; b += teams) {
                const int c = counts[(int64_t)b * experts + column];
                before += b < (int)blockIdx.x ? c : 0;
                total += c;
            }
            others[0][threadIdx.x] = before;
            others[1][threadIdx.x] = total;
        }
        __syncthreads();
        before = total = 0;
        if (e < experts)
            for (int i = 0; i < teams; ++i) {
                before += others[0][i * experts + e];
                total += others[1][i * experts + e];
            }
    }
    const int sum = wave_scan(total);
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    int first = sum - total, all = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        first += w < wave ? wave_sums[w] : 0;
        all += wave_sums[w];
    }
    if (e < experts) {
        int at = first + before;
        for (int w = 0; w < waves; ++w) {   // counts become the wavefronts' first rows
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
    if (wave >= waves) return;
    int* mine = local + wave * experts;
    const int64_t from = ((int64_t)blockIdx.x * waves + wave) * each;
    for (int p = 0; p < each && from + p < pairs; p += 64) {
        const int64_t at = from + p + lane;
        const int x = expert_of(indices, at, pairs, experts);
        const unsigned long long same = lanes_alike(x);
        int row = -1;
        if (x >= 0) row = mine[x] + __builtin_popcountll(same & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (x >= 0 && __builtin_ctzll(same) == lane) mine[x] += __builtin_popcountll(same);
        __builtin_amdgcn_wave_barrier();
        if (at < pairs) {
            place[at] = row;
            if (row >= 0) source[row] = (int)((unsigned)at / (unsigned)top);
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

// Y[t] = sum over j of w[t][j] O[place[t][j]], in order, in 32 bits: a wavefront takes 512 columns of a token, eight to a lane, and asks for four
// rows at a time; a workgroup's four lie side by side in a row as far as it goes (8192 tokens of eight rows of 4096 bf16: 138 us, 604 MB; a wavefront to a token 160).
// Bound: memory.
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void combine_kernel(int t, int top, int rows, int64_t n, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy, int across) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tokens = 4 / across;
    const int64_t token = (int64_t)blockIdx.x * tokens + wave / across, at = ((int64_t)blockIdx.y * across + wave % across) * 512 + (threadIdx.x & 63) * 8;
    if (token >= t || at >= n) return;
    const int* where = place + token * top;
    float acc[8] = {};
    for (int j0 = 0; j0 < top; j0 += 4) {
        float x[4][8], w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = j0 + j < top ? where[j0 + j] : -1;
            w[j] = j0 + j >= top ? 0.f : weights ? weights[token * top + j0 + j] : 1.f;
            if ((unsigned)row < (unsigned)rows)
                load8f<TYPE>(O, row, ldo, at, n, x[j]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(w[j], x[j][e], acc[e]);
    }
    store8f<TYPE>(Y, token, ldy, at, n, acc);
}

// dO[place[t][j]] = w[t][j] dY[t] and dw[t][j] = <dY[t], O[place[t][j]]>: a wavefront takes one pair and reads both rows once. Bound: memory
// (8192 tokens of eight rows of 4096 bf16: 211 us, 1.14 GB).
template <int TYPE>
__launch_bounds__(kThreads)
__global__ void combine_grad_kernel(int top, int rows, int64_t n, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place, const float* weights, void* dO, int64_t lddo,
                                    float* dweights, int64_t pairs) {
    const int lane = threadIdx.x & 63;
    const int64_t pair = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (pair >= pairs) return;
    const int64_t token = (unsigned)pair / (unsigned)top;
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
    const int64_t blocks = std::max(order_blocks(pairs), order_blocks(std::min(pairs, kManyPairs)));   // (one for more pairs serves fewer)
    return blocks <= 1 ? 0 : (size_t)(blocks + 1) * experts * sizeof(int);
}

hipError_t launch_expert_order(int t, int top, int experts, const int* indices, int* offsets, int* source, int* place, int* counts, hipStream_t st) {
    const int64_t pairs = (int64_t)t * top, blocks = order_blocks(pairs);
    const int each = pairs_of_wave(pairs);
    if (hipError_t e = allow_dynamic_lds<expert_count_kernel>(kOrderWaves * OZIMMU_MAX_EXPERTS * (int)sizeof(int)); e != hipSuccess) return e;
    if (hipError_t e = allow_dynamic_lds<expert_place_kernel>(kOrderWaves * OZIMMU_MAX_EXPERTS * (int)sizeof(int)); e != hipSuccess) return e;
    // few pairs: no more wavefronts than have some, and a thread for each expert
    const int waves = blocks > 1 ? kOrderWaves : (int)std::max<int64_t>(1, (pairs + each - 1) / each);
    const int threads = blocks > 1 ? kOrderThreads : std::max(64 * waves, (experts + 63) / 64 * 64), bytes = waves * experts * (int)sizeof(int);
    if (blocks > 1) expert_count_kernel<<<dim3((unsigned)blocks), dim3(threads), bytes, st>>>(pairs, experts, each, indices, counts);
    if (blocks > kSumBlocks) expert_sum_kernel<<<dim3((unsigned)(experts + 63) / 64), dim3(kOrderThreads), 0, st>>>((int)blocks, experts, counts);
    expert_place_kernel<<<dim3((unsigned)blocks), dim3(threads), bytes, st>>>(pairs, top, experts, waves, each, indices, counts, offsets, source, place);
    return hipGetLastError();
}

hipError_t launch_expert_combine(int t, int top, int rows, int64_t n, int type, const void* O, int64_t ldo, const int* place, const float* weights, void* Y, int64_t ldy, hipStream_t st) {
    const int64_t chunks = (n + 511) / 512;
    const int across = chunks >= 3 ? 4 : chunks == 2 ? 2 : 1, tokens = 4 / across;
    const dim3 grid((unsigned)((t + tokens - 1) / tokens), (unsigned)((chunks + across - 1) / across));
    return by_type(type, [&](auto kind) {
        combine_kernel<decltype(kind)::value><<<grid, dim3(kThreads), 0, st>>>(t, top, rows, n, O, ldo, place, weights, Y, ldy, across);
    });
}

hipError_t launch_expert_combine_grad(int t, int top, int rows, int64_t n, int type, const void* dY, int64_t lddy, const void* O, int64_t ldo, const int* place, const float* weights, void* dO,
                                      int64_t lddo, float* dweights, hipStream_t st) {
    const int64_t pairs = (int64_t)t * top, blocks = (pairs + 3) / 4, across = std::min<int64_t>(blocks, 1 << 23);      // (2^32 threads are too many for one dimension)
    const dim3 grid((unsigned)across, (unsigned)((blocks + across - 1) / across));
    return by_type(type, [&](auto kind) {
        combine_grad_kernel<decltype(kind)::value><<<grid, dim3(kThreads), 0, st>>>(top, rows, n, dY, lddy, O, ldo, place, weights, dO, lddo, dweights, pairs);
    });
}

}  // namespace ozimmu
