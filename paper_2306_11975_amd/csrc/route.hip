// The choice of experts for each token, and its gradient (gfx950). A wavefront takes a token; lane l holds experts l, l + 64, ...
//
// Scores s: softmax or sigmoid of the logits. Choice values s + bias; of `groups` equal runs of experts the top_groups best stay, a group's
// value being the sum of its two largest choice values; of what stays the `top` best are chosen, ties going to the lowest index. Scores and
// choice values are in 64 bits: neighbours among hundreds of experts come nearer than 32-bit roundings about once in 10^5 tokens, and then
// the index would depend on the rounding.
#include <algorithm>

#include "f8_common.h"

namespace ozimmu {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double shuffle_xor(double x, int d) { return __shfl_xor(x, d); }
__device__ __forceinline__ double wave_max(double x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = fmax(x, shuffle_xor(x, d));
    return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += shuffle_xor(x, d);
    return x;
}
// The larger value, of equals the lower index; -inf with index INT_MAX is nothing.
__device__ __forceinline__ void better(double& v, int& i, double v2, int i2) {
    const bool take = v2 > v || (v2 == v && i2 < i);
    v = take ? v2 : v;
    i = take ? i2 : i;
}
__device__ __forceinline__ void wave_best(double& v, int& i) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) better(v, i, shuffle_xor(v, d), __shfl_xor(i, d));
}

// Scores of the token's experts. bad: the row holds what has no order (a NaN; for softmax an infinity of logits).
template <int TYPE, int SLOTS>
__device__ __forceinline__ void scores(const RouteArgs& a, int64_t token, int lane, double (&l)[SLOTS], double (&s)[SLOTS], bool& bad) {
    typedef typename Elem<TYPE>::raw raw;
    const raw* row = static_cast<const raw*>(a.logits) + token * a.ldl;
    double top = -INFINITY;
    bad = false;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int e = k * 64 + lane;
        l[k] = e < a.experts ? (double)Elem<TYPE>::load(row[e]) : -INFINITY;
        bad |= l[k] != l[k] || (!a.sigmoid && l[k] == INFINITY);
        top = fmax(top, l[k]);
    }
    bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (a.sigmoid) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) s[k] = 1.0 / (1.0 + exp(-l[k]));
    } else {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            s[k] = l[k] == -INFINITY ? 0.0 : exp(l[k] - top);
            sum += s[k];
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) s[k] = sum > 0.0 ? s[k] / sum : 0.0;
    }
}

template <int TYPE, int SLOTS>
__launch_bounds__(kThreads)
__global__ void route_kernel(RouteArgs a, int* indices, float* weights) {
    __shared__ double values[kThreads / 64][SLOTS * 64];
    __shared__ unsigned long long kept[kThreads / 64][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (token >= a.t) return;
    double l[SLOTS], s[SLOTS], c[SLOTS];
    bool bad;
    scores<TYPE, SLOTS>(a, token, lane, l, s, bad);
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int e = k * 64 + lane;
        c[k] = l[k] == -INFINITY ? -INFINITY : a.bias ? s[k] + (double)a.bias[e] : s[k];
        bad |= c[k] != c[k];
    }
    bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (a.groups > 1) {
        const int per = a.experts / a.groups;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) values[wave][k * 64 + lane] = c[k];
        if (lane < 16) kept[wave][lane] = 0;
        __builtin_amdgcn_wave_barrier();
        // groups lane, lane + 64, ...: the two largest of each
        double g[16];
        const int rounds = (a.groups + 63) / 64;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            g[r] = -INFINITY;
            const int group = r * 64 + lane;
            if (r >= rounds || group >= a.groups) continue;
            double first = -INFINITY, second = -INFINITY;
            for (int e = 0; e < per; ++e) {
                const double x = values[wave][group * per + e];
                second = fmax(second, fmin(first, x));
                first = fmax(first, x);
            }
            g[r] = second == -INFINITY ? first : first + second;
        }
        for (int n = 0; n < a.top_groups; ++n) {
            double v = -INFINITY;
            int i = INT32_MAX;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (g[r] > -INFINITY) better(v, i, g[r], r * 64 + lane);
            wave_best(v, i);
            if (i == INT32_MAX) break;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r * 64 + lane == i) g[r] = -INFINITY;
            if (lane == 0) kept[wave][i >> 6] |= 1ull << (i & 63);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int group = min((k * 64 + lane) / per, a.groups - 1);
            if (!(kept[wave][group >> 6] >> (group & 63) & 1)) c[k] = -INFINITY;
        }
    }
    // the best, one after the other; lane j keeps choice j
    int mine = -1;
    double score = 0.0, logit = -INFINITY;
    if (!bad)
        for (int j = 0; j < a.top; ++j) {
            double v = -INFINITY;
            int i = INT32_MAX;
#pragma unroll
            for (int k = 0; k < SLOTS; ++k)
                if (c[k] > -INFINITY) better(v, i, c[k], k * 64 + lane);
            wave_best(v, i);
            if (i == INT32_MAX) break;
            double sc = 0.0, lg = 0.0;
#pragma unroll
            for (int k = 0; k < SLOTS; ++k)
                if (k == (i >> 6)) {
                    if (lane == (i & 63)) c[k] = -INFINITY;
                    sc = s[k];
                    lg = l[k];
                }
            sc = __shfl(sc, i & 63);
            lg = __shfl(lg, i & 63);
            if (lane == j) {
                mine = i;
                score = sc;
                logit = lg;
            }
        }
    double w = score;
    if (a.renormalize) {
        if (a.sigmoid) {
            w = score / (wave_sum(score) + 1e-20);
        } else {   // of the chosen logits alone: nothing underflows
            const double top = wave_max(logit);
            const double x = mine >= 0 ? exp(logit - top) : 0.0, sum = wave_sum(x);
            w = sum > 0.0 ? x / sum : 0.0;
        }
    }
    if (lane < a.top) {
        indices[token * a.top + lane] = mine;
        weights[token * a.top + lane] = bad ? __builtin_nanf("") : mine < 0 ? 0.f : (float)(w * (double)a.scale);
    }
}

template <int TYPE, int SLOTS>
__launch_bounds__(kThreads)
__global__ void route_grad_kernel(RouteArgs a, const int* indices, const float* dweights, void* dlogits, int64_t lddl) {
    typedef typename Elem<TYPE>::raw raw;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (token >= a.t) return;
    double l[SLOTS], s[SLOTS], g[SLOTS];
    bool bad;
    scores<TYPE, SLOTS>(a, token, lane, l, s, bad);
    int mine = lane < a.top ? indices[token * a.top + lane] : -1;
    if ((unsigned)mine >= (unsigned)a.experts) mine = -1;
    const double dw = mine >= 0 ? (double)dweights[token * a.top + lane] * (double)a.scale : 0.0;
    double score = 0.0, logit = -INFINITY;
    for (int j = 0; j < a.top; ++j) {   // lane j's choice: its score
        const int i = __shfl(mine, j);
        if (i < 0) continue;
        double sc = 0.0, lg = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (k == (i >> 6)) {
                sc = s[k];
                lg = l[k];
            }
        sc = __shfl(sc, i & 63);
        lg = __shfl(lg, i & 63);
        if (lane == j) {
            score = sc;
            logit = lg;
        }
    }
    // d: what goes to the chosen logit; for softmax scores that are not renormalised, every logit receives -s (sum of score gradients times scores)
    double d, all = 0.0;
    if (a.renormalize) {
        if (a.sigmoid) {
            const double total = wave_sum(score) + 1e-20, mean = wave_sum(dw * score) / total;
            d = (dw - mean) / total * score * (1.0 - score);
        } else {
            const double top = wave_max(logit);
            const double x = mine >= 0 ? exp(logit - top) : 0.0, sum = wave_sum(x), w = sum > 0.0 ? x / sum : 0.0;
            d = w * (dw - wave_sum(dw * w));
        }
    } else if (a.sigmoid) {
        d = dw * score * (1.0 - score);
    } else {
        d = dw * score;
        all = wave_sum(d);
    }
    const bool any = __builtin_amdgcn_ballot_w64(mine >= 0) != 0;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) g[k] = any && all != 0.0 ? -s[k] * all : 0.0;
    for (int j = 0; j < a.top; ++j) {
        const int i = __shfl(mine, j);
        const double x = __shfl(d, j);
        if (i < 0) continue;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (k * 64 + lane == i) g[k] += x;
    }
    raw* row = static_cast<raw*>(dlogits) + token * lddl;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int e = k * 64 + lane;
        if (e < a.experts) row[e] = Elem<TYPE>::store((float)(bad && any ? (double)__builtin_nanf("") : l[k] == -INFINITY ? 0.0 : g[k]));
    }
}

template <class F>
hipError_t by_shape(int type, int experts, F&& f) {
    auto by_slots = [&](auto kind) {
        if (experts <= 64)
            f(kind, std::integral_constant<int, 1>{});
        else if (experts <= 128)
            f(kind, std::integral_constant<int, 2>{});
        else if (experts <= 256)
            f(kind, std::integral_constant<int, 4>{});
        else if (experts <= 512)
            f(kind, std::integral_constant<int, 8>{});
        else
            f(kind, std::integral_constant<int, 16>{});
    };
    if (type == OZIMMU_F32)
        by_slots(std::integral_constant<int, OZIMMU_F32>{});
    else if (type == OZIMMU_BF16)
        by_slots(std::integral_constant<int, OZIMMU_BF16>{});
    else
        by_slots(std::integral_constant<int, OZIMMU_F16>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, int* indices, float* weights, hipStream_t st) {
    const dim3 grid((unsigned)((a.t + 3) / 4));
    return by_shape(a.type, a.experts, [&](auto kind, auto slots) {
        route_kernel<decltype(kind)::value, decltype(slots)::value><<<grid, dim3(kThreads), 0, st>>>(a, indices, weights);
    });
}

hipError_t launch_route_grad(const RouteArgs& a, const int* indices, const float* dweights, void* dlogits, int64_t lddl, hipStream_t st) {
    const dim3 grid((unsigned)((a.t + 3) / 4));
    return by_shape(a.type, a.experts, [&](auto kind, auto slots) {
        route_grad_kernel<decltype(kind)::value, decltype(slots)::value><<<grid, dim3(kThreads), 0, st>>>(a, indices, dweights, dlogits, lddl);
    });
}

}  // namespace ozimmu
