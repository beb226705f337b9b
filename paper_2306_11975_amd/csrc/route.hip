// The choice of experts for each token, and its gradient (gfx950). First the form that computes everything in 64 bits, a wavefront to a token, lane l
// with experts l, l + 64, ...: it serves groups that do not fill whole lanes. Below it the one that goes by 32 bits wherever those tell.
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

// The choice in 64 bits throughout. values, kept: LDS of this wavefront.
template <int TYPE, int SLOTS>
__device__ __forceinline__ void route_exactly(const RouteArgs& a, int64_t token, int lane, double* values, unsigned long long* kept, int* indices, float* weights) {
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
        for (int k = 0; k < SLOTS; ++k) values[k * 64 + lane] = c[k];
        if (lane < 16) kept[lane] = 0;
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
                const double x = values[group * per + e];
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
            if (lane == 0) kept[i >> 6] |= 1ull << (i & 63);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int group = min((k * 64 + lane) / per, a.groups - 1);
            if (!(kept[group >> 6] >> (group & 63) & 1)) c[k] = -INFINITY;
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
__global__ void route_exactly_kernel(RouteArgs a, int* indices, float* weights) {
    __shared__ double values[kThreads / 64][SLOTS * 64];
    __shared__ unsigned long long kept[kThreads / 64][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (token < a.t) route_exactly<TYPE, SLOTS>(a, token, lane, values[wave], kept[wave], indices, weights);
}

// ---- the same in 32 bits, where those tell

// Reductions over LANES lanes (a row of 16, or all 64), the result in each of them.
template <int CTRL>
__device__ __forceinline__ unsigned row_turned(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ double row_turned(double x) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return __longlong_as_double((long long)((unsigned long long)row_turned<CTRL>((unsigned)(b >> 32)) << 32 | row_turned<CTRL>((unsigned)b)));
}
template <int CTRL>
__device__ __forceinline__ float row_turned(float x) { return __uint_as_float(row_turned<CTRL>(__float_as_uint(x))); }
template <int CTRL>
__device__ __forceinline__ unsigned long long row_turned(unsigned long long x) {
    return (unsigned long long)row_turned<CTRL>((unsigned)(x >> 32)) << 32 | row_turned<CTRL>((unsigned)x);
}
template <int LANES, class T, class F>
__device__ __forceinline__ T over_lanes(T x, F&& f) {
    x = f(x, row_turned<0x128>(x));   // rotations of a row by 8, 4, 2 and 1
    x = f(x, row_turned<0x124>(x));
    x = f(x, row_turned<0x122>(x));
    x = f(x, row_turned<0x121>(x));
    if constexpr (LANES == 64) {
        x = f(x, __shfl_xor(x, 16));
        x = f(x, __shfl_xor(x, 32));
    }
    return x;
}
template <int LANES, class T>
__device__ __forceinline__ T most(T x) { return over_lanes<LANES>(x, [](T p, T q) { return p > q ? p : q; }); }
template <int LANES>
__device__ __forceinline__ unsigned least(unsigned x) { return over_lanes<LANES>(x, [](unsigned p, unsigned q) { return min(p, q); }); }
template <int LANES, class T>
__device__ __forceinline__ T sum_of(T x) { return over_lanes<LANES>(x, [](T p, T q) { return p + q; }); }

// SLOTS neighbouring experts of a lane.
template <int TYPE, int SLOTS>
__device__ __forceinline__ void load_experts(const typename Elem<TYPE>::raw* row, int experts, int lane, float (&l)[SLOTS]) {
    typedef typename Elem<TYPE>::raw raw;
    row += lane * SLOTS;
    constexpr int words = SLOTS * (int)sizeof(raw) / 4;
    raw r[SLOTS];
    if (words > 0 && lane * SLOTS + SLOTS <= experts) {
        typedef unsigned many __attribute__((ext_vector_type(words > 4 ? 4 : words > 0 ? words : 1)));
        typedef many many_any __attribute__((aligned(2)));
#pragma unroll
        for (int w = 0; w < (words + 3) / 4; ++w) reinterpret_cast<many*>(r)[w] = reinterpret_cast<const many_any*>(row)[w];
    } else {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (lane * SLOTS + k < experts) r[k] = row[k];
    }
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) l[k] = lane * SLOTS + k < experts ? Elem<TYPE>::load(r[k]) : -INFINITY;
}
// Bits that order like the values; 0 for what cannot be chosen.
template <class V> struct Bits;
template <> struct Bits<float> {
    typedef unsigned type;
    static __device__ __forceinline__ type of(float x) {
        const unsigned b = __float_as_uint(x + 0.f);   // (-0 is 0)
        return x == -INFINITY ? 0u : b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
    }
    static __device__ __forceinline__ float value(type k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
};
template <> struct Bits<double> {
    typedef unsigned long long type;
    static __device__ __forceinline__ type of(double x) {
        const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
        return x == -INFINITY ? 0ull : b ^ (b >> 63 ? ~0ull : 1ull << 63);
    }
};

// A group is `width` neighbouring lanes. From each lane's two largest values (-inf: none): whether its group is one of the best top_groups, by the
// sum of its two. V = float: unsure where a group that is kept and one that is not are too near each other to tell. What a sum may be off by: its two
// values' roundings and its own, 2^-24 of each, which outlast the sum where the two cancel, and the two scores' errors. A sum beyond 32 bits tells
// nothing but its sign.
template <int LANES, class V>
__device__ __forceinline__ bool in_best_groups(const RouteArgs& a, int lane, bool there, int width, V first, V second, float near_scores, bool& unsure) {
    typedef typename Bits<V>::type bits;
    for (int d = 1; d < width; d <<= 1) {
        const V f = __shfl_xor(first, d), g = __shfl_xor(second, d);
        second = max(max(second, g), min(first, f));
        first = max(first, f);
    }
    constexpr float kMost = 0x1.fffffep127f;
    const bool one = second == -INFINITY;
    V sum = one ? first : first + second;
    if constexpr (sizeof(V) == 4) sum = one ? sum : max(sum, -kMost);      // (-inf is a group of which nothing can be chosen)
    bits key = there ? Bits<V>::of(sum) : 0;
    bool keep = false;
    for (int n = 0; n < a.top_groups; ++n) {
        const bits best = most<LANES>(key);
        const int at = (int)least<LANES>(key == best ? (unsigned)lane : 64u) / width;
        if (best != 0 && lane / width == at) {
            keep = true;
            key = 0;
        }
    }
    if constexpr (sizeof(V) == 4) {   // which ones are kept matters, not their order: the least that a kept one may be against the most that another may
        const float off = 2.f * near_scores + fabsf(first) * 0x1p-22f + (one ? 0.f : fabsf(second) * 0x1p-22f);
        const bool beyond = !(fabsf(sum) < kMost);
        const float low = first == INFINITY ? INFINITY : beyond ? -INFINITY : sum - off, high = beyond ? sum : sum + off;
        const float kept = -most<LANES>(keep ? -low : -INFINITY), other = most<LANES>(key != 0 ? high : -INFINITY);
        unsure |= !(kept > other) && other > -INFINITY;
    }
    return keep;
}
template <int SLOTS, class V>
__device__ __forceinline__ void two_largest(const V (&c)[SLOTS], V& first, V& second) {
    first = second = -INFINITY;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        second = max(second, min(first, c[k]));
        first = max(first, c[k]);
    }
}

// Lane j < top keeps the expert of round j (0xffffffff: none), the one with the largest value, of equals the lowest.
template <int LANES, int SLOTS>
__device__ __forceinline__ unsigned choose_exactly(const RouteArgs& a, int lane, const double (&c)[SLOTS]) {
    unsigned long long key[SLOTS];
    unsigned mine = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) key[k] = Bits<double>::of(c[k]);
    for (int j = 0; j < a.top; ++j) {
        unsigned long long here = key[0];
        unsigned slot = 0;
#pragma unroll
        for (int k = 1; k < SLOTS; ++k) {
            slot = key[k] > here ? (unsigned)k : slot;
            here = key[k] > here ? key[k] : here;
        }
        const unsigned long long best = most<LANES>(here);
        const unsigned winner = least<LANES>(here == best && best != 0 ? (unsigned)lane * SLOTS + slot : 0xffffffffu);
        mine = lane == j ? winner : mine;
        const unsigned gone = winner - (unsigned)lane * SLOTS;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) key[k] = gone == (unsigned)k ? 0 : key[k];
    }
    return mine;
}

// A sorting network, Batcher's odd-even merge sort (1968): pairs of places, the larger value to the first.
template <int N>
struct Network {
    int first[80], second[80], count;
    constexpr Network() : first(), second(), count(0) {
        for (int p = 1; p < N; p *= 2)
            for (int k = p; k >= 1; k /= 2)
                for (int j = k % p; j <= N - 1 - k; j += 2 * k)
                    for (int i = 0; i < k && i + j + k < N; ++i)
                        if ((i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                            first[count] = i + j;
                            second[count++] = i + j + k;
                        }
    }
};
// The same by 32-bit values, whose last bits (those of SLOTS - 1) make room for the slot: each lane sorts its keys once, and a round takes the
// largest of their heads; the winner's move up.
template <int LANES, int SLOTS>
struct Sorted {
    static constexpr unsigned kSlot = SLOTS - 1;
    unsigned key[SLOTS];
    __device__ __forceinline__ explicit Sorted(const float (&c)[SLOTS]) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const unsigned b = Bits<float>::of(c[k]);
            key[k] = b == 0 ? 0 : (b & ~kSlot) | (kSlot - k);
        }
        constexpr Network<SLOTS> network;
        static_for<0, network.count>([&](auto n) {
            constexpr Network<SLOTS> w;
            constexpr int i = w.first[decltype(n)::value], j = w.second[decltype(n)::value];
            const unsigned high = max(key[i], key[j]), low = min(key[i], key[j]);
            key[i] = high;
            key[j] = low;
        });
    }
    // The expert (0xffffffff: none) and its value's bits.
    __device__ __forceinline__ unsigned next(int lane, unsigned& best) {
        const unsigned here = key[0] & ~kSlot;
        best = most<LANES>(here);
        const unsigned expert = (unsigned)lane * SLOTS + (kSlot - (key[0] & kSlot));
        const unsigned winner = least<LANES>(here == best && best != 0 ? expert : 0xffffffffu);
        const bool won = winner == expert && best != 0;
#pragma unroll
        for (int k = 0; k + 1 < SLOTS; ++k) key[k] = won ? key[k + 1] : key[k];
        key[SLOTS - 1] = won ? 0 : key[SLOTS - 1];
        return winner;
    }
};

// LANES lanes to a token (16: four tokens a wavefront), experts lane * SLOTS + k. The choice goes by 32-bit values where their order is beyond
// doubt: without a bias and groups by the logits themselves, whose order the scores have (sigmoid's down to -700), else by scores that are off by less than 2^-20 of the
// largest, plus their bias. Where two neighbours among the best top + 1 are as near as that, and not equal in all that they come from, those
// top + 1 are put in order by their 64-bit values (at 256 experts with sigmoid scores and a bias one token in some hundreds); where the last
// group kept and the next are as near (one token in some ten thousands), the groups by the 64-bit values of their best; where those top + 1 need
// not hold all that are that near, or the sum of all scores would be needed, the wavefront's tokens are chosen again from all 64-bit values. Each round finds the largest value, then the lowest expert that has it, and takes that out; lane j keeps the
// round's, so that neighbours and weights are looked at once, all together. Bound: the rounds' instructions.
// 16384 tokens, 256 experts in 8 groups, 8 of 4 groups, us: all in 64 bits 80, 64 lanes to a token 48, 16 lanes 26, the lanes' keys sorted 24,
// and 64-bit values of the few in doubt 17.
template <int TYPE, int LANES, int SLOTS>
__launch_bounds__(kThreads)
__global__ void route_kernel(RouteArgs a, int* indices, float* weights) {
    typedef typename Elem<TYPE>::raw raw;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t mine_token = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
    const bool there = mine_token < a.t;
    if (__builtin_amdgcn_ballot_w64(there) == 0) return;
    const int64_t token = there ? mine_token : a.t - 1;      // (rows beyond the last do it again, and write nothing)
    float l[SLOTS], b[SLOTS], c[SLOTS];
    load_experts<TYPE, SLOTS>(static_cast<const raw*>(a.logits) + token * a.ldl, a.experts, lane, l);
    if (a.bias) load_experts<OZIMMU_F32, SLOTS>(a.bias, a.experts, lane, b);
    bool odd = false, bad = false;      // what 64 bits may not tell apart; what has no order
    unsigned top_bits = 0;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        odd |= l[k] > 10.f && a.sigmoid;
        bad |= l[k] != l[k] || (!a.sigmoid && l[k] == INFINITY);
        if (!a.sigmoid) top_bits = max(top_bits, Bits<float>::of(l[k]));
    }
    const bool by_values = a.bias != nullptr || a.groups > 1;      // (the same for all)
    if (!a.sigmoid) top_bits = most<LANES>(top_bits);
    const float top_logit = Bits<float>::value(top_bits);
    float largest = 1.f;      // a score is at most that
    if (by_values) {
        if (a.sigmoid) {
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) c[k] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * l[k]));
        } else {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) {
                c[k] = l[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(1.44269504f * (l[k] - top_logit));
                sum += c[k];
            }
            largest = 1.f / sum_of<LANES>(sum);
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) c[k] *= largest;
        }
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if (a.bias) {
                bad |= l[k] != -INFINITY && c[k] + b[k] != c[k] + b[k];
                c[k] += b[k];
            }
            c[k] = l[k] == -INFINITY ? -INFINITY : c[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) c[k] = l[k];
    }
    // Scores: the argument of the exponential is rounded to 2^-23 of itself; |l| <= 10 for sigmoid, whose slope is at most 1 / 4, and for softmax
    // the argument's size times the score is below one half of the largest.
    const float near_scores = largest * 0x1p-20f;
    // (the values' last bits are gone; and logits nearer than 1e-9 may have one score in 64 bits)
    auto apart = [&](float v, float w) { return v - w > (by_values ? 2.f * near_scores : 1e-9f) + (fabsf(v) + fabsf(w)) * 0x1p-18f; };
    bool unsure = false, all = odd;     // neighbours too near; only the choice among all experts will tell
    const int width = a.groups > 1 ? a.experts / a.groups / SLOTS : 1;
    const bool some = lane * SLOTS < a.experts;
    if (a.groups > 1) {
        float first, second;
        two_largest(c, first, second);
        bool near_groups = false, keep = in_best_groups<LANES>(a, lane, some, width, first, second, near_scores, near_groups);
        if (!a.sigmoid) {
            all |= near_groups;
        } else if (__builtin_amdgcn_ballot_w64(near_groups)) {
            // the groups by 64-bit values of those that may be the two largest of their lane
            const float border = second == INFINITY ? second : second - (2.f * near_scores + fabsf(second) * 0x1p-21f);
            unsigned left = 0;
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) left |= c[k] > -INFINITY && c[k] >= border ? 1u << k : 0u;
            double first64 = -INFINITY, second64 = -INFINITY;
            while (__builtin_amdgcn_ballot_w64(left != 0)) {
                const unsigned slot = (unsigned)__builtin_ctz(left | 1u << 31);
                float logit = 0.f, bias = 0.f;
#pragma unroll
                for (int k = 0; k < SLOTS; ++k) {
                    logit = slot == (unsigned)k ? l[k] : logit;
                    if (a.bias) bias = slot == (unsigned)k ? b[k] : bias;
                }
                const double value = left ? 1.0 / (1.0 + exp(-(double)logit)) + (double)bias : -INFINITY;
                second64 = max(second64, min(first64, value));
                first64 = max(first64, value);
                left &= left - 1;
            }
            keep = in_best_groups<LANES>(a, lane, some, width, first64, second64, 0.f, near_groups);
        }
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) c[k] = keep ? c[k] : -INFINITY;
    }
    Sorted<LANES, SLOTS> sorted(c);
    unsigned mine = 0xffffffffu, mine_bits = 0;
    for (int j = 0; j <= a.top; ++j) {      // (lane top: the best that is not chosen)
        unsigned best;
        const unsigned winner = sorted.next(lane, best);
        mine = lane == j ? winner : mine;
        mine_bits = lane == j ? best : mine_bits;
    }
    constexpr unsigned long long kMask = LANES == 64 ? ~0ull : (1ull << (LANES & 63)) - 1;
    const int row0 = (threadIdx.x & 63) / LANES * LANES;
    float logit = -INFINITY, bias = 0.f;
    {   // neighbours: lane j against lane j - 1
        if (mine != 0xffffffffu) {
            logit = Elem<TYPE>::load((static_cast<const raw*>(a.logits) + token * a.ldl)[mine]);
            if (a.bias) bias = a.bias[mine];
        }
        const float v = Bits<float>::value((unsigned)__shfl_up((int)mine_bits, 1)), w = Bits<float>::value(mine_bits);
        const float logit_before = __shfl_up(logit, 1), bias_before = __shfl_up(bias, 1);      // (of all lanes: behind a condition they would be of some)
        const bool same = logit_before == logit && bias_before == bias;
        // (of equals the lowest came first; but behind the last chosen and its equal there may be a larger one yet, unless the values' lost
        // bits were zeros; and a smaller one with the same score in 64 bits, unless no other logit is that near: 16-bit ones are not, from 1e-6 on)
        bool near_other = false;
        if (TYPE != OZIMMU_F32 && !by_values && __builtin_amdgcn_ballot_w64(lane == a.top && same && fabsf(logit) <= 1e-6f)) {   // (the same for the wavefront)
            const float last = __shfl(logit, row0 + a.top);
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) near_other |= l[k] != last && fabsf(l[k] - last) < 2e-9f;
            near_other = (__builtin_amdgcn_ballot_w64(near_other) >> row0 & kMask) != 0;
        }
        const bool in_order = same && (lane < a.top || (TYPE != OZIMMU_F32 && !by_values && !near_other));
        if (lane > 0 && lane <= a.top && mine != 0xffffffffu) unsure |= !apart(v, w) && !in_order;
        // Scores that 64 bits do not tell apart: softmax has none so far below the largest; sigmoid's are 0 below -709.8, whatever the logit.
        if (mine != 0xffffffffu) all |= a.sigmoid ? !by_values && logit < -700.f : top_logit - logit > 600.f;
    }
    bad = (__builtin_amdgcn_ballot_w64(bad) >> row0 & kMask) != 0;
    const unsigned long long doubt = __builtin_amdgcn_ballot_w64(unsure && !bad);
    if (doubt) {   // (the same for the wavefront)
        // Where the one behind them is clearly less than the last chosen, the chosen are among these top + 1. Softmax with a bias or groups
        // needs the sum over all for their values.
        unsigned next_bits;
        sorted.next(lane, next_bits);
        const float last = Bits<float>::value((unsigned)__shfl((int)mine_bits, row0 + a.top - 1));
        const bool mine_doubt = (doubt >> row0 & kMask) != 0;
        all |= mine_doubt && ((!a.sigmoid && by_values) || (next_bits != 0 && !apart(last, Bits<float>::value(next_bits))));
        double d = -INFINITY;
        if (mine != 0xffffffffu) d = a.sigmoid ? 1.0 / (1.0 + exp(-(double)logit)) + (double)bias : (double)logit;
        int before = 0;
        for (int j = 0; j <= a.top; ++j) {
            const double other = __shfl(d, row0 + j);
            const unsigned expert = (unsigned)__shfl((int)mine, row0 + j);
            before += other > d || (other == d && expert < mine);
            all |= mine_doubt && !a.sigmoid && other != d && fabs(other - d) < 1e-9;
        }
        unsigned sure = 0xffffffffu;
        float of_sure = -INFINITY;
        for (int j = 0; j <= a.top; ++j) {
            const bool at = __shfl(mine != 0xffffffffu ? before : -1, row0 + j) == lane;
            const unsigned expert = (unsigned)__shfl((int)mine, row0 + j);
            const float value = __shfl(logit, row0 + j);
            sure = at ? expert : sure;
            of_sure = at ? value : of_sure;
        }
        if (mine_doubt) {
            mine = sure;
            logit = of_sure;
        }
    }
    const unsigned long long rest = __builtin_amdgcn_ballot_w64(all && !bad);
    if (rest) {
        double d[SLOTS], sum = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            d[k] = a.sigmoid ? 1.0 / (1.0 + exp(-(double)l[k])) : l[k] == -INFINITY ? 0.0 : exp((double)l[k] - (double)top_logit);
            sum += d[k];
        }
        sum = sum_of<LANES>(sum);
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if (!a.sigmoid) d[k] /= sum;
            if (a.bias) d[k] += (double)b[k];
            d[k] = l[k] == -INFINITY ? -INFINITY : d[k];
        }
        if (a.groups > 1) {
            double first, second;
            bool never = false;
            two_largest(d, first, second);
            const bool keep = in_best_groups<LANES>(a, lane, some, width, first, second, 0.f, never);
#pragma unroll
            for (int k = 0; k < SLOTS; ++k) d[k] = keep ? d[k] : -INFINITY;
        }
        const unsigned exact = choose_exactly<LANES, SLOTS>(a, lane, d);
        if (rest >> row0 & kMask) {
            mine = exact;
            logit = mine != 0xffffffffu ? Elem<TYPE>::load((static_cast<const raw*>(a.logits) + token * a.ldl)[mine]) : -INFINITY;
        }
    }
    // the weights from the chosen logits, in 64 bits
    const bool chosen = mine != 0xffffffffu && lane < a.top && !bad;
    double w;
    if (a.sigmoid) {
        w = chosen ? 1.0 / (1.0 + exp(-(double)logit)) : 0.0;
        if (a.renormalize) w /= sum_of<LANES>(w) + 1e-20;
    } else if (a.renormalize) {
        const float top = Bits<float>::value(most<LANES>(chosen ? Bits<float>::of(logit) : 0u));
        w = chosen ? exp((double)logit - (double)top) : 0.0;
        const double sum = sum_of<LANES>(w);
        w = sum > 0.0 ? w / sum : 0.0;
    } else {
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) sum += l[k] == -INFINITY ? 0.0 : exp((double)l[k] - (double)top_logit);
        sum = sum_of<LANES>(sum);
        w = chosen ? exp((double)logit - (double)top_logit) / sum : 0.0;
    }
    if (there && lane < a.top) {
        indices[token * a.top + lane] = chosen ? (int)mine : -1;
        weights[token * a.top + lane] = bad ? __builtin_nanf("") : chosen ? (float)(w * (double)a.scale) : 0.f;
    }
}

// The gradient where only the chosen scores have one: sigmoid, or renormalised softmax. Lane j computes choice j's; the row is zeros beside them.
// Bound: latency (indices, their logits, an exponential in 64 bits, the row). 16384 tokens of 256 experts, bf16, us: 6.7 (from all scores, as below, 25).
template <int TYPE, int LANES, int SLOTS>
__launch_bounds__(kThreads)
__global__ void route_grad_chosen_kernel(RouteArgs a, const int* indices, const float* dweights, void* dlogits, int64_t lddl) {
    typedef typename Elem<TYPE>::raw raw;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t token = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
    if (token >= a.t) return;      // (whole rows of lanes)
    int mine = lane < a.top ? indices[token * a.top + lane] : -1;
    if ((unsigned)mine >= (unsigned)a.experts) mine = -1;
    const double l = mine >= 0 ? (double)Elem<TYPE>::load((static_cast<const raw*>(a.logits) + token * a.ldl)[mine]) : -INFINITY;
    const double dw = mine >= 0 ? (double)dweights[token * a.top + lane] * (double)a.scale : 0.0;
    double d;
    if (a.sigmoid) {
        const double s = mine >= 0 ? 1.0 / (1.0 + exp(-l)) : 0.0;
        if (a.renormalize) {
            const double total = sum_of<LANES>(s) + 1e-20, w = s / total;      // (one choice: w is 1 and the gradient 0, not a rounding)
            d = (dw - sum_of<LANES>(dw * w)) / total * s * (1.0 - s);
        } else {
            d = dw * s * (1.0 - s);
        }
    } else {
        const float top = Bits<float>::value(most<LANES>(mine >= 0 ? Bits<float>::of((float)l) : 0u));
        const double x = mine >= 0 && l != -INFINITY ? exp(l - (double)top) : 0.0, sum = sum_of<LANES>(x), w = sum > 0.0 ? x / sum : 0.0;
        d = w * (dw - sum_of<LANES>(dw * w));
    }
    float g[SLOTS];
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) g[k] = 0.f;
    const float df = (float)d;
    for (int j = 0; j < a.top; ++j) {   // (an index that stands twice gets both)
        const int i = __shfl(mine, j, LANES);
        const float x = __shfl(df, j, LANES);
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) g[k] += i == lane * SLOTS + k ? x : 0.f;
    }
    raw* row = static_cast<raw*>(dlogits) + token * lddl + lane * SLOTS;
    raw r[SLOTS];
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) r[k] = Elem<TYPE>::store(g[k]);
    constexpr int words = SLOTS * (int)sizeof(raw) / 4;
    if (words > 0 && lane * SLOTS + SLOTS <= a.experts) {
        typedef unsigned many __attribute__((ext_vector_type(words > 4 ? 4 : words > 0 ? words : 1)));
        typedef many many_any __attribute__((aligned(2)));
#pragma unroll
        for (int w = 0; w < (words + 3) / 4; ++w) reinterpret_cast<many_any*>(row)[w] = reinterpret_cast<const many*>(r)[w];
    } else {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (lane * SLOTS + k < a.experts) row[k] = r[k];
    }
}

// That of softmax scores as they are: every logit has one, -s (sum of the chosen scores' gradients times the scores), and the chosen ones s dw beside it.
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
    double score = 0.0;
    for (int j = 0; j < a.top; ++j) {   // lane j's choice: its score
        const int i = __shfl(mine, j);
        if (i < 0) continue;
        double sc = 0.0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) sc = k == (i >> 6) ? s[k] : sc;
        sc = __shfl(sc, i & 63);
        score = lane == j ? sc : score;
    }
    const double d = dw * score, all = wave_sum(d);
    const bool any = __builtin_amdgcn_ballot_w64(mine >= 0) != 0;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) g[k] = any && all != 0.0 ? -s[k] * all : 0.0;
    for (int j = 0; j < a.top; ++j) {
        const int i = __shfl(mine, j);
        const double x = __shfl(d, j);
        if (i < 0) continue;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) g[k] += k * 64 + lane == i ? x : 0.0;
    }
    raw* row = static_cast<raw*>(dlogits) + token * lddl;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int e = k * 64 + lane;
        if (e < a.experts) row[e] = Elem<TYPE>::store((float)(bad && any ? (double)__builtin_nanf("") : l[k] == -INFINITY ? 0.0 : g[k]));
    }
}

template <class F>
hipError_t by_type(int type, F&& f) {
    if (type == OZIMMU_F32)
        f(std::integral_constant<int, OZIMMU_F32>{});
    else if (type == OZIMMU_BF16)
        f(std::integral_constant<int, OZIMMU_BF16>{});
    else
        f(std::integral_constant<int, OZIMMU_F16>{});
    return hipGetLastError();
}
// Slots of `lanes` lanes that hold the experts: a power of two.
int slots_of(int experts, int lanes) {
    int s = 1;
    while (s * lanes < experts) s *= 2;
    return s;
}
template <class F>
void by_slots(int slots, F&& f) {
    switch (slots) {
        case 1: f(std::integral_constant<int, 1>{}); break;
        case 2: f(std::integral_constant<int, 2>{}); break;
        case 4: f(std::integral_constant<int, 4>{}); break;
        case 8: f(std::integral_constant<int, 8>{}); break;
        default: f(std::integral_constant<int, 16>{}); break;
    }
}
// Groups that are whole lanes, a power of two of them.
bool groups_fit(const RouteArgs& a, int slots) {
    const int per = a.experts / a.groups;
    return a.groups == 1 || (per % slots == 0 && (per / slots & (per / slots - 1)) == 0);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, int* indices, float* weights, hipStream_t st) {
    const int few = slots_of(a.experts, 16), many = slots_of(a.experts, 64);
    return by_type(a.type, [&](auto kind) {
        constexpr int T = decltype(kind)::value;
        if (few <= 16 && a.top < 16 && groups_fit(a, few)) {
            by_slots(few, [&](auto slots) { route_kernel<T, 16, decltype(slots)::value><<<dim3((unsigned)((a.t + 15) / 16)), dim3(kThreads), 0, st>>>(a, indices, weights); });
        } else {
            by_slots(many, [&](auto slots) {
                constexpr int S = decltype(slots)::value;
                auto kernel = groups_fit(a, S) ? route_kernel<T, 64, S> : route_exactly_kernel<T, S>;
                kernel<<<dim3((unsigned)((a.t + 3) / 4)), dim3(kThreads), 0, st>>>(a, indices, weights);
            });
        }
    });
}

hipError_t launch_route_grad(const RouteArgs& a, const int* indices, const float* dweights, void* dlogits, int64_t lddl, hipStream_t st) {
    const int few = slots_of(a.experts, 16), many = slots_of(a.experts, 64);
    const bool chosen = a.sigmoid || a.renormalize;
    return by_type(a.type, [&](auto kind) {
        constexpr int T = decltype(kind)::value;
        if (chosen && few <= 16 && a.top <= 16) {
            by_slots(few, [&](auto slots) { route_grad_chosen_kernel<T, 16, decltype(slots)::value><<<dim3((unsigned)((a.t + 15) / 16)), dim3(kThreads), 0, st>>>(a, indices, dweights, dlogits, lddl); });
        } else {
            by_slots(many, [&](auto slots) {
                constexpr int S = decltype(slots)::value;
                auto kernel = chosen ? route_grad_chosen_kernel<T, 64, S> : route_grad_kernel<T, S>;
                kernel<<<dim3((unsigned)((a.t + 3) / 4)), dim3(kThreads), 0, st>>>(a, indices, dweights, dlogits, lddl);
            });
        }
    });
}

}  // namespace ozimmu
