// moe_scores.cuh -- selection of a token's experts by scores, with a bias and by groups (a part of moe_scored.cu).
//
//   s[e] = 1 / (1 + exp(-x[e])), or the softmax of the row;  c[e] = s[e] + bias[e]
//   a group's rank is its largest c, or the sum of its two largest; the best `top_groups` groups stay
//   the k largest c of these are taken;  weight = s (over the sum of the taken s, if asked for) times scale
//
// Without a bias the order of c is that of the logits, and no score is computed to find it.
//
// Who is taken is decided as in 64 bits: one rounding of 32 bits could exchange two experts, and a token would go elsewhere.  c is first computed
// in fp32, and its error is known: s has a relative error below 2^-22 (and in the softmax, where x - max is rounded, one of
// |x - max| 2^-24, which times exp(x - max) stays below 2^-25), so c is off by less than 2^-21 min(1, |c| + max|bias|) + 2^-23 |c| (+ 2^-24).
// Where two of those that are taken, or one and another that is not, lie closer than that, and are not equal logits with equal biases, the row
// is done again in 64 bits; of random logits and biases that is one row in some thousand.
//
// A warp takes a token, each lane PER consecutive experts.
#pragma once
#include <cstdint>

#include "divisor.cuh"
#include "moe_order.cuh"
#include "mx_kernels.h"

namespace ilw {
namespace {

__device__ __forceinline__ float none_of(float) { return __int_as_float(0xff800000); }
__device__ __forceinline__ double none_of(double) { return __longlong_as_double(0xfff0000000000000ll); }
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
// exp(x - best), where both may be infinite
template <typename V> __device__ __forceinline__ V exp_below(float x, float best) { return x == best ? V(1) : exp_of(V(x) - V(best)); }
// 1 / (1 + exp(-x)).  fp32: by the exponential that cannot overflow, for scores below its normal range.  64 bits, which only compare: as it is
// written, so that sums that are equal but for roundings (of the scores of x and -x) fall as plain operations let them.
template <typename V> __device__ __forceinline__ V sigmoid(float x);
template <> __device__ __forceinline__ float sigmoid<float>(float x) {
    const float e = expf(-fabsf(x));
    return (x >= 0.0f ? 1.0f : e) / (1.0f + e);
}
template <> __device__ __forceinline__ double sigmoid<double>(float x) { return 1.0 / (1.0 + exp(-(double)x)); }

// Values as unsigned numbers of the same order, 0 for -inf and NaN: their largest in a warp, by whole-word reductions.
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // (-0 is 0)
    return v > none_of(v) ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ uint64_t order_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
    return v > none_of(v) ? (b >> 63 ? ~b : b | 1ull << 63) : 0ull;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float key_value(uint64_t) { return 0.0f; }  // (not asked for)
template <typename V> struct Key { typedef uint32_t type; };
template <> struct Key<double> { typedef uint64_t type; };

// How far c may be off (see above).
__device__ __forceinline__ float doubt(const RouteScores &q, float c, float bias_max) {
    const float a = fabsf(c);
    return fminf(1.0f, a + bias_max) * 4.76837158e-07f + a * 1.1920929e-07f + (q.score == ILW_SCORE_SOFTMAX ? 5.96046448e-08f : 0.0f);
}

// The two largest of (a1, a2) and (b1, b2), each pair in order.
template <typename V> __device__ __forceinline__ void merge2(V &a1, V &a2, V b1, V b2) {
    const V low = a1 < b1 ? a1 : b1;
    a2 = a2 > b2 ? a2 : b2;
    a2 = a2 > low ? a2 : low;
    a1 = a1 > b1 ? a1 : b1;
}

// The experts of a token, the j-th in lane j's `mine` (-1: none); false if fp32 cannot tell (V double: never).  x: this lane's logits, -inf where
// no expert is to be taken; `best` their row's largest; `sum` their softmax's denominator.
template <typename V, int PER>
__device__ __forceinline__ bool choose(const MoeScoredParams &p, const float (&x)[PER], float best, V sum, float bias_max, int lane, int32_t &mine) {
    constexpr bool kCheck = sizeof(V) == 4;
    const RouteScores &q = p.scores;
    const V none = none_of(V());
    const int e0 = lane * PER;
    V c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = V(x[i]);
        if (q.bias) {
            const V s = q.score == ILW_SCORE_SIGMOID ? sigmoid<V>(x[i]) : exp_below<V>(x[i], best) / sum;
            const V v = s + V(e0 + i < p.E ? __ldg(q.bias + e0 + i) : 0.0f);
            c[i] = x[i] > none_of(0.0f) && v > none ? v : none;
        }
    }
    uint32_t groups = 0xffffffffu;  // those that stay
    bool sure = true;
    if (q.groups > 1) {
        V t1 = none, t2 = none;  // the two largest of group `lane`
        if (q.lanes_per_group) {  // a lane's experts are of one group, whose lanes are a power of two
#pragma unroll
            for (int i = 0; i < PER; ++i) merge2(t1, t2, c[i], none);
            for (int d = 1; d < q.lanes_per_group; d <<= 1) merge2(t1, t2, __shfl_xor_sync(0xffffffffu, t1, d), __shfl_xor_sync(0xffffffffu, t2, d));
            t1 = __shfl_sync(0xffffffffu, t1, lane * q.lanes_per_group);
            t2 = __shfl_sync(0xffffffffu, t2, lane * q.lanes_per_group);
        } else {
            for (int g = 0; g < q.groups; ++g) {
                V a1 = none, a2 = none;
                const int lo = g * q.group_size - e0;
#pragma unroll
                for (int i = 0; i < PER; ++i) merge2(a1, a2, i >= lo && i < lo + q.group_size ? c[i] : none, none);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) merge2(a1, a2, __shfl_xor_sync(0xffffffffu, a1, d), __shfl_xor_sync(0xffffffffu, a2, d));
                if (lane == g) t1 = a1, t2 = a2;
            }
        }
        V rank = t1;
        if (q.group_best == 2) {  // (of logits: their scores' sum, the softmax's without its denominator)
            if (!q.bias) {
                const bool sig = q.score == ILW_SCORE_SIGMOID;
                rank = t1 > none ? (sig ? sigmoid<V>((float)t1) : exp_below<V>((float)t1, best)) + (t2 > none ? (sig ? sigmoid<V>((float)t2) : exp_below<V>((float)t2, best)) : V(0))
                                 : none;
            } else if (t2 > none) {
                rank = t1 + t2;
            }
        }
        if (lane >= q.groups) rank = none;
        int place = 0;  // of this lane's group among all
        for (int g = 0; g < q.groups; ++g) {
            const V other = __shfl_sync(0xffffffffu, rank, g);
            place += other > rank || (other == rank && g < lane);
        }
        groups = __ballot_sync(0xffffffffu, lane < q.groups && place < q.top_groups && rank > none);
        if (kCheck && (q.bias || q.group_best == 2)) {
            // the last group that stays and the first that does not; who lies close to the other side's, and is not its equal, is in doubt
            const uint32_t last = __ballot_sync(0xffffffffu, lane < q.groups && place == q.top_groups - 1 && rank > none);
            const uint32_t next = __ballot_sync(0xffffffffu, lane < q.groups && place == q.top_groups && rank > none);
            if (last && next) {
                const bool stays = groups >> lane & 1;
                const int of = __ffs(stays ? next : last) - 1;
                // (a rank without a bias: one or two scores of a relative error, the softmax's without their denominator)
                const float off = q.bias ? doubt(q, (float)t1, bias_max) + (q.group_best == 2 && t2 > none ? doubt(q, (float)t2, bias_max) : 0.0f) + fabsf((float)rank) * 1.1920929e-07f
                                         : (float)rank * 4.76837158e-07f + (q.score == ILW_SCORE_SOFTMAX ? 1.1920929e-07f : 0.0f);
                const V other = __shfl_sync(0xffffffffu, rank, of), o1 = __shfl_sync(0xffffffffu, t1, of), o2 = __shfl_sync(0xffffffffu, t2, of);
                const float other_off = __shfl_sync(0xffffffffu, off, of);
                const bool close = rank > none && fabsf((float)(rank - other)) <= 2.0f * (off + other_off);
                if (__any_sync(0xffffffffu, close && !(!q.bias && t1 == o1 && (t2 == o2 || q.group_best == 1)))) sure = false;
            }
        }
    }
    typename Key<V>::type key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = (q.groups == 1 || (groups >> min(q.per_group.div(e0 + i), 31u) & 1)) && e0 + i < p.E ? order_key(c[i]) : 0;
    mine = -1;
    float last = 0.0f, last_x = 0.0f, last_b = 0.0f;  // c, logit and bias of the one taken before
    for (int j = 0; j < p.k; ++j) {
        typename Key<V>::type m = key[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < PER; ++i)
            if (key[i] > m) m = key[i], at = i;
        const typename Key<V>::type top = warp_max(m);
        if (top == 0) return sure;
        const int src = __ffs(__ballot_sync(0xffffffffu, m == top)) - 1;
        const int32_t e = __shfl_sync(0xffffffffu, e0 + at, src);
        if constexpr (kCheck) {
            if (q.bias) {
                float xe = 0.0f;
#pragma unroll
                for (int i = 0; i < PER; ++i) xe = i == at ? x[i] : xe;
                xe = __shfl_sync(0xffffffffu, xe, src);
                const float v = key_value(top), be = __ldg(q.bias + e);
                if (j > 0 && last - v <= doubt(q, last, bias_max) + doubt(q, v, bias_max) && !(xe == last_x && be == last_b)) sure = false;
                last = v, last_x = xe, last_b = be;
            }
        }
        if (lane == j) mine = e;
        if (lane == src) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i == at) key[i] = 0;
        }
    }
    if constexpr (kCheck) {
        if (q.bias) {  // is the last one taken clear of all that are left
            bool close = false;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (key[i] != 0) {
                    const float v = key_value(key[i]);
                    close |= last - v <= doubt(q, last, bias_max) + doubt(q, v, bias_max) && !(x[i] == last_x && __ldg(q.bias + e0 + i) == last_b);
                }
            if (__any_sync(0xffffffffu, close)) sure = false;
        }
    }
    return sure;
}

// The same in 64 bits, from the logits on.
template <int PER>
__device__ __noinline__ int32_t choose_exactly(const MoeScoredParams &p, const float *xs, float best, int lane) {
    float x[PER];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        x[i] = xs[i];
        if (p.scores.score == ILW_SCORE_SOFTMAX && x[i] > none_of(0.0f)) sum += exp_below<double>(x[i], best);
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    int32_t mine;
    choose<double, PER>(p, x, best, sum, 0.0f, lane, mine);
    return mine;
}

// Lane j: the weight of expert `e`, the j-th taken (-1: 0), whose logit is x.
__device__ __forceinline__ float weight_of(const MoeScoredParams &p, int32_t e, float x, float best, float sum) {
    const bool on = e >= 0;
    float s = 0.0f;
    if (p.scores.score == ILW_SCORE_SOFTMAX) {
        if (on) s = exp_below<float>(x, best);
        if (p.renormalize) {
            sum = s;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        }
    } else if (p.renormalize) {
        // exp(min(x, 0)) / (1 + exp(-|x|)), all times exp(-m) for the largest m of min(x, 0): scores too small for fp32 keep their ratios
        const float low = on ? fminf(x, 0.0f) : none_of(0.0f);
        float m = low;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (on) s = exp_below<float>(low, m) / (1.0f + expf(-fabsf(x)));
        sum = s;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    } else {
        if (on) s = sigmoid<float>(x);
        sum = 1.0f;
    }
    return on ? s / sum * p.scores.scale : 0.0f;
}

// Token t by one warp: lane j < k gets its j-th expert and weight.
template <typename T, int PER>
__device__ __forceinline__ void select_scored(const MoeScoredParams &p, int64_t t, bool wide, float bias_max, int lane, int32_t &expert, float &weight) {
    const T *row = (const T *)p.logits + t * p.ld;
    const float none = none_of(0.0f);
    const int e0 = lane * PER;
    float x[PER];
    constexpr int V = PER * sizeof(T) <= 16 ? PER : 16 / (int)sizeof(T);
    struct alignas(V * sizeof(T)) Pack {
        T v[V];
    };
    if (wide) {
#pragma unroll
        for (int i = 0; i < PER; i += V) {
            Pack y;
            if (e0 + i < p.E) y = *(const Pack *)(row + e0 + i);
#pragma unroll
            for (int j = 0; j < V; ++j) x[i + j] = e0 + i < p.E ? logit(to_f(y.v[j])) : none;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = e0 + i < p.E ? logit(to_f(row[e0 + i])) : none;
    }
    float best = x[0], sum = 1.0f;
#pragma unroll
    for (int i = 1; i < PER; ++i) best = fmaxf(best, x[i]);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
    if (p.scores.score == ILW_SCORE_SOFTMAX && (p.scores.bias || !p.renormalize)) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (x[i] > none) sum += exp_below<float>(x[i], best);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    if (!choose<float, PER>(p, x, best, sum, bias_max, lane, expert)) expert = choose_exactly<PER>(p, x, best, lane);
    weight = weight_of(p, expert, expert >= 0 ? to_f(row[expert]) : 0.0f, best, sum);
}

}  // namespace
}  // namespace ilw
