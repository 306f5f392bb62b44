// moe_scores.cuh -- selection of a token's experts by scores, with a bias and by groups (a part of moe_scored.cuh).
//
//   s[e] = 1 / (1 + exp(-x[e])), or the softmax of the row;  c[e] = s[e] + bias[e]
//   a group's rank is its largest c, or the sum of its two largest; the best `top_groups` groups stay
//   the k largest c of these are taken;  weight = s (over the sum of the taken s, if asked for) times scale
//
// Without a bias the order of c is that of the logits, and no score is computed to find it.
//
// Who is taken is decided as in 64 bits: one rounding of 32 bits could exchange two experts, and a token would go elsewhere.  c is first computed
// in fp32 with the fast exponential and reciprocal, and its error is bounded: of s by a relative 2^-21.5 (2^-22.5 and 2^-23 of the two
// functions, roundings), a softmax's denominator by 23 roundings more (chains of 17 sums, exponentials), so 2^-19 in all; for the two roundings of
// an exponent y = x or x - max, |y| 2^-23 relative to exp(-|y|), which stays below 2^-24; of the sum with the bias by 2^-24 |c|.  So c is off by
// less than doubt() = u min(1, |c| + max|bias|) + 2^-23 |c| + 2^-24, with u 2^-21 for the sigmoid and 2^-19 for the softmax.
// Where two of those that are taken, or one and another that is not, lie closer than their doubts, and are not equal logits with equal biases,
// they are ordered again in 64 bits by the whole warp (one row in some hundred of random logits and biases), and so are groups that lie that close.
// 64-bit operations have some 1/60 of the rate of fp32 here, and one row that is done again holds up its warp, so it is those few values and not the row
// (2084 tokens of 112 experts, softmax, 7 of 16 groups: 30 us with whole rows, so 23).
#pragma once
#include <cstdint>

#include "divisor.cuh"
#include "moe_order.cuh"
#include "mx_kernels.h"

namespace ilw {
namespace {

// Words of a token's ranks (an odd number, so that tokens meet in no bank).
__host__ __device__ inline int rank_words(const RouteScores &q) { return q.groups > 1 ? 2 * q.groups | 1 : 0; }

constexpr float kNone = -__builtin_huge_valf();

// ---- the exact way: a warp a token, each lane PER consecutive experts, in 64 bits

__device__ __forceinline__ double none64() { return __longlong_as_double(0xfff0000000000000ll); }
// exp(x - best), where both may be infinite
__device__ __forceinline__ float exp_below(float x, float best) { return x == best ? 1.0f : expf(x - best); }
// (Out of line, like all that 64 bits take: where few tokens take this way, fetching its instructions is most of it.)
__device__ __noinline__ double exp64(double x) { return exp(x); }
__device__ __forceinline__ double exp_below64(float x, float best) { return x == best ? 1.0 : exp64((double)x - (double)best); }
// 1 / (1 + exp(-x)).  fp32: by the exponential that cannot overflow, for scores below its normal range.  64 bits, which only compare: as it is
// written, so that sums that are equal but for roundings (of the scores of x and -x) fall as plain operations let them.
__device__ __forceinline__ float sigmoid(float x) {
    const float e = expf(-fabsf(x));
    return (x >= 0.0f ? 1.0f : e) / (1.0f + e);
}

// A value as an unsigned number of the same order, 0 for -inf and NaN; the largest in a warp.
__device__ __forceinline__ uint64_t order_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);  // (-0 is 0)
    return v > none64() ? (b >> 63 ? ~b : b | 1ull << 63) : 0ull;
}
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ double key_value(uint64_t k) { return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k)); }

// Scores of a row in 64 bits: of its logit x, given the row's largest and, for the softmax, its denominator.
struct Exact {
    int32_t score;
    float best;
    double sum;
    __device__ __forceinline__ double operator()(float x) const {
        const bool sigmoid = score == ILW_SCORE_SIGMOID;
        const double e = !sigmoid && x == best ? 1.0 : exp64(sigmoid ? -(double)x : (double)x - (double)best);
        return (sigmoid ? 1.0 : e) / (sigmoid ? 1.0 + e : sum);
    }
};
template <typename T> __device__ __forceinline__ Exact exact_scores(const MoeScoredParams &p, const T *row, int lane) {
    Exact s = {p.scores.score, kNone, 0.0};
    if (s.score == ILW_SCORE_SIGMOID) return s;
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) s.best = fmaxf(s.best, logit(to_f(row[e])));
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) s.best = fmaxf(s.best, __shfl_xor_sync(0xffffffffu, s.best, d));
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) {
        const float x = logit(to_f(row[e]));
        if (x > kNone) s.sum += exp_below64(x, s.best);
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) s.sum += __shfl_xor_sync(0xffffffffu, s.sum, d);
    return s;
}

// The experts of a token with biases, the j-th in lane j (-1: none): all of it in 64 bits, each lane PER consecutive experts.  (Comparisons are of keys: those of
// 64-bit numbers would be the slower part.)
template <typename T, int PER>
__device__ __noinline__ int32_t choose_exactly(const MoeScoredParams &p, const T *row, int lane) {
    const RouteScores &q = p.scores;
    const int e0 = lane * PER;
    const Exact score = exact_scores(p, row, lane);
    uint64_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float x = e0 + i < p.E ? logit(to_f(row[e0 + i])) : kNone;
        key[i] = x > kNone ? order_key(score(x) + (double)__ldg(q.bias + e0 + i)) : 0;
    }
    if (q.groups > 1) {
        uint64_t mine1 = 0, mine2 = 0;  // the two largest of group `lane`
        for (int g = 0; g < q.groups; ++g) {
            uint64_t m1 = 0, m2 = 0;  // this lane's two largest of the group
            const int lo = g * q.group_size - e0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i >= lo && i < lo + q.group_size) {
                    m2 = max(m2, min(m1, key[i]));
                    m1 = max(m1, key[i]);
                }
            const uint64_t t1 = warp_max(m1);
            const int holder = __ffs(__ballot_sync(0xffffffffu, m1 == t1)) - 1;
            const uint64_t t2 = warp_max(lane == holder ? m2 : m1);
            if (lane == g) mine1 = t1, mine2 = t2;
        }
        uint64_t rank = mine1;
        if (q.group_best == 2 && mine2) rank = order_key(key_value(mine1) + key_value(mine2));
        int place = 0;  // of this lane's group among all
        for (int g = 0; g < q.groups; ++g) {
            const uint64_t other = __shfl_sync(0xffffffffu, rank, g);
            place += other > rank || (other == rank && g < lane);
        }
        const uint32_t stay = __ballot_sync(0xffffffffu, lane < q.groups && place < q.top_groups && rank);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e0 + i < p.E && !(stay >> q.per_group.div(e0 + i) & 1)) key[i] = 0;
    }
    int32_t mine = -1;
    for (int j = 0; j < p.k; ++j) {
        uint64_t m = key[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < PER; ++i)
            if (key[i] > m) m = key[i], at = i;
        const uint64_t top = warp_max(m);
        if (top == 0) break;
        const int src = __ffs(__ballot_sync(0xffffffffu, m == top)) - 1;
        const int32_t e = __shfl_sync(0xffffffffu, e0 + at, src);
        if (lane == j) mine = e;
        if (lane == src) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i == at) key[i] = 0;
        }
    }
    return mine;
}

// The same where only the order of those taken, and of some that were left, is in doubt: lane l has candidate `e` (-1: none), and the first
// p.k places of them all go to out_e.
template <typename T>
__device__ __noinline__ void order_exactly(const MoeScoredParams &p, const T *row, int32_t e, int candidates, int32_t *out_e, int lane) {
    const Exact score = exact_scores(p, row, lane);
    const uint64_t key = e >= 0 ? order_key(score(to_f(row[e])) + (double)__ldg(p.scores.bias + e)) : 0;
    int place = 0;
    for (int l = 0; l < candidates; ++l) {
        const uint64_t other = __shfl_sync(0xffffffffu, key, l);
        const int32_t o = __shfl_sync(0xffffffffu, e, l);
        place += other > key || (other == key && o < e);
    }
    if (e >= 0 && place < p.k) out_e[place] = e;
}

// The groups of a token that stay, where fp32 cannot tell: `stay` by their ranks in fp32, of which the `doubtful` may have gone to the wrong side.  Those
// clear of all of the other side keep theirs; the doubtful ranks are computed in 64 bits, and as many of them stay as did.
template <typename T>
__device__ __noinline__ uint32_t groups_exactly(const MoeScoredParams &p, const T *row, uint32_t stay, uint32_t doubtful, int lane) {
    const RouteScores &q = p.scores;
    const Exact score = exact_scores(p, row, lane);
    uint64_t rank = 0;  // of group `lane`
    for (uint32_t left = doubtful; left; left &= left - 1) {
        const int g = __ffs(left) - 1;
        uint64_t m1 = 0, m2 = 0;  // this lane's two largest of the group
#pragma unroll 1
        for (int i = lane; i < q.group_size; i += 32) {
            const int e = g * q.group_size + i;
            const float x = logit(to_f(row[e]));
            const uint64_t key = x > kNone ? order_key(score(x) + (q.bias ? (double)__ldg(q.bias + e) : 0.0)) : 0;
            m2 = max(m2, min(m1, key));
            m1 = max(m1, key);
        }
        const uint64_t t1 = warp_max(m1);
        const int holder = __ffs(__ballot_sync(0xffffffffu, m1 == t1)) - 1;
        const uint64_t t2 = warp_max(lane == holder ? m2 : m1);
        if (lane == g) rank = q.group_best == 2 && t2 ? order_key(key_value(t1) + key_value(t2)) : t1;
    }
    int place = 0;  // of this lane's group among the doubtful
    for (uint32_t left = doubtful; left; left &= left - 1) {
        const int g = __ffs(left) - 1;
        const uint64_t other = __shfl_sync(0xffffffffu, rank, g);
        place += other > rank || (other == rank && g < lane);
    }
    const uint32_t in = __ballot_sync(0xffffffffu, rank && place < __popc(stay & doubtful));
    return (stay & ~doubtful) | (in & doubtful);
}

// ---- the fast way: L lanes a token, its row in shared memory, its experts in 16 search groups as in moe.cu

__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// How far c may be off (see above).
struct Doubt {
    float unit, bias_max;
    __device__ __forceinline__ Doubt(int32_t score, float bias_max) : unit(score == ILW_SCORE_SIGMOID ? 4.76837158e-07f : 1.90734863e-06f), bias_max(bias_max) {}
    __device__ __forceinline__ float operator()(float c) const { return fmaf(fminf(1.0f, fabsf(c) + bias_max), unit, fmaf(fabsf(c), 1.1920929e-07f, 5.96046448e-08f)); }
};

// The lower end of a rank that may be off by `off` (anywhere, where both are infinite).
__device__ __forceinline__ float low_end(float rank, float off) {
    const float end = rank - off;
    return end > kNone ? end : kNone;
}

// The two largest of n values from `at` on (16-byte aligned if n is a multiple of four).
__device__ __forceinline__ void top2(const float *at, int n, float &t1, float &t2) {
    t1 = t2 = kNone;
    auto take = [&](float v) {
        t2 = fmaxf(t2, fminf(t1, v));
        t1 = fmaxf(t1, v);
    };
    if (n % 4 == 0) {
        for (int i = 0; i < n; i += 4) {
            const float4 v = *(const float4 *)(at + i);
            take(v.x), take(v.y), take(v.z), take(v.w);
        }
    } else {
        for (int i = 0; i < n; ++i) take(at[i]);
    }
}
template <int L> __device__ __forceinline__ float max_of_lanes(float v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
template <int L> __device__ __forceinline__ float min_of_lanes(float v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v = fminf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
template <int L> __device__ __forceinline__ float sum_of_lanes(float v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
template <int L> __device__ __forceinline__ uint32_t any_of_lanes(uint32_t v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v |= __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// The experts of a token by L lanes (lane q of them here; all 32 lanes of the warp call it) to out_e, in order; not 0 if fp32 cannot tell that
// order.  `row` holds its logits and is lost, but for the c of those left; `logits` are its row in memory; `bias` [E] and its largest magnitude; ranks [2 groups]: room.
// best and sum: largest logit, and the softmax's denominator if that is needed.  least: the smallest c taken.
template <typename T, int L, int S>
__device__ __forceinline__ uint32_t select_scored(const MoeScoredParams &p, const T *logits, const float *bias, float bias_max, float *row, float *ranks, int q,
                                              int32_t *out_e, float *out_w, float &best, float &sum, float &least) {
    constexpr int G = kGroups / L;  // this lane's search groups: q, L + q, ...
    const RouteScores &r = p.scores;
    const Doubt doubt(r.score, bias_max);
    const bool softmax = r.score == ILW_SCORE_SOFTMAX;
    best = kNone, sum = 1.0f;
    if (softmax) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const float4 *x = (const float4 *)(row + (L * i + q) * S);
#pragma unroll
            for (int c = 0; c < S / 4; ++c) best = fmaxf(fmaxf(fmaxf(best, x[c].x), fmaxf(x[c].y, x[c].z)), x[c].w);
        }
        best = max_of_lanes<L>(best);
        if (bias || !p.renormalize) {  // by group and in four parts: short chains of roundings
            float4 part = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
            for (int i = 0; i < G; ++i) {
                const float4 *x = (const float4 *)(row + (L * i + q) * S);
                float4 of = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int c = 0; c < S / 4; ++c) {
                    const float4 v = x[c];
                    of.x += v.x > kNone ? exp_below(v.x, best) : 0.0f, of.y += v.y > kNone ? exp_below(v.y, best) : 0.0f;
                    of.z += v.z > kNone ? exp_below(v.z, best) : 0.0f, of.w += v.w > kNone ? exp_below(v.w, best) : 0.0f;
                }
                part.x += of.x, part.y += of.y, part.z += of.z, part.w += of.w;
            }
            sum = sum_of_lanes<L>((part.x + part.y) + (part.z + part.w));
        }
    }
    const float over_sum = fast_rcp(sum), log2e = 1.44269504f;
    auto score = [&](float x) {
        if (softmax) return x == best ? over_sum : fast_exp2((x - best) * log2e) * over_sum;
        return fast_rcp(1.0f + fast_exp2(x * -log2e));
    };
    if (bias) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            float4 *x = (float4 *)(row + (L * i + q) * S);
            const float4 *b = (const float4 *)(bias + (L * i + q) * S);
#pragma unroll
            for (int c = 0; c < S / 4; ++c) {
                float4 v = x[c];
                const float4 w = b[c];
                auto add = [&](float y, float z) {
                    const float u = score(y) + z;
                    return y > kNone && u > kNone ? u : kNone;
                };
                x[c] = make_float4(add(v.x, w.x), add(v.y, w.y), add(v.z, w.z), add(v.w, w.w));
            }
        }
        __syncwarp();
    }
    if (r.groups > 1) {
        float *offs = ranks + r.groups;  // how far each rank may be off
        for (int g = q; g < r.groups; g += L) {
            float t1, t2, off = 0.0f;
            top2(row + g * r.group_size, r.group_size, t1, t2);
            float rank = t1;
            if (r.group_best == 2 && t1 > kNone) {
                if (!bias) {  // (of logits: the sum of their scores, the softmax's without its denominator)
                    rank = score(t1) + (t2 > kNone ? score(t2) : 0.0f);
                    off = fmaf(rank, 6.7434957e-07f, 1.1920929e-07f);
                } else if (t2 > kNone) {
                    rank = t1 + t2;
                }
            }
            if (bias) off = doubt(t1) + (r.group_best == 2 && t2 > kNone ? doubt(t2) : 0.0f) + fabsf(rank) * 1.1920929e-07f;
            // (a sum past fp32's largest number may be any such, and a group of them is still one)
            ranks[g] = t1 > kNone ? fmaxf(rank, -3.40282347e+38f) : kNone, offs[g] = off;
        }
        __syncwarp();
        uint32_t stay = 0;
        // who stays, and the intervals that ranks lie in: the least end of those that stay, the greatest of the others
        const bool inexact = bias || r.group_best == 2;  // (one logit without a bias is exact)
        float least_in = __int_as_float(0x7f800000), most_out = kNone;
        for (int g = q; g < r.groups; g += L) {
            const float mine = ranks[g], off = 2.0f * offs[g];
            int place = 0;
            for (int o = 0; o < r.groups; ++o) {
                const float other = ranks[o];
                place += other > mine || (other == mine && o < g);
            }
            if (mine > kNone) {
                if (place < r.top_groups) stay |= 1u << g, least_in = fminf(least_in, low_end(mine, off));
                else most_out = fmaxf(most_out, mine + off);
            }
        }
        stay = any_of_lanes<L>(stay);
        least_in = min_of_lanes<L>(least_in), most_out = max_of_lanes<L>(most_out);
        uint32_t doubtful = 0;  // groups whose interval meets one of the other side
        if (inexact && least_in <= most_out)
            for (int g = q; g < r.groups; g += L) {
                const float mine = ranks[g], off = 2.0f * offs[g];
                if (mine > kNone && (stay >> g & 1 ? low_end(mine, off) <= most_out : mine + off >= least_in)) doubtful |= 1u << g;
            }
        doubtful = any_of_lanes<L>(doubtful);
        bool close = doubtful && bias;
        if (doubtful && !bias) {  // of the same logits they are equal, and the first of them stay
            float a1, a2, b1, b2;
            top2(row + (__ffs(doubtful) - 1) * r.group_size, r.group_size, a1, a2);
            for (int g = q; g < r.groups; g += L)
                if (doubtful >> g & 1) {
                    top2(row + g * r.group_size, r.group_size, b1, b2);
                    if (a1 != b1 || a2 != b2) close = true;
                }
        }
        for (uint32_t again = __ballot_sync(0xffffffffu, any_of_lanes<L>(close) && q == 0); again; again &= again - 1) {
            const int l = __ffs(again) - 1, lane = threadIdx.x & 31;
            const T *x = (const T *)__shfl_sync(0xffffffffu, (unsigned long long)logits, l);
            const uint32_t exact = groups_exactly<T>(p, x, __shfl_sync(0xffffffffu, stay, l), __shfl_sync(0xffffffffu, doubtful, l), lane);
            if (l / L == lane / L) stay = exact;  // (a token of this warp's)
        }
        __syncwarp();
        for (int g = q; g < r.groups; g += L)
            if (!(stay >> g & 1)) {
                float *at = row + g * r.group_size;
                if (r.group_size % 4 == 0)
                    for (int i = 0; i < r.group_size; i += 4) *(float4 *)(at + i) = make_float4(kNone, kNone, kNone, kNone);
                else
                    for (int i = 0; i < r.group_size; ++i) at[i] = kNone;
            }
        __syncwarp();
    }
    float top[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
        const float4 *x = (const float4 *)(row + (L * i + q) * S);
        float m = kNone;
#pragma unroll
        for (int c = 0; c < S / 4; ++c) m = fmaxf(fmaxf(fmaxf(m, x[c].x), fmaxf(x[c].y, x[c].z)), x[c].w);
        top[i] = m;
    }
    // the same logit and the same bias
    auto equal = [&](int a, int b) { return to_f(logits[a]) == to_f(logits[b]) && bias[a] == bias[b]; };
    float before = __int_as_float(0x7f800000);
    int taken = 0;
    uint32_t unsure = 0;
    bool close = false;  // the last two taken
    for (int j = 0; j < p.k; ++j) {
        // the largest search group, the first of equal ones
        float m = top[0];
        int g = 0;
#pragma unroll
        for (int i = 1; i < G; ++i)
            if (top[i] > m) m = top[i], g = i;
        g = L * g + q;
#pragma unroll
        for (int d = 1; d < L; d <<= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
            const int g2 = __shfl_xor_sync(0xffffffffu, g, d);
            if (m2 > m || (m2 == m && g2 < g)) m = m2, g = g2;
        }
        if (close && !equal(out_e[j - 2], out_e[j - 1])) unsure = 1;
        const bool on = m > kNone;
        if (on && g % L == q) {  // its lane takes the first expert with that value
            const float4 *x = (const float4 *)(row + g * S);
            int at = S;
            float rest = kNone;
#pragma unroll
            for (int c = 0; c < S / 4; ++c) {
                const float4 v = x[c];
                const float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool hit = u[w] == m && at == S;
                    at = hit ? 4 * c + w : at;
                    rest = fmaxf(rest, hit ? kNone : u[w]);
                }
            }
            row[g * S + min(at, S - 1)] = kNone;
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (i == g / L) top[i] = rest;
            out_e[j] = g * S + at;
            out_w[j] = m;  // (without a bias the logit)
        }
        if (!on && q == 0) out_e[j] = -1;
        close = bias && on && j > 0 && before - m <= doubt(before) + doubt(m);
        if (on) before = m, taken = j + 1;
        __syncwarp();
    }
    if (bias) {
        if (close && !equal(out_e[p.k - 2], out_e[p.k - 1])) unsure = 1;
        // is the last one taken clear of all that are left
        float m = top[0];
#pragma unroll
        for (int i = 1; i < G; ++i) m = fmaxf(m, top[i]);
        const float off = doubt(before);
        if (taken == p.k && m > kNone && before - m <= off + doubt(m)) {
            const int e = out_e[p.k - 1];
            for (int i = 0; i < G; ++i)
                for (int c = 0; c < S; ++c) {
                    const float v = row[(L * i + q) * S + c];
                    if (v > kNone && before - v <= off + doubt(v) && !equal((L * i + q) * S + c, e)) unsure = 1;
                }
        }
    }
    least = taken == p.k ? before : __int_as_float(0x7f800000);
    return any_of_lanes<L>(unsure);
}

// The weights of a token's experts to out_w, by its L lanes, an expert each in turn.
template <typename T, int L>
__device__ __forceinline__ void weigh_scored(const MoeScoredParams &p, const T *logits, int q, const int32_t *out_e, float *out_w, float best, float sum, bool biased) {
    const bool softmax = p.scores.score == ILW_SCORE_SOFTMAX;
    // renormalised: exp(x), of sigmoids exp(min(x, 0)) / (1 + exp(-|x|)), all times exp(-m) for the largest m of those x or min(x, 0) that are taken,
    // so that scores too small for fp32 keep their ratios (a bias may leave a softmax's largest logits untaken)
    const bool ratios = p.renormalize;
    float m = kNone;
    for (int j = q; j < p.k; j += L)
        if (out_e[j] >= 0) {
            const float x = biased ? to_f(logits[out_e[j]]) : out_w[j];
            out_w[j] = x;
            m = fmaxf(m, softmax ? x : fminf(x, 0.0f));
        }
    m = ratios ? max_of_lanes<L>(m) : best;
    float of = 0.0f;
    for (int j = q < p.k ? q + (p.k - 1 - q) / L * L : -1; j >= q; j -= L) {  // (the small ones first)
        const float x = out_w[j];
        float s = 0.0f;
        if (out_e[j] >= 0) s = softmax ? exp_below(x, m) : ratios ? exp_below(fminf(x, 0.0f), m) / (1.0f + expf(-fabsf(x))) : sigmoid(x);
        out_w[j] = s;
        of += s;
    }
    if (p.renormalize) sum = sum_of_lanes<L>(of);
    for (int j = q; j < p.k; j += L) out_w[j] = out_e[j] >= 0 ? out_w[j] / sum * p.scores.scale : 0.0f;
}

// A warp's tokens, L lanes each, the first of them token t0 of the call: this lane's token's experts and weights to out_e and out_w.
template <typename T, int L, int S>
__device__ __forceinline__ void route_tokens(const MoeScoredParams &p, int64_t t0, bool is_token, const float *bias, float bias_max, float *row, float *ranks,
                                             int32_t *out_e, int entries, float *out_w) {
    const int lane = threadIdx.x & 31, q = lane % L;
    const T *logits = (const T *)p.logits + (t0 + (is_token ? lane / L : 0)) * p.ld;
    float best, sum, least;
    const uint32_t unsure = select_scored<T, L, S>(p, logits, bias, bias_max, row, ranks, q, out_e, out_w, best, sum, least);
    const Doubt doubt(p.scores.score, bias_max);
    uint32_t again = __ballot_sync(0xffffffffu, unsure && is_token && q == 0);
    while (again) {
        const int l = __ffs(again) - 1, t = l / L;  // a token of this warp's
        again &= again - 1;
        int32_t *to = out_e + (t - lane / L) * entries;
        float *its = row + (t - lane / L) * (kGroups * S + 4);
        const T *x = (const T *)p.logits + (t0 + t) * p.ld;
        const float low = __shfl_sync(0xffffffffu, least, l);
        // candidates: those taken, and those left whose c comes close to the least of them
        int32_t hits = 0;
        uint32_t which = 0;
        for (int i = 0; i < S / 2; ++i) {
            const float v = its[32 * i + lane];
            const bool hit = v > kNone && low - v <= doubt(low) + doubt(v);
            which |= (uint32_t)hit << i;
            hits += hit;
        }
        int32_t before = hits;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += y;
        }
        const int32_t n = p.k + __shfl_sync(0xffffffffu, before, 31);
        if (n <= 32) {
            __syncwarp();
            int32_t *list = (int32_t *)its + before - hits;  // (what the row held has been read)
            for (; which; which &= which - 1) *list++ = 32 * (__ffs(which) - 1) + lane;
            __syncwarp();
            const int32_t e = lane < p.k ? to[lane] : lane < n ? ((int32_t *)its)[lane - p.k] : -1;
            __syncwarp();
            order_exactly<T>(p, x, e, n, to, lane);
        } else {
            const int32_t e = choose_exactly<T, S / 2>(p, x, lane);
            if (lane < p.k) to[lane] = e;
        }
    }
    __syncwarp();
    weigh_scored<T, L>(p, logits, q, out_e, out_w, best, sum, bias != nullptr);
}

}  // namespace
}  // namespace ilw
