// The choice of moe_route_scored: scores by softmax or sigmoid, a bias that counts for the choice alone, the best groups, the best
// experts of those, their weights.
//
// Everything behind the logits is in 64 bits: two values that differ by less than the error of an fp32 exponential would change
// places with any other way to compute it.
#include <hip/hip_runtime.h>

#include <climits>

#include "qmoe_internal.h"

namespace qmoe {
namespace {

constexpr int kSlots = kMaxExperts / 64;
constexpr int kTokens = 4;            // tokens a workgroup, one wave each

struct Rule {
    const float *choice_bias;
    int sigmoid, groups, take, best, renorm;
    float factor;
};

// An order of doubles as integers: NaN below everything, -0 and 0 equal.
__device__ __forceinline__ long long order_key(double v) {
    const long long b = __builtin_bit_cast(long long, v + 0.0);
    return v != v ? LLONG_MIN : b ^ ((b >> 63) & LLONG_MAX);
}
__device__ __forceinline__ long long lane_of(long long v, int lane) {
    const int lo = __builtin_amdgcn_readlane((int)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
    return (long long)hi << 32 | (unsigned)lo;
}
__device__ __forceinline__ double lane_of(double v, int lane) { return __builtin_bit_cast(double, lane_of(__builtin_bit_cast(long long, v), lane)); }
__device__ __forceinline__ long long wave_max(long long v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A wave has a token; lane l has experts l, l + 64, ...
__global__ __launch_bounds__(64 * kTokens) void score_topk(const float *__restrict__ logits, const Rule rule, int32_t *__restrict__ topk_idx,
                                                           float *__restrict__ topk_w, int N, int E, int k) {
    __shared__ double value[kTokens][kMaxExperts];
    const int wv = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int t = blockIdx.x * kTokens + wv;
    if (t >= N) return;                                  // no barrier follows: a wave reads what it wrote itself
    const float *lg = logits + (long)t * E;
    float x[kSlots];
#pragma unroll
    for (int c = 0; c < kSlots; ++c) x[c] = l + 64 * c < E ? lg[l + 64 * c] : -INFINITY;
    double s[kSlots];
    if (rule.sigmoid) {
#pragma unroll
        for (int c = 0; c < kSlots; ++c) s[c] = 1.0 / (1.0 + exp(-(double)x[c]));
    } else {
        float m = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < kSlots; ++c) {
            s[c] = l + 64 * c < E ? exp((double)x[c] - (double)m) : 0.0;
            sum += s[c];
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int c = 0; c < kSlots; ++c) s[c] /= sum;
    }
    long long key[kSlots];
#pragma unroll
    for (int c = 0; c < kSlots; ++c) {
        const int e = l + 64 * c;
        double v = s[c];
        if (e < E) {
            if (rule.choice_bias != nullptr) v += (double)rule.choice_bias[e];
            value[wv][e] = v;
        }
        key[c] = order_key(v);
    }
    unsigned long long taken_groups = ~0ull;             // bit g: the token may choose from group g
    const int size = E / rule.groups;
    if (rule.take < rule.groups) {
        long long worth = LLONG_MIN;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // lanes read what others of their wave wrote
        if (l < rule.groups) {
            double best[kMaxGroupBest];
#pragma unroll
            for (int i = 0; i < kMaxGroupBest; ++i) best[i] = -INFINITY;
            for (int i = 0; i < size; ++i) {
                double v = value[wv][l * size + i];
#pragma unroll
                for (int j = 0; j < kMaxGroupBest; ++j) {            // kept in descending order
                    const double b = best[j];
                    const bool more = v > b;
                    best[j] = more ? v : b;
                    v = more ? b : v;
                }
            }
            double sum = best[0];
#pragma unroll
            for (int j = 1; j < kMaxGroupBest; ++j)
                if (j < rule.best) sum += best[j];
            worth = order_key(sum);
        }
        int rank = 0;
        for (int g = 0; g < rule.groups; ++g) {
            const long long o = lane_of(worth, g);
            rank += o > worth || (o == worth && g < l) ? 1 : 0;
        }
        taken_groups = __ballot(l < rule.groups && rank < rule.take);
    }
    unsigned long long left[kSlots];
#pragma unroll
    for (int c = 0; c < kSlots; ++c) {
        const int e = l + 64 * c;
        const bool in = e < E && (taken_groups >> (e / size) & 1);
        left[c] = __ballot(in);
        if (!in) key[c] = LLONG_MIN;
    }
    double mine = 0.0;
    int mine_e = 0;
    for (int j = 0; j < k; ++j) {
        long long m = LLONG_MIN;
#pragma unroll
        for (int c = 0; c < kSlots; ++c) m = max(m, left[c] >> l & 1 ? key[c] : LLONG_MIN);
        m = wave_max(m);
        int e = 0;
#pragma unroll
        for (int c = kSlots - 1; c >= 0; --c) {
            const unsigned long long b = __ballot(key[c] == m) & left[c];
            if (b) e = 64 * c + __builtin_ctzll(b);
        }
        double sv = 0.0;
#pragma unroll
        for (int c = 0; c < kSlots; ++c)
            if (c == e >> 6) {
                left[c] &= ~(1ull << (e & 63));
                sv = s[c];
            }
        sv = lane_of(sv, e & 63);
        if (l == j) {
            mine = sv;
            mine_e = e;
        }
    }
    const double sum = wave_sum(l < k ? mine : 0.0);
    if (l < k) {
        const double w = !rule.renorm ? mine : sum == 0.0 ? 1.0 / k : mine / sum;
        topk_idx[(long)t * k + l] = mine_e;
        topk_w[(long)t * k + l] = (float)(w * (double)rule.factor);
    }
}

}  // namespace

hipError_t launch_score(const RouteArgs &a, hipStream_t s) {
    const moe_scoring &c = *a.scoring;
    const Rule rule{c.choice_bias, c.score == MOE_SCORE_SIGMOID, c.groups, c.top_groups, c.group_best, c.renormalise, c.factor};
    score_topk<<<dim3((a.N + kTokens - 1) / kTokens), dim3(64 * kTokens), 0, s>>>(a.logits, rule, a.topk_idx, a.topk_w, a.N, a.E, a.k);
    return hipGetLastError();
}

}  // namespace qmoe
