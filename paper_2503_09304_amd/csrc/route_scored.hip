// moe_route_scored: the gate GEMM in ranges of the hidden size, and the choice behind it: scores by softmax or sigmoid, a bias that counts for the choice
// alone, the best groups, the best experts of those, their weights.
//
// Everything behind the logits is in 64 bits: two values that differ by less than the error of an fp32 exponential would change places with any other way
// to compute it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <type_traits>

#include "lds_loads.h"
#include "qmoe_internal.h"

namespace qmoe {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- gate GEMM ----

constexpr int kMostRanges = 16, kMostWaves = 16;
constexpr int EB = 2;                 // experts a lane (4, in half as many waves: nothing won)
constexpr int kStage = 128;           // columns of the hidden size that stand in LDS at once

// Products of TT * 16 tokens with all experts over a range of the hidden size: a wave has 16 * EB = 32 experts (and, where experts are few, one of `slices` parts of the range),
// lane l's operands are those from EB * (l%16) on.  Row-major weights [H][E] (E a multiple of EB): it takes EB elements of each of 8 rows and turns them over in
// registers, so no transposed copy is written first.  Tokens stand in LDS, a stage ahead; the next stage's weights of a step are asked for as soon as this
// stage's have become operands, between the products.
// Bound by latency where tokens are few (a range has few stages, each a way to memory), else by that and the tokens' bytes together: 8192 tokens, H 4096: on 64 experts 28 us
// with the choice, on 160 41 to 44, where the bytes alone take 13.  Tried: weights through LDS (27 to 29 us for this kernel alone instead of 30; 61 tokens 8.9 instead of 6.6).
template <int TT, bool PACKED>
__global__ __launch_bounds__(64 * kMostWaves) void gate_ranges(const uint16_t *x, const uint16_t *Wg, float *part, int N, int H, int E,
                                                                   int blocks, int slices, int range) {
    extern __shared__ __align__(16) char lds[];
    constexpr int STEPS = kStage / 32, PIECES = kStage / 8, STAGE_BYTES = TT * 16 * kStage * 2, ASKS = PACKED ? EB : 8;      // a step's loads
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, t16 = l & 15, g = l >> 4;
    const int pb = w % blocks, sl = w / blocks;
    const int t0 = blockIdx.x * (TT * 16), from = blockIdx.y * range, to = min(H, from + range);
    const int per = ((to - from + slices - 1) / slices + 31) / 32 * 32, k0 = min(to, from + sl * per), k1 = min(to, k0 + per);
    char *const mine = lds + sl * 2 * STAGE_BYTES;
    // The blocks' waves of a slice bring its tokens.  Token t's piece p (8 columns) stands in place p ^ t of its 16, so that the 16 tokens of a read use all banks.
    const auto bring = [&](int k, int buf) {
        for (int j = pb; j < TT * STEPS; j += blocks) {
            const int i = j * 64 + l, t = i / PIECES, at = k + ((i % PIECES) ^ (t & 15)) * 8;
            to_lds((const char *)(x + (long)min(t0 + t, N - 1) * H + (at < H ? at : 0)), mine + buf * STAGE_BYTES + j * 1024);
        }
    };
    typedef unsigned int words __attribute__((ext_vector_type(EB / 2)));
    const int e0 = pb * (16 * EB) + EB * t16;
    u32x4 packed[STEPS][EB];
    words raw[STEPS][8];
    const auto ask = [&](int s, int k) {
        const int row = min(k + 32 * s + 8 * g, H - 8);  // behind the range: not multiplied
        if constexpr (PACKED) {
#pragma unroll
            for (int h = 0; h < EB; ++h) packed[s][h] = *reinterpret_cast<const u32x4 *>(Wg + (long)min(e0 + h, E - 1) * H + row);
        } else {
            const uint16_t *p = Wg + (long)row * E + min(e0, E - EB);
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[s][i] = *reinterpret_cast<const words *>(p + (long)i * E);
        }
    };
    f32x4 acc[TT][EB];
#pragma unroll
    for (int n = 0; n < TT; ++n)
#pragma unroll
        for (int h = 0; h < EB; ++h) acc[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int rounds = (per + kStage - 1) / kStage;      // of all slices alike: they share the barriers
    bring(min(k0, H - 1) & ~31, 0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) ask(s, k0);
    const auto stage = [&](int i, auto more) {
        const int k = k0 + i * kStage;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STEPS * ASKS) : "memory");      // this wave's pieces are in LDS: the weights were asked for behind them
        __syncthreads();
        if constexpr (decltype(more)::value) bring(k + kStage, (i + 1) & 1);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            bf16x8 now[EB], a[TT];
#pragma unroll
            for (int n = 0; n < TT; ++n)
                a[n] = *reinterpret_cast<const bf16x8 *>(mine + (i & 1) * STAGE_BYTES + (n * 16 + t16) * (PIECES * 16) + ((4 * s + g) ^ t16) * 16);
#pragma unroll
            for (int h = 0; h < EB; ++h) {
                if constexpr (PACKED) {
                    now[h] = __builtin_bit_cast(bf16x8, packed[s][h]);
                } else {
                    u32x4 v;
#pragma unroll
                    for (int r = 0; r < 4; ++r)          // rows 2r and 2r + 1
                        v[r] = __builtin_amdgcn_perm(raw[s][2 * r + 1][h / 2], raw[s][2 * r][h / 2], h % 2 ? 0x07060302u : 0x05040100u);
                    now[h] = __builtin_bit_cast(bf16x8, v);
                }
            }
            if constexpr (decltype(more)::value) ask(s, k + kStage);
            if (k + 32 * s >= k1) continue;
#pragma unroll
            for (int n = 0; n < TT; ++n) {
#pragma unroll
                for (int h = 0; h < EB; ++h) acc[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n], now[h], acc[n][h], 0, 0, 0);
            }
        }
    };
    for (int i = 0; i + 1 < rounds; ++i) stage(i, std::true_type{});
    stage(rounds - 1, std::false_type{});
    if (slices > 1) {
        f32x4 *red = reinterpret_cast<f32x4 *>(lds);
        __syncthreads();                                 // the tokens have been read
        if (sl > 0)
#pragma unroll
            for (int n = 0; n < TT; ++n)
#pragma unroll
                for (int h = 0; h < EB; ++h) red[((w - blocks) * (EB * TT) + EB * n + h) * 64 + l] = acc[n][h];
        __syncthreads();
        if (sl > 0) return;
        for (int i = 1; i < slices; ++i)
#pragma unroll
            for (int n = 0; n < TT; ++n)
#pragma unroll
                for (int h = 0; h < EB; ++h) {
                    const f32x4 o = red[((w + (i - 1) * blocks) * (EB * TT) + EB * n + h) * 64 + l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][h][e] += o[e];
                }
    }
    typedef float floats __attribute__((ext_vector_type(EB)));
#pragma unroll
    for (int n = 0; n < TT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + n * 16 + 4 * g + i;
            float *o = part + ((long)blockIdx.y * N + t) * E + e0;
            if (t >= N || e0 >= E) continue;
            if (E % EB == 0) {
                floats v;
#pragma unroll
                for (int h = 0; h < EB; ++h) v[h] = acc[n][h][i];
                *reinterpret_cast<floats *>(o) = v;
            } else {
#pragma unroll
                for (int h = 0; h < EB; ++h)
                    if (e0 + h < E) o[h] = acc[n][h][i];
            }
        }
}

// ---- choice ----

constexpr int kTokens = 4;            // tokens a workgroup, one wave each

struct Rule {
    const float *logit_bias, *choice_bias;
    int sigmoid, groups, take, renorm;
    float factor;
};

// Largest value of the wave's 64 lanes, in every lane; `least` is nobody's loss (one instruction a step, where a step's own value in its place takes two).
template <class T>
__device__ __forceinline__ T wave_max(T v, T least) {
    const auto step = [&](auto ctrl) {
        v = max(v, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, least), __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    step(std::integral_constant<int, 0x111>{});          // row_shr 1, 2, 4, 8; row_bcast 15 and 31: lane 63 holds the wave's
    step(std::integral_constant<int, 0x112>{});
    step(std::integral_constant<int, 0x114>{});
    step(std::integral_constant<int, 0x118>{});
    step(std::integral_constant<int, 0x142>{});
    step(std::integral_constant<int, 0x143>{});
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ double lane_of(double v, int lane) {
    const long long b = __builtin_bit_cast(long long, v);
    const int lo = __builtin_amdgcn_readlane((int)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __builtin_bit_cast(double, (long long)hi << 32 | (unsigned)lo);
}
// Sum over the wave, in every lane.
__device__ __forceinline__ double wave_sum(double v) {
    const auto step = [&](auto ctrl, auto rows) {        // lanes without a source, and rows that are not asked, add 0
        const long long b = __builtin_bit_cast(long long, v);
        const int lo = __builtin_amdgcn_update_dpp(0, (int)b, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v += __builtin_bit_cast(double, (long long)hi << 32 | (unsigned)lo);
    };
    typedef std::integral_constant<int, 0xf> All;
    step(std::integral_constant<int, 0x111>{}, All{});   // row_shr 1, 2, 4, 8: lane 15 of a row holds the row's sum
    step(std::integral_constant<int, 0x112>{}, All{});
    step(std::integral_constant<int, 0x114>{}, All{});
    step(std::integral_constant<int, 0x118>{}, All{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});      // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3: lane 63 holds the wave's
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return lane_of(v, 63);
}

// An order of doubles as pairs of integers, the high words first: NaN below everything, -0 and 0 equal.  A high word of INT_MIN is left for what must not be chosen.
struct Key {
    int hi;
    unsigned lo;
};
__device__ __forceinline__ Key key_of(double v) {
    const long long b = __builtin_bit_cast(long long, v + 0.0), k = b ^ ((b >> 63) & LLONG_MAX);
    return v != v ? Key{INT_MIN + 1, 0u} : Key{(int)(k >> 32), (unsigned)k};
}
__device__ __forceinline__ double largest_first(double &a, double b) {       // a: the larger, returns the other
    const double other = fmin(a, b);
    a = fmax(a, b);
    return other;
}

// A wave has a token, lane l experts l, l + 64, ..., NS in all.  SPLIT: NS waves have a token, 64 experts each up to the scores, and one of them chooses: fewer
// instructions one after the other where tokens leave the chip idle (61 tokens on 256 experts 6.4 us instead of 10.4).  BEST: values that a group's worth is the sum
// of (0: all groups count).  Bound by latency: for each expert chosen a search over the wave whose steps wait for
// each other, and the exponentials and divisions of 64 bits; half of the issue is free (8192 tokens on 160 experts 14.5 us, 6 of 160 in 8 groups).  A single plane of sums is the logits' own array, read and written in place: a wave reads what it
// writes itself and nothing else, lanes behind the last expert its first (another wave may be writing the last one).
template <int NS, int BEST, bool SPLIT>
__global__ __launch_bounds__(64 * (SPLIT ? NS : kTokens)) void score_topk(const float *part, int planes, float *logits, const Rule rule,
                                                                          int32_t *__restrict__ topk_idx, float *__restrict__ topk_w, int N, int E, int k) {
    constexpr int ROWS = SPLIT ? 1 : kTokens, M = SPLIT ? 1 : NS;        // M: slots of this wave
    __shared__ double value[BEST || SPLIT ? ROWS : 1][BEST || SPLIT ? NS * 64 : 1], score[ROWS][NS * 64];
    __shared__ double across[SPLIT ? 2 : 1][NS];
    const int wv = threadIdx.x >> 6, l = threadIdx.x & 63, row = SPLIT ? 0 : wv, c0 = SPLIT ? wv : 0;
    const int t = blockIdx.x * ROWS + row;
    if (t >= N) return;                                  // without SPLIT: no barrier follows, a wave reads what it wrote itself
    float x[M];
    if (planes == 0) {
#pragma unroll
        for (int c = 0; c < M; ++c) x[c] = l + 64 * (c + c0) < E ? logits[(long)t * E + l + 64 * (c + c0)] : -INFINITY;
    } else {
        float q[M][kMostRanges];                         // all asked for before the first is used (one by one: a token on 256 experts 23 us instead of 14)
        const float *p = part + (long)t * E;
#pragma unroll
        for (int z = 0; z < kMostRanges; ++z)
            if (z < planes)
#pragma unroll
                for (int c = 0; c < M; ++c) q[c][z] = p[(long)z * N * E + (l + 64 * (c + c0) < E ? l + 64 * (c + c0) : 64 * (c + c0))];
#pragma unroll
        for (int c = 0; c < M; ++c) {
            const int e = l + 64 * (c + c0);
            float v = q[c][0];
#pragma unroll
            for (int z = 1; z < kMostRanges; ++z)
                if (z < planes) v += q[c][z];
            if (rule.logit_bias != nullptr) v += rule.logit_bias[min(e, E - 1)];
            if (e < E) logits[(long)t * E + e] = v;
            x[c] = e < E ? v : -INFINITY;
        }
    }
    double s[M];
    if (rule.sigmoid) {
#pragma unroll
        for (int c = 0; c < M; ++c) s[c] = 1.0 / (1.0 + exp(-(double)x[c]));
    } else {
        float m = x[0];
#pragma unroll
        for (int c = 1; c < M; ++c) m = fmaxf(m, x[c]);
        m = wave_max(m, -INFINITY);
        if constexpr (SPLIT) {
            if (l == 0) across[0][wv] = m;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < NS; ++c) m = fmaxf(m, (float)across[0][c]);
        }
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < M; ++c) {
            s[c] = l + 64 * (c + c0) < E ? exp((double)x[c] - (double)m) : 0.0;
            sum += s[c];
        }
        sum = wave_sum(sum);
        if constexpr (SPLIT) {
            if (l == 0) across[1][wv] = sum;
            __syncthreads();
            sum = across[1][0];
#pragma unroll
            for (int c = 1; c < NS; ++c) sum += across[1][c];
        }
        const double inv = 1.0 / sum;
#pragma unroll
        for (int c = 0; c < M; ++c) s[c] *= inv;
    }
    Key key[NS];
#pragma unroll
    for (int c = 0; c < M; ++c) {
        const int e = l + 64 * (c + c0);
        double v = s[c];
        if (rule.choice_bias != nullptr) v += (double)rule.choice_bias[min(e, E - 1)];
        if constexpr (BEST > 0 || SPLIT) value[row][e] = v;
        score[row][e] = s[c];
        if constexpr (!SPLIT) key[c] = key_of(v);
    }
    if constexpr (SPLIT) {
        __syncthreads();
        if (wv > 0) return;
#pragma unroll
        for (int c = 0; c < NS; ++c) key[c] = key_of(value[0][l + 64 * c]);
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // lanes read what others of their wave wrote
    }
#pragma unroll
    for (int c = 0; c < NS; ++c)
        if (l + 64 * c >= E) key[c].hi = INT_MIN;
    if constexpr (BEST > 0) {
        // 64 / groups lanes, rounded down to a power of two, look through a group and put together what they found.
        const int size = E / rule.groups, log_lanes = 31 - __builtin_clz(64 / rule.groups), lanes = 1 << log_lanes, grp = l >> log_lanes;
        double best[BEST];
#pragma unroll
        for (int i = 0; i < BEST; ++i) best[i] = -INFINITY;
        for (int i0 = l & (lanes - 1); i0 < size && grp < rule.groups; i0 += 4 * lanes) {        // at most 8 values a lane
            double v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = value[row][grp * size + min(i0 + i * lanes, size - 1)];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                double o = i0 + i * lanes < size && v[i] == v[i] ? v[i] : -INFINITY;       // a NaN adds nothing to its group's worth
#pragma unroll
                for (int j = 0; j < BEST; ++j) o = largest_first(best[j], o);
            }
        }
        for (int o = 1; o < lanes; o <<= 1) {
            double other[BEST];
#pragma unroll
            for (int j = 0; j < BEST; ++j) other[j] = __shfl_xor(best[j], o, 64);
#pragma unroll
            for (int i = 0; i < BEST; ++i) {
                double v = other[i];
#pragma unroll
                for (int j = 0; j < BEST; ++j) v = largest_first(best[j], v);
            }
        }
        double worth = best[0];
#pragma unroll
        for (int j = 1; j < BEST; ++j) worth += best[j];
        const Key mine = key_of(worth);
        int rank = 0;
        for (int n = 0; n < rule.groups; ++n) {
            const int hi = __builtin_amdgcn_readlane(mine.hi, n << log_lanes);
            const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)mine.lo, n << log_lanes);
            rank += hi > mine.hi || (hi == mine.hi && (lo > mine.lo || (lo == mine.lo && n < grp))) ? 1 : 0;
        }
        const unsigned long long kept = __ballot(rank < rule.take);
        const unsigned inv = 65536u / size + 1;          // e / size = e * inv / 65536 for e below 256
#pragma unroll
        for (int c = 0; c < NS; ++c)
            if (!(kept >> (((l + 64 * c) * inv >> 16) << log_lanes & 63) & 1)) key[c].hi = INT_MIN;
    }
    int mine_e = 0;
    for (int j = 0; j < k; ++j) {
        int top = key[0].hi;
#pragma unroll
        for (int c = 1; c < NS; ++c) top = max(top, key[c].hi);
        top = wave_max(top, INT_MIN);
        unsigned long long at[NS];
        int n = 0;
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            at[c] = __ballot(key[c].hi == top);
            n += __builtin_popcountll(at[c]);
        }
        if (n > 1) {                                     // values that differ in the low word alone, or not at all
            unsigned low = 0;
#pragma unroll
            for (int c = 0; c < NS; ++c) low = max(low, key[c].hi == top ? key[c].lo : 0u);
            low = wave_max(low, 0u);
#pragma unroll
            for (int c = 0; c < NS; ++c) at[c] = __ballot(key[c].hi == top && key[c].lo == low);
        }
        int e = 0;
#pragma unroll
        for (int c = NS - 1; c >= 0; --c)
            if (at[c]) e = 64 * c + __builtin_ctzll(at[c]);
#pragma unroll
        for (int c = 0; c < NS; ++c)
            if (l + 64 * c == e) key[c].hi = INT_MIN;
        if (l == j) mine_e = e;
    }
    const double mine = score[row][mine_e];
    const double sum = rule.renorm ? wave_sum(l < k ? mine : 0.0) : 0.0;
    if (l < k) {
        const double w = !rule.renorm ? mine : sum == 0.0 ? 1.0 / k : mine / sum;
        topk_idx[(long)t * k + l] = mine_e;
        topk_w[(long)t * k + l] = (float)(w * (double)rule.factor);
    }
}

}  // namespace

hipError_t launch_score(const RouteArgs &a, const float *part, int planes, hipStream_t s) {
    const moe_scoring &c = *a.scoring;
    const Rule rule{c.logit_bias, c.choice_bias, c.score == MOE_SCORE_SIGMOID, c.groups, c.top_groups, c.renormalise, c.factor};
    // SPLIT against not, logits included, H 2048, us: 61 tokens 11.4 / 13.1 on 128 experts, 11.7 / 15.8 on 256; 2048 tokens 15.8 / 17.3, 20.1 / 21.8; 4096 19.3 / 19.9, 25.2 / 25.8; 8192 29.1 /
    // 27.3, 38.1 / 37.3.
    const bool split = a.N <= 4096 && a.E > 64;
    const auto go = [&](auto ns, auto best) {
        constexpr int NS = decltype(ns)::value, BEST = decltype(best)::value;
        if (NS > 1 && split) score_topk<NS, BEST, (NS > 1)><<<dim3(a.N), dim3(64 * NS), 0, s>>>(part, planes, a.logits, rule, a.topk_idx, a.topk_w, a.N, a.E, a.k);
        else score_topk<NS, BEST, false><<<dim3((a.N + kTokens - 1) / kTokens), dim3(64 * kTokens), 0, s>>>(part, planes, a.logits, rule, a.topk_idx, a.topk_w, a.N, a.E, a.k);
    };
    const auto by_best = [&](auto ns) {
        if (c.top_groups == c.groups) go(ns, std::integral_constant<int, 0>{});
        else if (c.group_best == 1) go(ns, std::integral_constant<int, 1>{});
        else if (c.group_best == 2) go(ns, std::integral_constant<int, 2>{});
        else if (c.group_best == 3) go(ns, std::integral_constant<int, 3>{});
        else go(ns, std::integral_constant<int, 4>{});
    };
    if (a.E <= 64) by_best(std::integral_constant<int, 1>{});
    else if (a.E <= 128) by_best(std::integral_constant<int, 2>{});
    else if (a.E <= 192) by_best(std::integral_constant<int, 3>{});
    else by_best(std::integral_constant<int, 4>{});
    return hipGetLastError();
}

hipError_t launch_gate_scored(const RouteArgs &a, hipStream_t s) {
    const int tt = a.N <= 512 ? 1 : a.N <= 2048 ? 2 : 4, tiles = (a.N + tt * 16 - 1) / (tt * 16);
    const int blocks = (a.E + 16 * EB - 1) / (16 * EB);
    // Tokens a workgroup: few while ranges can be enough workgroups all the same, as a range's products and sums are one after the other then (61 tokens on 256 experts, H 4096: 16 / 32 / 64
    // a workgroup 11.2 / 11.3 / 12.8 us with the choice; 512 on 128 11.9 / 12.0 / 14.4); with many tokens the weights' way to the workgroups counts (8192 on 256: 87 / 56 / 52).
    // Ranges: as many as give 256 workgroups, 16 at most, what the scratch holds.  Their parts: up to 16 waves, 4 parts.  Both of a stage's columns at least.
    const long fit = (long)a.k * a.H / a.E;              // the context's room for k rows of H floats a token
    long ranges = std::max(1l, std::min({256l / tiles, (long)kMostRanges, (long)a.H / kStage, fit}));
    const int range = (int)(((a.H + ranges - 1) / ranges + 63) / 64 * 64);
    ranges = (a.H + range - 1) / range;
    const int slices = std::max(1, std::min({4, kMostWaves / blocks, (range + kStage - 1) / kStage}));
    float *part = ranges > 1 ? a.scratch : a.logits;
    const auto go = [&](auto t, auto packed) {
        constexpr int TT = decltype(t)::value;
        const size_t lds = std::max<size_t>((size_t)slices * 2 * TT * 16 * kStage * 2, (size_t)(slices - 1) * blocks * EB * TT * 1024);
        gate_ranges<TT, decltype(packed)::value><<<dim3(tiles, (unsigned)ranges), dim3(64 * blocks * slices), lds, s>>>((const uint16_t *)a.x, (const uint16_t *)a.Wg, part, a.N, a.H, a.E,
                                                                                                                        blocks, slices, range);
    };
    const auto by_layout = [&](auto t) { a.packed ? go(t, std::true_type{}) : go(t, std::false_type{}); };
    if (tt == 1) by_layout(std::integral_constant<int, 1>{});
    else if (tt == 2) by_layout(std::integral_constant<int, 2>{});
    else by_layout(std::integral_constant<int, 4>{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_score(a, part, (int)ranges, s) : e;
}

}  // namespace qmoe
