// dense_linear for some tokens to some thousand: bound by the matrix, then by a wave's instructions and its products.
//
// A workgroup has 16 * SHARE * RB rows, NT * 16 tokens and a range of columns; it goes through them in blocks of 128.  Weights, their scales and the tokens of a block all
// come to LDS past the registers, AHEAD blocks before their use: what is under way hides the latency of memory, which registers could not hold (64 tokens by 6144 x 4096
// 18.9 us with weights straight into registers, 13.6 so; more than two blocks ahead change nothing).  They are asked for between a block's products: all at once they keep a wave
// from its first product (256 by 6144 x 4096 24.5 us, 20.5 so).  61 tokens by 4096 x 14336 11.3 us and its ranges' sums; 256 by 6144 x 4096 17 us, 0.75 PFLOP/s.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dense_linear.h"
#include "dense_plan.h"

namespace qdense {
namespace {


template <int N>
__device__ __forceinline__ void wait_but() {             // for all loads but the last N of this wave
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
template <int C, int R>
__device__ __forceinline__ void wait_for(int later) {    // for all but the loads, C each, of `later` blocks, R at most
    if constexpr (R == 0) wait_but<0>();
    else if (later >= R) wait_but<C * R>();
    else wait_for<C, R - 1>(later);
}

// SHARE waves have rows of their own and the tokens in common; KS times as many share the rows, each with every KS-th block of the range, and their sums meet in LDS.  SHARE 4, KS 2: a wave
// alone on its SIMD issues an instruction every four or five clocks at best (64 tokens by 6144 x 4096 in tiles of 2x1 12.9 us with KS 1, 10.0 with 2, 9.6 with 4; 256 in tiles of 4x2
// 20.5 and 18.1).  SHARE 1, KS 4: small matrices; each wave has tokens of its own, and no barrier stands between blocks.
template <int XT, int NT, int RB, int KS, int SHARE, int AHEAD>
__global__ __launch_bounds__(64 * KS * SHARE) void linear_some(const LinearArgs a, long first_wg, int range_blocks) {
    constexpr int kWaves = KS * SHARE;
    constexpr int PIECES = XT == X_BF16 ? 16 : 8;        // of 16 bytes, in a token's 128 columns
    constexpr int TOK = NT * 16, X = TOK * PIECES * 16, PLACES = X / 1024, LOADS = PLACES < SHARE ? 1 : PLACES / SHARE, WAVE = RB * 1280, SLOT = KS * X + kWaves * WAVE, SLOTS = AHEAD + 1;
    constexpr int COUNT = LOADS + RB + 1;                // a wave's loads for a block (16 tokens in 8 bits: two waves bring the same)
    constexpr bool TOGETHER = SHARE > 1;                 // waves that share tokens
    static_assert(kSomeBlocks % KS == 0, "all of a round's blocks have their scales in place");
    static_assert(PLACES % SHARE % 2 == 0 && SLOT % 256 == 0, "whole loads");
    constexpr int SUMS = KS == 1 ? 0 : kWaves * RB * NT * 1024;
    static_assert(COUNT * AHEAD < 64, "the counter of loads under way has six bits");
    __shared__ __align__(16) char lds[SLOTS * SLOT > SUMS ? SLOTS * SLOT : SUMS];
    __shared__ uint32_t xb[XT == X_BF16 ? 1 : kSomeBlocks][XT == X_BF16 ? 1 : TOK];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, g = l >> 4, t16 = l & 15;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16, row_wgs = (row_tiles + RB * SHARE - 1) / (RB * SHARE);
    long wg = first_wg + blockIdx.x;
    const int rt = (int)(wg % row_wgs) * (RB * SHARE) + w / KS * RB, wk = w % KS, ws = w / KS;
    wg /= row_wgs;
    const int z = (int)(wg % a.ranges), t0 = (int)(wg / a.ranges) * TOK, from = z * range_blocks, n = min(blocks, from + range_blocks) - from;
    const uint8_t *codes[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) codes[r] = a.codes + ((long)min(rt + r, row_tiles - 1) * blocks + from) * 1024;
    const uint8_t *const scales = a.scales + (long)min(rt, row_tiles - 1) * sets * 256;
    const uint32_t scale_at = (uint32_t)(min(rt + (l >> 4) % RB, row_tiles - 1) - min(rt, row_tiles - 1)) * (sets * 256) + t16 * 16;         // RB tiles' 256 bytes, 16 lanes each
    constexpr int ORDERS = TOGETHER ? 1 : LOADS;          // tokens whose places in 16 are the same have their pieces in the same order
    const char *src[LOADS];
    int first_piece[ORDERS];
    {
        constexpr int PER = 64 / PIECES;                 // tokens of a wave's load
        static_assert(!TOGETHER || SHARE * PER % 16 == 0, "one order");
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int t = (ws + SHARE * j) % PLACES * PER + l / PIECES, p = l % PIECES, q = XT == X_BF16 ? p ^ (t & 15) : p ^ (t >> 1 & 7);
            src[j] = a.x.p + (long)min(t0 + t, a.n_tokens - 1) * a.x.ts * (XT == X_BF16 ? 2 : 1);
            if (j < ORDERS) first_piece[j] = XT == X_BF16 ? 4 * (q & 3) + (q >> 2) : XT == X_FP8 ? q : 2 * (q & 3) + (q >> 2);
        }
    }
    const int k_bytes = a.K * (XT == X_BF16 ? 2 : 1);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds, mine = __builtin_amdgcn_readfirstlane(base + KS * X + w * WAVE),
                   piece0 = __builtin_amdgcn_readfirstlane(base + wk * X + ws % PLACES * 1024);
    const auto ask = [&](int i, int b, int slot) {       // the i-th part of what block b needs
        const uint32_t to = slot * SLOT;
        if (i < RB) {
            to_lds_off<64>(codes[i] + (long)b * 1024, l * 16, mine + to + i * 1024);
        } else if (i == RB) {
            to_lds_off<16 * RB>(scales + ((from + b) >> 2) * 256, scale_at, mine + to + RB * 1024);
        } else {
            const int j = i - RB - 1, at = ((from + b) * PIECES + first_piece[j % ORDERS]) * 16;
            to_lds_at(src[j] + (at < k_bytes ? at : 0), piece0 + to + j * (SHARE * 1024));        // behind the last column: weights are zero there
        }
    };
    // The tokens' scale bytes, four a block, of the kSomeBlocks blocks from block b0 of the range on.
    const auto bring_scales = [&](int b0) {
        const int all = a.K / 32;
        for (int i = tid; i < min(n - b0, kSomeBlocks) * TOK; i += 64 * kWaves) {
            const int b = i / TOK, t = i % TOK;
            const uint8_t *s = a.x.scale + (long)min(t0 + t, a.n_tokens - 1) * all;
            uint32_t v = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) v |= (uint32_t)s[min(4 * (from + b0 + b) + e, all - 1)] << 8 * e;
            xb[b][t] = v;
        }
    };
    if constexpr (XT != X_BF16) bring_scales(0);
    f32x4 acc[RB][NT];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int m = 0; m < NT; ++m) acc[r][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int mine_n = (n - wk + KS - 1) / KS, rounds = TOGETHER ? (n + KS - 1) / KS : mine_n;        // this wave's blocks: wk, wk + KS, ...; waves that share tokens go on together
    for (int i = 0; i < min(AHEAD, mine_n); ++i)
#pragma unroll
        for (int k = 0; k < COUNT; ++k) ask(k, wk + i * KS, i);
    if constexpr (!TOGETHER && XT != X_BF16) __syncthreads();
    int slot = 0, next = AHEAD;
    const auto block = [&](int i, auto more) {
        const int b = wk + i * KS;
        wait_for<COUNT, AHEAD - 1>(mine_n - 1 - i);      // this wave's pieces of block b are in LDS
        if constexpr (TOGETHER) __syncthreads();         // everybody's; and the block before, in whose place the next one comes, has been read
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (XT != X_BF16 && TOGETHER)
            if (i > 0 && i * KS % kSomeBlocks == 0) {    // a range that is longer than the scales' place, as all waves see (KS divides it)
                bring_scales(i * KS);
                __syncthreads();
            }
        if constexpr (AHEAD == 1) {
            if (i + 1 < mine_n) {
#pragma unroll
                for (int k = 0; k < COUNT; ++k) ask(k, b + KS, next);
            }
        }
        if (KS > 1 && TOGETHER && i >= mine_n) return;              // the last round of an odd number of blocks
        const char *x = lds + slot * SLOT + wk * X, *wt = lds + slot * SLOT + KS * X + w * WAVE;
        u32x4 c[RB];
        uint32_t sc[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            c[r] = *reinterpret_cast<const u32x4 *>(wt + r * 1024 + l * 16);
            sc[r] = *reinterpret_cast<const uint32_t *>(wt + RB * 1024 + r * 256 + l * 4) >> 8 * ((from + b) & 3) & 255;
        }
        products<XT, RB, NT>(acc, c, sc, x, xb[XT == X_BF16 ? 0 : b % kSomeBlocks], g, t16, [&](int at, int n) {
            if constexpr (AHEAD > 1 && decltype(more)::value) {      // beside the first half of the products: all at once they would keep the wave from them
#pragma unroll
                for (int k = 0; k < COUNT; ++k)
                    if (k * n / 2 / COUNT == at) ask(k, b + AHEAD * KS, next);
            }
        });
        slot = slot + 1 == SLOTS ? 0 : slot + 1;
        next = next + 1 == SLOTS ? 0 : next + 1;
    };
    if constexpr (AHEAD == 1) {
        for (int i = 0; i < rounds; ++i) block(i, std::false_type{});
    } else {
        for (int i = 0; i < mine_n - AHEAD; ++i) block(i, std::true_type{});
        for (int i = max(0, mine_n - AHEAD); i < rounds; ++i) block(i, std::false_type{});
    }
    if constexpr (KS > 1) {
        f32x4 *red = reinterpret_cast<f32x4 *>(lds);
        __syncthreads();                                 // all blocks have been read
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int m = 0; m < NT; ++m) red[(w * (RB * NT) + r * NT + m) * 64 + l] = acc[r][m];
        __syncthreads();
        for (int i = wk; i < RB * NT; i += KS) {         // a tile's sums in the order of the waves
            f32x4 v = red[(ws * KS * (RB * NT) + i) * 64 + l];
#pragma unroll
            for (int k = 1; k < KS; ++k) {
                const f32x4 o = red[((ws * KS + k) * (RB * NT) + i) * 64 + l];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += o[e];
            }
            const int t = t0 + i % NT * 16 + t16, o = (rt + i / NT) * 16 + g * 4;
            if (t < a.n_tokens && o < a.R) {
                if (a.ranges == 1) store4(a, t, o, v);
                else *reinterpret_cast<f32x4 *>(a.part + ((long)z * a.n_tokens + t) * (row_tiles * 16l) + o) = v;
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int t = t0 + i * 16 + t16;
        if (t >= a.n_tokens) continue;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int o = (rt + r) * 16 + g * 4;
            if (o >= a.R) continue;
            if (a.ranges == 1) store4(a, t, o, acc[r][i]);
            else *reinterpret_cast<f32x4 *>(a.part + ((long)z * a.n_tokens + t) * (row_tiles * 16l) + o) = acc[r][i];
        }
    }
}

}  // namespace

hipError_t launch_linear_some(const LinearArgs &a, int tiles, int rows, int ks, int share, int range_blocks, hipStream_t s) {
    const auto go = [&](auto xt, auto nt, auto rb, auto ks, auto share) {
        constexpr int XT = decltype(xt)::value, NT = decltype(nt)::value, RB = decltype(rb)::value, KS = decltype(ks)::value, SHARE = decltype(share)::value;
        constexpr int kWaves = KS * SHARE, PER = RB * SHARE;
        const long row_wgs = ((a.R + 15) / 16 + PER - 1) / PER, all = row_wgs * a.ranges * ((a.n_tokens + NT * 16 - 1) / (NT * 16));
        constexpr long kMost = 1 << 21;                  // workgroups of 1024 threads that a launch may have
        const auto run = [&](auto ahead) {
            for (long at = 0; at < all; at += kMost)
                linear_some<XT, NT, RB, KS, SHARE, decltype(ahead)::value><<<dim3((unsigned)(all - at < kMost ? all - at : kMost)), dim3(64 * kWaves), 0, s>>>(a, at, range_blocks);
        };
        // Where a CU has one workgroup, LDS has room for two blocks ahead (512 tokens by 6144 x 4096 33.5 us, 30.9 so; for two workgroups one block ahead is better: 8192 by 4096 x 4096 222).
        if constexpr (NT * RB == 16) all <= 256 ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 1>{});
        else run(std::integral_constant<int, SHARE == 1 && XT == X_BF16 ? 1 : 2>{});
    };
    const auto by_size = [&](auto xt) {
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        typedef std::integral_constant<int, 4> Four;
        if (share == 1) go(xt, Two{}, One{}, Four{}, One{});
        else if (tiles == 1) ks == 2 ? go(xt, One{}, One{}, Two{}, Four{}) : go(xt, One{}, One{}, Four{}, Four{});
        else if (tiles == 2 && rows == 1) ks == 1 ? go(xt, Two{}, One{}, One{}, Four{}) : go(xt, Two{}, One{}, Two{}, Four{});
        else if (tiles == 2) go(xt, Two{}, Two{}, Two{}, Four{});
        else if (rows == 2) ks == 1 ? go(xt, Four{}, Two{}, One{}, Four{}) : go(xt, Four{}, Two{}, Two{}, Four{});
        else go(xt, Four{}, Four{}, One{}, Four{});
    };
    if (a.x_type == DENSE_BF16) by_size(std::integral_constant<int, X_BF16>{});
    else if (a.out_type == DENSE_BF16) by_size(std::integral_constant<int, X_FP8>{});
    else by_size(std::integral_constant<int, X_WIDE>{});
    return hipGetLastError();
}

}  // namespace qdense
