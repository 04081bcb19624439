// dense_linear: products with matrices of 4-bit weights, and dense_pack4 that lays them out.
//
//     out[t, r] = sum_c x[t, c] w[r, c],   w = e2m1 element * 2^(byte - 127), a byte for every 32 columns
//
// Matrix instructions with the weights as the first operand (16 rows) and the tokens as the second (16 tokens).  A tile of the
// matrix (16 rows, 128 columns) is 1 KiB in the order of the lanes: lane l has row l%16 and the 32 columns from 32*(l/16) on, which
// share a scale byte.  That is the scaled instruction's operand as it is (fp8 rows), and, since the order of columns inside a
// product is free, four operands of the bf16 instruction: its step s takes the 8 columns from 32*(l/16) + 8 s on, of weights and tokens
// alike.  Weights become bf16 exactly, two elements an instruction.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "dense_linear.h"

namespace qdense {
namespace {

// Few tokens: bound by the matrix.  Each wave has RB tiles of 16 rows and a slice of the columns, and streams its part of the matrix, D tiles ahead of their
// use; KS waves of a workgroup share rows and add their sums in LDS.  The tokens' columns of the workgroup's range are in LDS from the start, 16-byte pieces
// in the places that read() says, so that the lanes of one read use all banks.
constexpr int kWaves = 8;

template <int XT, int NT, int RB, int KS, int D>
__global__ __launch_bounds__(64 * kWaves) void linear_few(const LinearArgs a, long first_wg, int range_blocks) {
    extern __shared__ __align__(16) char lds[];
    constexpr int PIECES = XT == X_BF16 ? 16 : 8;        // of 16 bytes, in a token's 128 columns
    constexpr int GROUPS = kWaves / KS;
    const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 4;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16, row_wgs = (row_tiles + GROUPS * RB - 1) / (GROUPS * RB);
    long wg = first_wg + blockIdx.x;
    const int z = (int)(wg % a.ranges);
    wg /= a.ranges;
    const int rt = (int)(wg % row_wgs) * (GROUPS * RB) + w / KS * RB, t0 = (int)(wg / row_wgs) * (NT * 16);
    const int from = z * range_blocks, n_blocks = min(blocks, from + range_blocks) - from, n_tok = min(NT * 16, a.n_tokens - t0);
    const int per = (n_blocks + KS - 1) / KS, s0 = min(n_blocks, w % KS * per), s1 = min(n_blocks, s0 + per);
    const uint8_t *codes[RB], *scales[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const long tile = min(rt + r, row_tiles - 1);
        codes[r] = a.codes + (tile * blocks + from) * 1024 + l * 16;
        scales[r] = a.scales + tile * sets * 256 + l * 4;
    }
    u32x4 c[D][RB];
    uint32_t sc[D][RB];
    const auto ask = [&](int u, int b) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            c[u][r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes[r] + (long)b * 1024));
            sc[u][r] = *reinterpret_cast<const uint32_t *>(scales[r] + ((from + b) >> 2) * 256);
        }
    };
#pragma unroll
    for (int u = 0; u < D; ++u)
        if (s0 + u < s1) ask(u, s0 + u);
    // Tokens to LDS.
    const int row = n_blocks * PIECES * 16;              // bytes of a token there
    uint8_t *xb = reinterpret_cast<uint8_t *>(lds) + (n_tok * row + 1023) / 1024 * 1024;       // the last wave's load may write up to there
    {
        const int pieces = n_tok * n_blocks * PIECES, k_pieces = a.K / (XT == X_BF16 ? 8 : 16);
        for (int i0 = w * 64; i0 < pieces; i0 += 64 * kWaves) {
            const int i = min(i0 + l, pieces - 1), t = i / (n_blocks * PIECES), p = i - t * (n_blocks * PIECES), b = p / PIECES;
            const int q = XT == X_BF16 ? (p ^ t) & 15 : (p ^ t >> 1) & 7;
            const int piece = (from + b) * PIECES + (XT == X_BF16 ? 4 * (q & 3) + (q >> 2) : XT == X_FP8 ? q : 2 * (q & 3) + (q >> 2));
            to_lds(a.x.p + (t0 + t) * a.x.ts * (XT == X_BF16 ? 2 : 1) + (piece < k_pieces ? piece : 0) * 16, lds + i0 * 16);       // behind the last column weights are zero
        }
        if constexpr (XT != X_BF16) {
            const int n = a.K / 32;
            for (int i = tid; i < n_tok * n_blocks * 4; i += 64 * kWaves) {
                const int t = i / (n_blocks * 4), k = from * 4 + i - t * (n_blocks * 4);
                xb[i] = a.x.scale[(long)(t0 + t) * n + min(k, n - 1)];
            }
        }
    }
    f32x4 acc[RB][NT];
    int at[NT], sw[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int t = min(n * 16 + (l & 15), n_tok - 1);
        at[n] = t * row;
        sw[n] = XT == X_BF16 ? ((t & 15) ^ g) * 16 : ((t >> 1 & 7) ^ g) * 16;
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's pieces are in LDS
    __syncthreads();
    for (int b0 = s0; b0 < s1; b0 += D) {
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int b = b0 + u;
            if (b >= s1) break;
            const int shift = 8 * ((from + b) & 3);
            if constexpr (XT == X_FP8) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const u32x4 lo = *reinterpret_cast<const u32x4 *>(lds + at[n] + b * 128 + sw[n]);
                    const u32x4 hi = *reinterpret_cast<const u32x4 *>(lds + at[n] + b * 128 + (sw[n] ^ 64));
                    const int byte = xb[at[n] / 32 + b * 4 + g];
                    const i32x8 v = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        const i32x8 wv = {(int)c[u][r][0], (int)c[u][r][1], (int)c[u][r][2], (int)c[u][r][3], 0, 0, 0, 0};
                        acc[r][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, v, acc[r][n], 4, 0, 0, (int)(sc[u][r] >> shift & 255), 0, byte);
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    bf16x8 wv[RB];
#pragma unroll
                    for (int r = 0; r < RB; ++r) wv[r] = weights8(c[u][r][s], power(sc[u][r] >> shift & 255));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        bf16x8 v;
                        if constexpr (XT == X_BF16) {
                            v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(lds + at[n] + b * 256 + (sw[n] ^ 64 * s)));
                        } else {
                            const u32x2 o = *reinterpret_cast<const u32x2 *>(lds + at[n] + b * 128 + (sw[n] ^ 64 * (s >> 1)) + 8 * (s & 1));
                            v = widened8(o[0], o[1], power(xb[at[n] / 32 + b * 4 + g]));
                        }
#pragma unroll
                        for (int r = 0; r < RB; ++r) acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[r], v, acc[r][n], 0, 0, 0);
                    }
                }
            }
            if (b + D < s1) ask(u, b + D);
        }
    }
    if constexpr (KS > 1) {
        f32x4 *red = reinterpret_cast<f32x4 *>(lds);
        __syncthreads();                                 // the tokens have been read
        if (w % KS)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) red[(w * (RB * NT) + r * NT + n) * 64 + l] = acc[r][n];
        __syncthreads();
        if (w % KS) return;
#pragma unroll 1
        for (int k = 1; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const f32x4 o = red[((w + k) * (RB * NT) + r * NT + n) * 64 + l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][n][e] += o[e];
                }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int t = t0 + n * 16 + (l & 15);
        if (t >= a.n_tokens) continue;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int o = (rt + r) * 16 + g * 4;
            if (o >= a.R) continue;
            if (a.ranges == 1) store4(a, t, o, acc[r][n]);
            else *reinterpret_cast<f32x4 *>(a.part + ((long)z * a.n_tokens + t) * (row_tiles * 16l) + o) = acc[r][n];
        }
    }
}

// The ranges' sums, added in their order.
__global__ __launch_bounds__(256) void join_ranges(const LinearArgs a) {
    const int quads = (a.R + 15) / 16 * 4;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long)a.n_tokens * quads) return;
    const int t = (int)(i / quads), r = (int)(i % quads) * 4;
    if (r >= a.R) return;
    const long plane = (long)a.n_tokens * quads * 4;
    const float *from = a.part + (long)t * quads * 4 + r;
    f32x4 v = *reinterpret_cast<const f32x4 *>(from);
    for (int z = 1; z < a.ranges; ++z) {
        const f32x4 o = *reinterpret_cast<const f32x4 *>(from + z * plane);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += o[e];
    }
    store4(a, t, r, v);
}

// One thread for 16 bytes of codes (32 columns of a row) and their scale byte.
__global__ __launch_bounds__(256) void pack4(const uint8_t *codes, const uint8_t *scales, int R, int K, uint8_t *dc, uint8_t *ds) {
    const int blocks = (K + 127) / 128, sets = (K + 511) / 512;
    const long n = (long)((R + 15) / 16) * sets * 4 * 64, step = (long)gridDim.x * 256;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int l = (int)(i & 63), b = (int)((i >> 6) % (sets * 4));
        const long tile = (i >> 6) / (sets * 4), row = tile * 16 + (l & 15);
        const int k = b * 128 + 32 * (l >> 4);
        const bool in = row < R && k < K;
        if (b < blocks) {
            const u32x4 zero = {0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(dc + (tile * blocks + b) * 1024 + l * 16) = in ? *reinterpret_cast<const u32x4 *>(codes + (row * K + k) / 2) : zero;
        }
        ds[(tile * sets + b / 4) * 256 + l * 4 + b % 4] = in ? scales[row * (K / 32) + k / 32] : 127;
    }
}

constexpr size_t kMostLds = 128 * 1024;

}  // namespace

// How a call is cut into workgroups.
struct Plan {
    bool many;
    int tiles;                    // of 16 tokens, a workgroup's
    int ks;                       // few: waves that share rows
    int ranges, range_blocks;     // of 128 columns
    size_t lds;                   // few
};
static void cut(Plan &p, int blocks, int ranges) {
    p.range_blocks = (blocks + ranges - 1) / ranges;
    p.ranges = (blocks + p.range_blocks - 1) / p.range_blocks;
}
static Plan few_of(int n_tokens, int R, int K, bool bf16, int ranges) {
    const int blocks = (K + 127) / 128, row_tiles = (R + 15) / 16;
    Plan f{};
    f.tiles = n_tokens <= 16 ? 1 : n_tokens <= 32 ? 2 : 4;
    const int rb = f.tiles == 4 ? 2 : 1, tokens = std::min(n_tokens, f.tiles * 16), token_tiles = (n_tokens + f.tiles * 16 - 1) / (f.tiles * 16);
    const size_t per_block = (size_t)tokens * (bf16 ? 256 : 132);
    const int most = (int)std::min<size_t>(blocks, kMostLds / per_block);
    cut(f, blocks, std::max(ranges, (blocks + most - 1) / most));
    const long units = (long)((row_tiles + rb - 1) / rb) * token_tiles * f.ranges;
    f.ks = 1;
    while (f.ks < 8 && units * f.ks < 2048 && f.range_blocks >= 2 * f.ks) f.ks *= 2;
    f.lds = std::max<size_t>((size_t)f.range_blocks * per_block + 1024, (size_t)(f.ks > 1 ? kWaves * rb * f.tiles * 1024 : 0));
    return f;
}
static Plan many_of(int n_tokens, int R, int K, int tiles, int ranges) {
    Plan f{};
    f.many = true;
    f.tiles = tiles;
    cut(f, (K + 127) / 128, ranges);
    return f;
}
// Us that a plan takes, by what was measured (H 1024 to 14336, 1024 to 32000 rows, 1 to 2048 tokens; most within 15 %): a launch 3; what a CU has to take in, at 28 bytes
// a ns, 20 where LDS leaves room for one workgroup; tiles of many tokens per block of 128 columns and workgroup on a CU; ranges cost a launch, and their sums are written and read.
static float us_of(const Plan &p, int n_tokens, int R, int K, bool bf16) {
    const int row_tiles = (R + 15) / 16, token_tiles = (n_tokens + p.tiles * 16 - 1) / (p.tiles * 16);
    const float join = p.ranges == 1 ? 0.f : (p.many ? 4.f : 2.2f) + (float)p.ranges * n_tokens * R * 8.f / 6e6f;
    if (p.many) {
        const long wgs = (long)((row_tiles + 15) / 16) * token_tiles * p.ranges, on_cu = (wgs + 255) / 256;
        const float block = p.tiles == 8 ? (bf16 ? on_cu > 1 ? 1.5f : 1.75f : 0.95f) : (bf16 ? on_cu > 1 ? 0.83f : 0.95f : 0.6f);
        return 3.f + (float)on_cu * p.range_blocks * block + join;
    }
    const int per = kWaves / p.ks * (p.tiles == 4 ? 2 : 1);
    const long wgs = (long)((row_tiles + per - 1) / per) * token_tiles * p.ranges, on_cu = (wgs + 255) / 256;
    const float x = (float)std::min(n_tokens, p.tiles * 16) * (bf16 ? 256.f : 132.f) * p.range_blocks, w = (float)per * p.range_blocks * 1088.f;
    return 3.f + (float)on_cu * (x + w) / (p.lds > 80 * 1024 ? 20e3f : 28e3f) + join;
}
static Plan plan_of(int n_tokens, int R, int K, bool bf16) {
    const int blocks = (K + 127) / 128;
    Plan best{};
    float least = 0.f;
    const auto look = [&](const Plan &p) {
        const float us = us_of(p, n_tokens, R, K, bf16);
        if (best.tiles == 0 || us < least) {
            best = p;
            least = us;
        }
    };
    for (const int z : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (z > blocks) break;
        if (n_tokens <= 64) look(few_of(n_tokens, R, K, bf16, z));
        if (n_tokens > 16) look(many_of(n_tokens, R, K, 4, z));
        if (n_tokens > 64) look(many_of(n_tokens, R, K, 8, z));
    }
    return best;
}

int linear_ranges(int n_tokens, int R, int K, int x_type, int) { return plan_of(n_tokens, R, K, x_type == DENSE_BF16).ranges; }

hipError_t launch_linear(const LinearArgs &a, hipStream_t s) {
    Plan f = plan_of(a.n_tokens, a.R, a.K, a.x_type == DENSE_BF16);
    if (f.ranges > a.ranges) f = many_of(a.n_tokens, a.R, a.K, a.n_tokens > 64 ? 8 : 4, 1);        // no workspace
    const int row_tiles = (a.R + 15) / 16;
    const auto go = [&](auto xt, auto nt, auto ks) {
        constexpr int XT = decltype(xt)::value, NT = decltype(nt)::value, KS = decltype(ks)::value, RB = NT == 4 ? 2 : 1, D = NT == 4 ? 4 : 8, PER = kWaves / KS * RB;
        const long all = (long)((row_tiles + PER - 1) / PER) * ((a.n_tokens + NT * 16 - 1) / (NT * 16)) * f.ranges;
        constexpr long kMost = 1 << 22;                  // workgroups of 512 threads that a launch may have
        for (long at = 0; at < all; at += kMost)
            linear_few<XT, NT, RB, KS, D><<<dim3((unsigned)std::min(kMost, all - at)), dim3(64 * kWaves), f.lds, s>>>(a, at, f.range_blocks);
    };
    const auto by_slices = [&](auto xt, auto nt) {
        if (f.ks == 1) go(xt, nt, std::integral_constant<int, 1>{});
        else if (f.ks == 2) go(xt, nt, std::integral_constant<int, 2>{});
        else if (f.ks == 4) go(xt, nt, std::integral_constant<int, 4>{});
        else go(xt, nt, std::integral_constant<int, 8>{});
    };
    const auto by_tokens = [&](auto xt) {
        if (f.tiles == 1) by_slices(xt, std::integral_constant<int, 1>{});
        else if (f.tiles == 2) by_slices(xt, std::integral_constant<int, 2>{});
        else by_slices(xt, std::integral_constant<int, 4>{});
    };
    if (f.many) {
        const hipError_t e = launch_linear_many(a, f.tiles, f.range_blocks, s);
        if (e != hipSuccess) return e;
    } else if (a.x_type == DENSE_BF16) by_tokens(std::integral_constant<int, X_BF16>{});
    else if (a.out_type == DENSE_BF16) by_tokens(std::integral_constant<int, X_FP8>{});
    else by_tokens(std::integral_constant<int, X_WIDE>{});
    if (f.ranges > 1) {
        const long n = (long)a.n_tokens * row_tiles * 4;
        join_ranges<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_pack4(const uint8_t *codes, const uint8_t *scales, int R, int K, uint8_t *dst_codes, uint8_t *dst_scales, hipStream_t s) {
    const long n = (long)((R + 15) / 16) * ((K + 511) / 512) * 256;
    pack4<<<dim3((unsigned)std::min<long>((n + 255) / 256, 1 << 16)), dim3(256), 0, s>>>(codes, scales, R, K, dst_codes, dst_scales);
    return hipGetLastError();
}

}  // namespace qdense
