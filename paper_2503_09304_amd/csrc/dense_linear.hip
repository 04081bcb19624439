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
#include "dense_plan.h"

namespace qdense {
namespace {

// Up to 16 tokens: bound by the matrix, and, as it is small, by the launch and the first bytes (one token by 6144 x 4096 5.3 us, 2.5 TB/s, of which 3.6 are there for any size;
// more rows than CUs' waves hold at once, and more tokens, go through linear_some).  A wave has 16 rows and a slice of the columns, and streams its part of the matrix, AHEAD tiles ahead of their use; KS waves of a
// workgroup share rows and add their sums in LDS.  The tokens' columns of the workgroup's range are in LDS from the start.
constexpr int kWaves = kFewWaves;

template <int XT, int KS>
__global__ __launch_bounds__(64 * kWaves) void linear_few(const LinearArgs a, long first_wg, int range_blocks) {
    extern __shared__ __align__(16) char lds[];
    constexpr int PIECES = XT == X_BF16 ? 16 : 8;        // of 16 bytes, in a token's 128 columns
    constexpr int GROUPS = kWaves / KS, AHEAD = 8;
    const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 4;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16, row_wgs = (row_tiles + GROUPS - 1) / GROUPS;
    long wg = first_wg + blockIdx.x;
    const int z = (int)(wg % a.ranges);
    wg /= a.ranges;
    const int rt = (int)(wg % row_wgs) * GROUPS + w / KS, t0 = (int)(wg / row_wgs) * kFewTokens;
    const int from = z * range_blocks, n_blocks = min(blocks, from + range_blocks) - from, n_tok = min(kFewTokens, a.n_tokens - t0);
    const int per = (n_blocks + KS - 1) / KS, s0 = min(n_blocks, w % KS * per), s1 = min(n_blocks, s0 + per);
    const long tile = min(rt, row_tiles - 1);
    const uint8_t *codes = a.codes + (tile * blocks + from) * 1024 + l * 16, *scales = a.scales + tile * sets * 256 + l * 4;
    u32x4 c[AHEAD];
    uint32_t sc[AHEAD];
    const auto ask = [&](int u, int b) {
        c[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + (long)b * 1024));
        sc[u] = *reinterpret_cast<const uint32_t *>(scales + ((from + b) >> 2) * 256);
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (s0 + u < s1) ask(u, s0 + u);
    // Tokens to LDS, pieces in such an order that the lanes of one read use all banks.
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
    const int tok = min(l & 15, n_tok - 1);
    const char *x = lds + tok * row;
    const uint8_t *xs = xb + tok * (n_blocks * 4) + g;
    const int sw = XT == X_BF16 ? (tok ^ g) * 16 : (tok >> 1 ^ g) * 16;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's pieces are in LDS
    __syncthreads();
    for (int b0 = s0; b0 < s1; b0 += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int b = b0 + u;
            if (b >= s1) break;
            const uint32_t wbyte = sc[u] >> 8 * ((from + b) & 3) & 255;
            if constexpr (XT == X_FP8) {
                const u32x4 lo = *reinterpret_cast<const u32x4 *>(x + b * 128 + sw), hi = *reinterpret_cast<const u32x4 *>(x + b * 128 + (sw ^ 64));
                const i32x8 v = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
                const i32x8 wv = {(int)c[u][0], (int)c[u][1], (int)c[u][2], (int)c[u][3], 0, 0, 0, 0};
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, v, acc, 4, 0, 0, (int)wbyte, 0, (int)xs[b * 4]);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    bf16x8 v;
                    if constexpr (XT == X_BF16) {
                        v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(x + b * 256 + (sw ^ 64 * s)));
                    } else {
                        const u32x2 o = *reinterpret_cast<const u32x2 *>(x + b * 128 + (sw ^ 64 * (s >> 1)) + 8 * (s & 1));
                        v = widened8(o[0], o[1], power(xs[b * 4]));
                    }
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(weights8(c[u][s], power(wbyte)), v, acc, 0, 0, 0);
                }
            }
            if (b + AHEAD < s1) ask(u, b + AHEAD);
        }
    }
    if constexpr (KS > 1) {
        f32x4 *red = reinterpret_cast<f32x4 *>(lds);
        __syncthreads();                                 // the tokens have been read
        if (w % KS) red[w * 64 + l] = acc;
        __syncthreads();
        if (w % KS) return;
#pragma unroll
        for (int k = 1; k < KS; ++k) {
            const f32x4 o = red[(w + k) * 64 + l];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += o[e];
        }
    }
    const int t = t0 + (l & 15), o = rt * 16 + g * 4;
    if (t >= a.n_tokens || o >= a.R) return;
    if (a.ranges == 1) store4(a, t, o, acc);
    else *reinterpret_cast<f32x4 *>(a.part + ((long)z * a.n_tokens + t) * (row_tiles * 16l) + o) = acc;
}

// The ranges' sums, added in their order: a launch, and a way to memory and back (61 tokens, 4096 rows, 8 ranges 4.7 us).
__global__ __launch_bounds__(256) void join_ranges(const LinearArgs a) {
    const unsigned quads = (unsigned)(a.R + 15) / 16 * 4, i = blockIdx.x * 256 + threadIdx.x;       // 2^23 at most, as the workspace has 256 MB
    if (i >= a.n_tokens * quads) return;
    const int t = (int)(i / quads), r = (int)(i % quads) * 4;
    if (r >= a.R) return;
    const long plane = (long)a.n_tokens * quads * 4;
    const float *from = a.part + (long)t * quads * 4 + r;
    constexpr int U = 8;                                 // asked for before the first is added
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    for (int z0 = 0; z0 < a.ranges; z0 += U) {
        f32x4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (z0 + u < a.ranges) o[u] = *reinterpret_cast<const f32x4 *>(from + (z0 + u) * plane);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (z0 + u < a.ranges) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += o[u][e];
            }
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

}  // namespace

size_t linear_workspace(int n_tokens, int R, int K, int x_type) { return workspace_of(plan_of(n_tokens, R, K, x_type == DENSE_BF16, kMostWorkspace), n_tokens, R); }

hipError_t launch_linear(LinearArgs a, size_t workspace_bytes, hipStream_t s) {
    const Plan p = plan_with(a.n_tokens, a.R, a.K, a.x_type == DENSE_BF16, workspace_bytes);
    if (p.tiles == 8) return launch_linear_many(a, s);
    a.ranges = p.ranges;
    const int row_tiles = (a.R + 15) / 16;
    if (p.share > 0) {
        const hipError_t e = launch_linear_some(a, p.tiles, p.rows, p.ks, p.share, p.range_blocks, s);
        if (e != hipSuccess) return e;
    } else {
        const auto go = [&](auto xt, auto ks) {
            constexpr int XT = decltype(xt)::value, KS = decltype(ks)::value, PER = kWaves / KS;
            const long all = (long)((row_tiles + PER - 1) / PER) * ((a.n_tokens + kFewTokens - 1) / kFewTokens) * p.ranges;
            constexpr long kMost = 1 << 22;              // workgroups of 512 threads that a launch may have
            for (long at = 0; at < all; at += kMost)
                linear_few<XT, KS><<<dim3((unsigned)std::min(kMost, all - at)), dim3(64 * kWaves), p.lds, s>>>(a, at, p.range_blocks);
        };
        const auto by_slices = [&](auto xt) {
            if (p.ks == 1) go(xt, std::integral_constant<int, 1>{});
            else if (p.ks == 2) go(xt, std::integral_constant<int, 2>{});
            else if (p.ks == 4) go(xt, std::integral_constant<int, 4>{});
            else go(xt, std::integral_constant<int, 8>{});
        };
        if (a.x_type == DENSE_BF16) by_slices(std::integral_constant<int, X_BF16>{});
        else if (a.out_type == DENSE_BF16) by_slices(std::integral_constant<int, X_FP8>{});
        else by_slices(std::integral_constant<int, X_WIDE>{});
    }
    if (p.ranges > 1) {
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
