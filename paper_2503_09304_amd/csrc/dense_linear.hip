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

// A lane's part of 16 tokens by 128 columns: 32 columns of one token, zero behind the last one.
template <int XT>
struct XTile {
    u32x4 v[XT == X_BF16 ? 4 : 2];
    uint32_t byte;
    // row: of this lane's token; k: first column of the tile
    __device__ __forceinline__ void load(const char *row, const uint8_t *scale, int k, int g, int K) {
        const u32x4 zero = {0, 0, 0, 0};
        const int mine = k + 32 * g;
        const bool in = mine < K;
        if constexpr (XT == X_BF16) {
            const u32x4 *from = reinterpret_cast<const u32x4 *>(row + 2 * (in ? mine : 0));
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const u32x4 r = from[s];
                v[s] = in ? r : zero;
            }
        } else {
            byte = scale[(in ? mine : 0) / 32];
            byte = in ? byte : 127;
            if constexpr (XT == X_FP8) {          // the scaled instruction's 8-bit operand: columns 16 g .. and 64 + 16 g ..
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int at = k + 64 * s + 16 * g;
                    const u32x4 r = *reinterpret_cast<const u32x4 *>(row + (at < K ? at : 0));
                    v[s] = at < K ? r : zero;
                }
            } else {
                const u32x4 *from = reinterpret_cast<const u32x4 *>(row + (in ? mine : 0));
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const u32x4 r = from[s];
                    v[s] = in ? r : zero;
                }
            }
        }
    }
    __device__ __forceinline__ bf16x8 step(int s) const {
        if constexpr (XT == X_BF16) return __builtin_bit_cast(bf16x8, v[s]);
        else return widened8(v[s / 2][2 * (s % 2)], v[s / 2][2 * (s % 2) + 1], power(byte));
    }
};

// acc += w x of one tile of the matrix.
template <int XT, int NT>
__device__ __forceinline__ void multiply(f32x4 (&acc)[NT], const u32x4 &w, uint32_t wbyte, const XTile<XT> (&x)[NT]) {
    if constexpr (XT == X_FP8) {
        const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const i32x8 b = {(int)x[n].v[0][0], (int)x[n].v[0][1], (int)x[n].v[0][2], (int)x[n].v[0][3],
                             (int)x[n].v[1][0], (int)x[n].v[1][1], (int)x[n].v[1][2], (int)x[n].v[1][3]};
            acc[n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[n], 4, 0, 0, (int)wbyte, 0, (int)x[n].byte);
        }
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const bf16x8 a = weights8(w[s], power(wbyte));
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[n].step(s), acc[n], 0, 0, 0);
        }
    }
}

// Few tokens: bound by the matrix.  A workgroup has RB * 16 rows, NT * 16 tokens and a range of columns, which its W waves share
// out; their sums meet in LDS.
template <int XT, int NT, int RB, int W>
__global__ __launch_bounds__(64 * W) void linear_few(const LinearArgs a) {
    __shared__ f32x4 red[W][RB * NT][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, g = l >> 4;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16;
    const int per_range = (blocks + a.ranges - 1) / a.ranges, from = min(blocks, (int)blockIdx.z * per_range), to = min(blocks, from + per_range);
    const int per = (to - from + W - 1) / W, b0 = min(to, from + w * per), b1 = min(to, b0 + per);
    const int rt = blockIdx.x * RB, t0 = blockIdx.y * (NT * 16);
    const char *row[NT];
    const uint8_t *scale[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const long t = min(t0 + n * 16 + (l & 15), a.n_tokens - 1);
        row[n] = a.x.p + t * a.x.ts * (XT == X_BF16 ? 2 : 1);
        scale[n] = a.x.scale + t * (a.K / 32);
    }
    const uint8_t *codes[RB], *scales[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const long tile = min(rt + r, row_tiles - 1);
        codes[r] = a.codes + tile * blocks * 1024 + l * 16;
        scales[r] = a.scales + tile * sets * 256 + l * 4;
    }
    f32x4 acc[RB][NT];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int U = NT == 1 ? 4 : NT == 2 ? 2 : 1;
    for (int b = b0; b < b1; b += U) {
        u32x4 c[U][RB];
        uint32_t sc[U][RB];
        XTile<XT> x[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = min(b + u, b1 - 1);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                c[u][r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes[r] + (long)at * 1024));
                sc[u][r] = *reinterpret_cast<const uint32_t *>(scales[r] + (at >> 2) * 256) >> 8 * (at & 3) & 255;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) x[u][n].load(row[n], scale[n], at * 128, g, a.K);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u < b1) {
#pragma unroll
                for (int r = 0; r < RB; ++r) multiply<XT, NT>(acc[r], c[u][r], sc[u][r], x[u]);
            }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) red[w][r * NT + n][l] = acc[r][n];
    __syncthreads();
    for (int i = w; i < RB * NT; i += W) {
        f32x4 v = red[0][i][l];
#pragma unroll
        for (int j = 1; j < W; ++j) {
            const f32x4 o = red[j][i][l];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += o[e];
        }
        const int t = t0 + (i % NT) * 16 + (l & 15), r = (rt + i / NT) * 16 + g * 4;
        if (t < a.n_tokens && r < a.R) {
            if (a.ranges == 1) store4(a, t, r, v);
            else *reinterpret_cast<f32x4 *>(a.part + ((long)blockIdx.z * a.n_tokens + t) * (row_tiles * 16l) + r) = v;
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

}  // namespace

int linear_ranges(int n_tokens, int R, int K, int x_type, int out_type) { return 1; }

hipError_t launch_linear(const LinearArgs &a, hipStream_t s) {
    if (a.n_tokens > 128) return launch_linear_many(a, s);
    const int row_tiles = (a.R + 15) / 16;
    const auto go = [&](auto xt, auto nt, auto rb, auto w) {
        constexpr int RB = decltype(rb)::value, NT = decltype(nt)::value, W = decltype(w)::value;
        linear_few<decltype(xt)::value, NT, RB, W><<<dim3((row_tiles + RB - 1) / RB, (a.n_tokens + NT * 16 - 1) / (NT * 16), a.ranges), dim3(64 * W), 0, s>>>(a);
    };
    const auto by_tokens = [&](auto xt) {
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        typedef std::integral_constant<int, 4> Four;
        typedef std::integral_constant<int, 8> Eight;
        if (a.n_tokens <= 16) go(xt, One{}, One{}, Eight{});
        else if (a.n_tokens <= 32) go(xt, Two{}, One{}, Eight{});
        else go(xt, Four{}, Four{}, Four{});
    };
    if (a.x_type == DENSE_BF16) by_tokens(std::integral_constant<int, X_BF16>{});
    else if (a.out_type == DENSE_BF16) by_tokens(std::integral_constant<int, X_FP8>{});
    else by_tokens(std::integral_constant<int, X_WIDE>{});
    if (a.ranges > 1) {
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
