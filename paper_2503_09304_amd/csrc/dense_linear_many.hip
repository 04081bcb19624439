// dense_linear for many tokens: a tile of 256 rows by 128 tokens a workgroup.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dense_linear.h"

namespace qdense {
namespace {

constexpr int kTokens = 128, kTiles = 8, kRowTiles = 4, kWaves = 4;      // a workgroup's tokens, in tiles of 16; a wave's tiles of 16 rows

template <int XT>
__global__ __launch_bounds__(64 * kWaves, XT == X_WIDE ? 1 : 2) void linear_many(const LinearArgs a, long first_wg) {
    constexpr int PIECES = XT == X_BF16 ? 16 : 8;        // of 16 bytes, in a token's 128 columns
    constexpr int STAGE = kTokens * PIECES * 16, LOADS = STAGE / 1024 / kWaves;
    __shared__ __align__(16) char xs[2][STAGE];
    __shared__ uint32_t xb[2][kTokens];
    const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 4, t16 = l & 15;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16;
    const int row_wgs = (row_tiles + kRowTiles * kWaves - 1) / (kRowTiles * kWaves);
    const long wg = first_wg + blockIdx.x;
    const int t0 = (int)(wg / row_wgs) * kTokens, rt = (int)(wg % row_wgs) * (kRowTiles * kWaves) + w * kRowTiles;
    const uint8_t *codes[kRowTiles], *scales[kRowTiles];
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) {
        const long tile = min(rt + r, row_tiles - 1);
        codes[r] = a.codes + tile * blocks * 1024 + l * 16;
        scales[r] = a.scales + tile * sets * 256 + l * 4;
    }
    // The pieces that this lane brings to LDS: of token `st[j]`, and in which order pieces stand there (see read()).
    const char *src[LOADS];
    int first_piece;
    {
        constexpr int PER = 64 / PIECES;                 // tokens of a wave's load
        const int p = l % PIECES;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int t = (w + kWaves * j) * PER + l / PIECES;
            src[j] = a.x.p + (long)min(t0 + t, a.n_tokens - 1) * a.x.ts * (XT == X_BF16 ? 2 : 1);
        }
        const int t = w * PER + l / PIECES;              // kWaves * PER is a multiple of 16: the same for all j
        const int q = XT == X_BF16 ? p ^ (t & 15) : p ^ (t >> 1 & 7);
        first_piece = XT == X_BF16 ? 4 * (q & 3) + (q >> 2) : XT == X_FP8 ? q : 2 * (q & 3) + (q >> 2);
    }
    const int k_bytes = a.K * (XT == X_BF16 ? 2 : 1);
    const uint8_t *xscale = XT == X_BF16 ? nullptr : a.x.scale + (long)min(t0 + (tid & (kTokens - 1)), a.n_tokens - 1) * (a.K / 32);
    uint32_t next_xb[4] = {0, 0, 0, 0};
    const auto bring = [&](int b, int buf) {
        const int at = (b * PIECES + first_piece) * 16, from = at < k_bytes ? at : 0;        // behind the last column: weights are zero there
#pragma unroll
        for (int j = 0; j < LOADS; ++j) to_lds(src[j] + from, &xs[buf][(w + kWaves * j) * 1024]);
    };
    const auto bring_scales = [&](int b) {
        if constexpr (XT != X_BF16) {
            const int n = a.K / 32, at = 4 * b;
#pragma unroll
            for (int i = 0; i < 4; ++i) next_xb[i] = xscale[min(at + i, n - 1)];
        }
    };
    u32x4 c[kRowTiles];
    uint32_t sc[kRowTiles];
    const auto weights_of = [&](int b) {
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            c[r] = *reinterpret_cast<const u32x4 *>(codes[r] + (long)b * 1024);
            sc[r] = *reinterpret_cast<const uint32_t *>(scales[r] + (b >> 2) * 256);
        }
    };
    f32x4 acc[kRowTiles][kTiles];
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) acc[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    bring(0, 0);
    bring_scales(0);
    weights_of(0);
    for (int b = 0; b < blocks; ++b) {
        const int buf = b & 1;
        if constexpr (XT != X_BF16)
            if (tid < kTokens) xb[buf][tid] = next_xb[0] | next_xb[1] << 8 | next_xb[2] << 16 | next_xb[3] << 24;
        u32x4 cc[kRowTiles];
        uint32_t cs[kRowTiles];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // this wave's pieces are in LDS
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            cc[r] = c[r];
            cs[r] = sc[r] >> 8 * (b & 3) & 255;
        }
        if (b + 1 < blocks) {
            bring(b + 1, buf ^ 1);
            bring_scales(b + 1);
            weights_of(b + 1);
        }
        const char *x = xs[buf];
        if constexpr (XT == X_FP8) {
            const int at = t16 * 128, sw = t16 >> 1;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const u32x4 lo = *reinterpret_cast<const u32x4 *>(x + n * 2048 + at + ((g ^ sw) * 16));
                const u32x4 hi = *reinterpret_cast<const u32x4 *>(x + n * 2048 + at + (((4 + g) ^ sw) * 16));
                const int byte = xb[buf][n * 16 + t16] >> 8 * g & 255;
                const i32x8 v = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) {
                    const i32x8 wv = {(int)cc[r][0], (int)cc[r][1], (int)cc[r][2], (int)cc[r][3], 0, 0, 0, 0};
                    acc[r][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, v, acc[r][n], 4, 0, 0, (int)cs[r], 0, byte);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                bf16x8 wv[kRowTiles];
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) wv[r] = weights8(cc[r][s], power(cs[r]));
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    bf16x8 v;
                    if constexpr (XT == X_BF16) {
                        v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(x + n * 4096 + t16 * 256 + (((4 * s + g) ^ t16) * 16)));
                    } else {
                        const u32x2 o = *reinterpret_cast<const u32x2 *>(x + n * 2048 + t16 * 128 + (((4 * (s >> 1) + g) ^ (t16 >> 1)) * 16) + 8 * (s & 1));
                        v = widened8(o[0], o[1], power(xb[buf][n * 16 + t16] >> 8 * g & 255));
                    }
#pragma unroll
                    for (int r = 0; r < kRowTiles; ++r) acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[r], v, acc[r][n], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        const int t = t0 + n * 16 + t16;
        if (t < a.n_tokens)
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r)
                if ((rt + r) * 16 + g * 4 < a.R) store4(a, t, (rt + r) * 16 + g * 4, acc[r][n]);
    }
}

}  // namespace

hipError_t launch_linear_many(const LinearArgs &a, hipStream_t s) {
    const long row_wgs = ((a.R + 15) / 16 + kRowTiles * kWaves - 1) / (kRowTiles * kWaves), all = row_wgs * ((a.n_tokens + kTokens - 1) / kTokens);
    constexpr long kMost = 1 << 23;
    for (long at = 0; at < all; at += kMost) {
        const dim3 grid((unsigned)(all - at < kMost ? all - at : kMost)), block(64 * kWaves);
        if (a.x_type == DENSE_BF16) linear_many<X_BF16><<<grid, block, 0, s>>>(a, at);
        else if (a.out_type == DENSE_BF16) linear_many<X_FP8><<<grid, block, 0, s>>>(a, at);
        else linear_many<X_WIDE><<<grid, block, 0, s>>>(a, at);
    }
    return hipGetLastError();
}

}  // namespace qdense
