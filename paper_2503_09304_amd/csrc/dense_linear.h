// What the kernels of dense_linear share: how weights and 8-bit rows become operands, and the store of results.
#pragma once

#include <hip/hip_runtime.h>

#include "lds_loads.h"
#include "qdense_internal.h"

namespace qdense {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// How rows of x are multiplied: bf16; fp8 by the scaled instruction; fp8 widened to bf16 (fp32 outputs).
enum { X_BF16 = 0, X_FP8 = 1, X_WIDE = 2 };

// 8 weights (a word of codes) as bf16, in hardware: exact for every scale byte (0 is 2^-127, 255 NaN), but infinite from 2^128 on (bytes 253 and 254), which bf16 does not have.
__device__ __forceinline__ bf16x8 weights8(uint32_t w, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return __builtin_bit_cast(bf16x8, r);
}
// 8 e4m3 elements as bf16: exact from 2^-133 to below 2^128; parts below that (scale bytes 0 to 2) are rounded, larger ones (bytes from 247 on) are infinite.
__device__ __forceinline__ bf16x8 widened8(uint32_t lo, uint32_t hi, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }

// Products of a block of 128 columns: a wave's RB * 16 rows (codes c, scale bytes sc) by NT * 16 tokens, which stand in LDS (x; their scale bytes xb, four a token): pieces of 16
// bytes, a token's in an order by its place in 16, so that the lanes of one read use all banks.  The tokens' operands are asked for AHEAD products of RB before theirs, and weights
// are widened during the step before theirs; left to the compiler, operands come two at a time and are waited for.  between(i, n): called behind each of the n groups of products,
// for loads that would keep the wave from its products if they were asked for together.
template <int XT, int RB, int NT, class Between>
__device__ __forceinline__ void products(f32x4 (&acc)[RB][NT], const u32x4 (&c)[RB], const uint32_t (&sc)[RB], const char *x, const uint32_t *xb, int g, int t16,
                                         const Between &between) {
    if constexpr (XT == X_FP8) {
        constexpr int AHEAD = NT < 2 ? NT : 2;
        u32x4 lo[NT], hi[NT];
        uint32_t byte[NT];
        const int at = t16 * 128, sw = t16 >> 1;
        const auto fetch = [&](int n) {
            lo[n] = *reinterpret_cast<const u32x4 *>(x + n * 2048 + at + ((g ^ sw) * 16));
            hi[n] = *reinterpret_cast<const u32x4 *>(x + n * 2048 + at + (((4 + g) ^ sw) * 16));
            byte[n] = xb[n * 16 + t16];
        };
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) fetch(n);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (n + AHEAD < NT) fetch(n + AHEAD);
            const i32x8 v = {(int)lo[n][0], (int)lo[n][1], (int)lo[n][2], (int)lo[n][3], (int)hi[n][0], (int)hi[n][1], (int)hi[n][2], (int)hi[n][3]};
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const i32x8 w = {(int)c[r][0], (int)c[r][1], (int)c[r][2], (int)c[r][3], 0, 0, 0, 0};
                acc[r][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, v, acc[r][n], 4, 0, 0, (int)sc[r], 0, (int)(byte[n] >> 8 * g & 255));
            }
            between(n, NT);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else if constexpr (XT == X_BF16) {
        constexpr int AHEAD = 3, ALL = 4 * NT;
        bf16x8 v[AHEAD + 1], w[2][RB];
        const auto fetch = [&](int i) { v[i % (AHEAD + 1)] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(x + i % NT * 4096 + t16 * 256 + (((4 * (i / NT) + g) ^ t16) * 16))); };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < RB; ++r) w[0][r] = weights8(c[r][0], power(sc[r]));
#pragma unroll
        for (int i = 0; i < ALL; ++i) {
            const int s = i / NT, n = i % NT;
            if (i + AHEAD < ALL) fetch(i + AHEAD);
#pragma unroll
            for (int r = 0; r < RB; ++r)
                if (s < 3 && r * NT / RB == n) w[(s + 1) & 1][r] = weights8(c[r][s + 1], power(sc[r]));
#pragma unroll
            for (int r = 0; r < RB; ++r) acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[s & 1][r], v[i % (AHEAD + 1)], acc[r][n], 0, 0, 0);
            between(i, ALL);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf16x8 w[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) w[r] = weights8(c[r][s], power(sc[r]));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const u32x2 o = *reinterpret_cast<const u32x2 *>(x + n * 2048 + t16 * 128 + (((4 * (s >> 1) + g) ^ (t16 >> 1)) * 16) + 8 * (s & 1));
                const bf16x8 v = widened8(o[0], o[1], power(xb[n * 16 + t16] >> 8 * g & 255));
#pragma unroll
                for (int r = 0; r < RB; ++r) acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[r], v, acc[r][n], 0, 0, 0);
                between(s * NT + n, 4 * NT);
            }
        }
    }
}

// Four rows r .. r+3 of one token.
__device__ __forceinline__ void store4(const LinearArgs &a, int t, int r, const f32x4 &v) {
    if (a.out_type == DENSE_F32) {
        float *to = (float *)a.out.p + t * a.out.ts + r;
        if (r + 4 <= a.R && ((uintptr_t)to & 15) == 0) *reinterpret_cast<f32x4 *>(to) = v;
        else
            for (int i = 0; i < 4 && r + i < a.R; ++i) to[i] = v[i];
    } else {
        uint16_t *to = (uint16_t *)a.out.p + t * a.out.ts + r;
        const u32x2 p = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (r + 4 <= a.R && ((uintptr_t)to & 7) == 0) *reinterpret_cast<u32x2 *>(to) = p;
        else
            for (int i = 0; i < 4 && r + i < a.R; ++i) to[i] = (uint16_t)(p[i / 2] >> 16 * (i % 2));
    }
}

}  // namespace qdense
