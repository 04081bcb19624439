// What the kernels of dense_linear share: how weights and 8-bit rows become operands, and the store of results.
#pragma once

#include <hip/hip_runtime.h>

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

// 8 weights (a word of codes) as bf16: exact for every scale byte (0 is 2^-127, 255 NaN), in hardware.
__device__ __forceinline__ bf16x8 weights8(uint32_t w, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return __builtin_bit_cast(bf16x8, r);
}
// 8 e4m3 elements as bf16: exact.
__device__ __forceinline__ bf16x8 widened8(uint32_t lo, uint32_t hi, float scale) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }

// 16 bytes a lane from memory to LDS, lane l's at `to` + 16 l.  In assembly: the compiler would wait for it in front of every read of LDS that it cannot tell
// apart.  Nothing is returned; the caller waits (vmcnt) before the barrier behind which the bytes are read.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"          // that m0 is reserved: nothing else here uses it
__device__ __forceinline__ void to_lds_at(const char *from, uint32_t at) {        // at: of the wave's, in LDS
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void to_lds(const char *from, const char *to) {
    to_lds_at(from, __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)to));
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
