// Loads from memory to LDS past the registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

// 16 bytes a lane, lane l's at `to` + 16 l.  In assembly: the compiler would wait for it in front of every read of LDS that it cannot tell
// apart.  Nothing is returned; the caller waits (vmcnt) before the barrier behind which the bytes are read.  Between the write of m0, which gives the place in LDS,
// and the load the hardware wants a wait state, which the compiler does not insert in here: an s_nop, or the write of exec.  Without it a load may go to the place
// of the one before.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"          // that m0 is reserved: nothing else in these kernels uses it
__device__ __forceinline__ void to_lds_at(const char *from, uint32_t at) {        // at: of the wave's, in LDS
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "m0", "memory");
}
// The same from one place of the wave's, `off` bytes behind it, by the first LANES lanes (where all 64 are at work).
template <int LANES>
__device__ __forceinline__ void to_lds_off(const uint8_t *from, uint32_t off, uint32_t at) {
    static_assert(LANES == 16 || LANES == 32 || LANES == 64, "whole halves of the wave, or a quarter");
    if constexpr (LANES == 64) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(from), "s"(at) : "m0", "memory");
    else if constexpr (LANES == 32)
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b32 exec_hi, 0\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b32 exec_hi, -1" ::"v"(off), "s"(from), "s"(at) : "m0", "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, 0xffff\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(off), "s"(from), "s"(at) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void to_lds(const char *from, const char *to) {
    to_lds_at(from, __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)to));
}
