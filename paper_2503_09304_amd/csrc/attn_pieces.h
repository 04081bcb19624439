// Packed work of different lengths dealt out to workgroups: which sequence, and which piece of it, a workgroup's number means.
// Every wave finds out for itself, from the lengths on the device: 64 sequences at a time, one a lane.
#pragma once
#include <hip/hip_runtime.h>

namespace qattn {

// Sum over the wave, in every lane.
__device__ __forceinline__ long wave_sum(long v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Sequence and piece of number `item`, where sequence b has pieces(b) pieces: {-1, pieces in all} if there is no such item.
template <class F>
__device__ __forceinline__ int2 find_piece(int n_seqs, int item, F &&pieces) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < n_seqs; b0 += 64) {
        const int n = b0 + lane < n_seqs ? pieces(b0 + lane) : 0;
        int upto = n;                                                 // pieces of this lane's sequence and those before it
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const unsigned long long past = __ballot(before + upto > item);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            return {b0 + l, item - before - __shfl(upto - n, l, 64)};
        }
        before += __shfl(upto, 63, 64);
    }
    return {-1, before};
}

}  // namespace qattn
