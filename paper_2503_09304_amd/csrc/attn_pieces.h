// Packed work of different lengths dealt out to workgroups: which sequence, and which piece of it, a workgroup's number means.
// Every wave finds out for itself, from the lengths on the device: 64 sequences at a time, one a lane.
#pragma once
#include <hip/hip_runtime.h>

namespace qattn {

// Sums of the lanes up to each lane (of 32 bits, saturated), by DPP moves: 4 within rows of 16, then the rows' last lanes to the rows behind.
// Six of the LDS permutations that shuffles are made of would take 0.3 us of a kernel's start.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_from(uint32_t v) {
    return __builtin_elementwise_add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = add_from<0x111, 0xF>(v);      // row_shr:1
    v = add_from<0x112, 0xF>(v);      // row_shr:2
    v = add_from<0x114, 0xF>(v);      // row_shr:4
    v = add_from<0x118, 0xF>(v);      // row_shr:8
    v = add_from<0x142, 0xA>(v);      // row_bcast:15 into rows 1 and 3
    return add_from<0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }

struct Piece {
    int seq, piece, size;             // size: what size(seq) is
};

// Sequence and piece of number `item`, where sequence b has size(b) of something, pieces(size) pieces of it: seq -1 if there is no such item.
template <class S, class F>
__device__ __forceinline__ Piece find_piece(int n_seqs, uint32_t item, S &&size, F &&pieces) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int b0 = 0; b0 < n_seqs; b0 += 64) {
        const int len = b0 + lane < n_seqs ? size(b0 + lane) : 0;
        const uint32_t n = b0 + lane < n_seqs ? pieces(len) : 0, upto = wave_scan(n);
        const unsigned long long past = __ballot(before + upto > item);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            return {b0 + l, (int)(item - before - (uint32_t)__builtin_amdgcn_readlane((int)(upto - n), l)), __builtin_amdgcn_readlane(len, l)};
        }
        before += last_lane(upto);
    }
    return {-1, 0, 0};
}

}  // namespace qattn
