// Internal declarations shared by the host side of the dense calls and their kernels (the public ABI is include/qdense.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qdense.h"

namespace qdense {

constexpr int kMaxDim = 32768;

struct Rows {
    char *p;
    uint8_t *scale;
    long ts, hs;                  // elements
};

struct NormArgs {
    Rows x, add, total, out;      // add.p, total.p may be nullptr
    const void *weight;           // may be nullptr
    long rows;                    // n_tokens * heads
    int heads, dim;
    int add_type, out_type, weight_type;
    float shift, eps;
};
hipError_t launch_norm(const NormArgs &a, hipStream_t s);

struct LinearArgs {
    Rows x, out;
    const uint8_t *codes, *scales;
    int n_tokens, R, K;
    int x_type, out_type;
    int ranges;                   // ranges of columns in workgroups of their own (launch_linear sets it)
    float *part;                  // workspace, [range][n_tokens][rows up to a multiple of 16]; may be nullptr
};
// What a call's ranges need of a workspace, 0 without any: see dense_linear.hip.
size_t linear_workspace(int n_tokens, int R, int K, int x_type);
hipError_t launch_linear(LinearArgs a, size_t workspace_bytes, hipStream_t s);
hipError_t launch_linear_some(const LinearArgs &a, int tiles, int rows, int ks, int share, int range_blocks, hipStream_t s);
hipError_t launch_linear_many(const LinearArgs &a, hipStream_t s);
hipError_t launch_pack4(const uint8_t *codes, const uint8_t *scales, int R, int K, uint8_t *dst_codes, uint8_t *dst_scales, hipStream_t s);

}  // namespace qdense
