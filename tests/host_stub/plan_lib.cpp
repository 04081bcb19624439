// The rule that picks dense_linear's kernel (dense_plan.h), for a test to call.
#include "dense_plan.h"

static void give(const qdense::Plan &p, int n_tokens, int R, int K, int bf16, int *out, float *us, long *bytes) {
    const int v[] = {p.tiles, p.rows, p.ks, p.share, p.ranges, p.range_blocks};
    for (int i = 0; i < 6; ++i) out[i] = v[i];
    *us = qdense::us_of(p, n_tokens, R, K, bf16);
    *bytes = (long)qdense::workspace_of(p, n_tokens, R);
}

extern "C" void plan(int n_tokens, int R, int K, int bf16, long bytes, int *out, float *us, long *need) {
    give(qdense::plan_with(n_tokens, R, K, bf16, (size_t)bytes), n_tokens, R, K, bf16, out, us, need);
}
