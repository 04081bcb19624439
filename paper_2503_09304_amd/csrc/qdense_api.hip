// Host side of the dense calls (include/qdense.h): argument checks, sizes, launches.  No device code here.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "qdense_internal.h"
#include "qmoe_internal.h"

using qmoe::set_error;

namespace {

int32_t hip_result(hipError_t e, const char *what) {
    return e == hipSuccess ? MOE_OK : set_error(MOE_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int element_bytes(int type) { return type == DENSE_F32 ? 4 : type == DENSE_BF16 ? 2 : 1; }

// Rows that are read or written 16 bytes at a time.
int32_t check_rows(const dense_rows *r, int heads, const char *call, const char *name) {
    if (!r || !r->data) return set_error(MOE_E_ARG, "%s: %s is null", call, name);
    if (!aligned(r->data, 16)) return set_error(MOE_E_ARG, "%s: %s is not 16-byte aligned", call, name);
    const int per = 16 / element_bytes(r->type);
    if (r->token_stride < 0 || r->token_stride % per || (heads > 1 && (r->head_stride < 0 || r->head_stride % per)))
        return set_error(MOE_E_ARG, "%s: strides of %s must be multiples of 16 bytes and not negative", call, name);
    if ((r->type == DENSE_FP8) != (r->scale != nullptr)) return set_error(MOE_E_ARG, "%s: fp8 rows have a scale, others have none (%s)", call, name);
    return MOE_OK;
}

// Rows of one type that stand at the same place.
bool same_rows(const dense_rows *a, const dense_rows *b, int n_tokens, int heads) {
    return a->type == b->type && (n_tokens == 1 || a->token_stride == b->token_stride) && (heads == 1 || a->head_stride == b->head_stride);
}

// Rows that are written do not overlap: neither those of one token or one head, nor, where heads of a token reach past the next token and the other way round,
// head h of a token with the two tokens between whose rows it begins.
int32_t check_apart(const dense_rows *r, int n_tokens, int heads, int dim, const char *call, const char *name) {
    typedef __int128 wide;
    const wide ts = r->token_stride, hs = r->head_stride;
    bool apart = (n_tokens == 1 || ts >= dim) && (heads == 1 || hs >= dim);
    if (apart && n_tokens > 1 && heads > 1 && ts < (heads - 1) * hs + dim && hs < (n_tokens - 1) * ts + dim)
        for (int h = 1; h < heads && apart; ++h) {
            const wide t = h * hs / ts, past = h * hs % ts;
            apart = (t >= n_tokens || past >= dim) && (t + 1 >= n_tokens || ts - past >= dim);
        }
    return apart ? MOE_OK : set_error(MOE_E_ARG, "%s: rows of %s overlap", call, name);
}

qdense::Rows rows(const dense_rows *r) {
    return r ? qdense::Rows{(char *)r->data, r->scale, (long)r->token_stride, (long)r->head_stride} : qdense::Rows{nullptr, nullptr, 0, 0};
}

bool matrix_ok(int64_t R, int64_t K) { return R >= 1 && R <= 1 << 24 && K >= 32 && K <= 1 << 20 && K % 32 == 0; }

int32_t check_matrix(const dense_matrix4 *w, const char *call) {
    if (!w) return set_error(MOE_E_ARG, "%s: the matrix is null", call);
    if (!matrix_ok(w->rows, w->cols)) return set_error(MOE_E_ARG, "%s: rows must be 1..2^24, cols a multiple of 32 from 32 to 2^20", call);
    if (!w->codes || !w->scales) return set_error(MOE_E_ARG, "%s: codes or scales is null", call);
    if (!aligned(w->codes, 16) || !aligned(w->scales, 16)) return set_error(MOE_E_ARG, "%s: codes and scales must be 16-byte aligned", call);
    return MOE_OK;
}

constexpr int kMostTokens = 1 << 24;

}  // namespace

extern "C" {

int32_t dense_norm(const dense_rows *x, const dense_rows *add, const dense_rows *total, const dense_rows *out, const void *weight,
                   int32_t weight_type, float shift, float eps, int32_t n_tokens, int32_t heads, int32_t dim, void *stream) {
    const char *call = "dense_norm";
    int32_t rc;
    if (n_tokens < 0 || n_tokens > 1 << 30) return set_error(MOE_E_ARG, "%s: n_tokens must be 0..2^30", call);
    if (heads < 1 || heads > 1024 || (int64_t)n_tokens * heads > 1 << 30) return set_error(MOE_E_ARG, "%s: heads must be 1..1024, n_tokens * heads at most 2^30", call);
    if (!x || !out) return set_error(MOE_E_ARG, "%s: x or out is null", call);
    if (x->type != DENSE_BF16) return set_error(MOE_E_ARG, "%s: x must be bf16", call);
    if (out->type != DENSE_BF16 && out->type != DENSE_FP8) return set_error(MOE_E_ARG, "%s: out must be bf16 or fp8", call);
    if (add && add->type != DENSE_BF16 && add->type != DENSE_F32) return set_error(MOE_E_ARG, "%s: add must be bf16 or fp32", call);
    if (total && (!add || total->type != add->type)) return set_error(MOE_E_ARG, "%s: total needs add, and has its type", call);
    const int step = out->type == DENSE_FP8 ? 32 : 8;
    if (dim < step || dim > qdense::kMaxDim || dim % step) return set_error(MOE_E_ARG, "%s: dim must be a multiple of %d, at most %d", call, step, qdense::kMaxDim);
    if (!(eps > 0.f) || !std::isfinite(eps)) return set_error(MOE_E_ARG, "%s: eps must be positive", call);
    if (weight) {
        if (weight_type != DENSE_BF16 && weight_type != DENSE_F32) return set_error(MOE_E_ARG, "%s: weights must be bf16 or fp32", call);
        if (!aligned(weight, 16)) return set_error(MOE_E_ARG, "%s: weight is not 16-byte aligned", call);
        if (!std::isfinite(shift)) return set_error(MOE_E_ARG, "%s: shift is not finite", call);
    }
    if (n_tokens == 0) return MOE_OK;
    if ((rc = check_rows(x, heads, call, "x")) || (add && (rc = check_rows(add, heads, call, "add"))) ||
        (total && (rc = check_rows(total, heads, call, "total"))) || (rc = check_rows(out, heads, call, "out")) ||
        (total && (rc = check_apart(total, n_tokens, heads, dim, call, "total"))) || (rc = check_apart(out, n_tokens, heads, dim, call, "out")))
        return rc;
    if (total && (total->data == out->data || total->data == x->data || (total->data == add->data && !same_rows(total, add, n_tokens, heads))))
        return set_error(MOE_E_ARG, "%s: total may be add, row by row, and otherwise overlaps nothing", call);
    if ((out->data == x->data && !same_rows(out, x, n_tokens, heads)) || (add && out->data == add->data && !same_rows(out, add, n_tokens, heads)))
        return set_error(MOE_E_ARG, "%s: out may be x or add, row by row, and otherwise overlaps nothing", call);
    const qdense::NormArgs a{rows(x), rows(add), rows(total), rows(out), weight, (long)n_tokens * heads, heads, dim, add ? add->type : DENSE_BF16,
                             out->type, weight_type, shift, eps};
    return hip_result(qdense::launch_norm(a, (hipStream_t)stream), call);
}

size_t dense_matrix4_code_bytes(int32_t R, int32_t K) {
    if (!matrix_ok(R, K)) {
        set_error(MOE_E_ARG, "dense_matrix4_code_bytes: rows must be 1..2^24, cols a multiple of 32 from 32 to 2^20");
        return 0;
    }
    return ((size_t)R + 15) / 16 * (((size_t)K + 127) / 128) * 1024;
}

size_t dense_matrix4_scale_bytes(int32_t R, int32_t K) {
    if (!matrix_ok(R, K)) {
        set_error(MOE_E_ARG, "dense_matrix4_scale_bytes: rows must be 1..2^24, cols a multiple of 32 from 32 to 2^20");
        return 0;
    }
    return ((size_t)R + 15) / 16 * (((size_t)K + 511) / 512) * 256;
}

int32_t dense_pack4(const uint8_t *codes, const uint8_t *scales, const dense_matrix4 *w, void *stream) {
    const char *call = "dense_pack4";
    int32_t rc;
    if ((rc = check_matrix(w, call))) return rc;
    if (!codes || !scales) return set_error(MOE_E_ARG, "%s: codes or scales is null", call);
    if (!aligned(codes, 16)) return set_error(MOE_E_ARG, "%s: codes must be 16-byte aligned", call);
    if (codes == w->codes || scales == w->scales) return set_error(MOE_E_ARG, "%s: cannot pack in place", call);
    return hip_result(qdense::launch_pack4(codes, scales, w->rows, w->cols, (uint8_t *)w->codes, (uint8_t *)w->scales, (hipStream_t)stream), call);
}

size_t dense_linear_workspace_bytes(int32_t n_tokens, int32_t R, int32_t K, int32_t x_type, int32_t out_type) {
    if (n_tokens < 1 || n_tokens > kMostTokens || !matrix_ok(R, K) || (x_type != DENSE_BF16 && x_type != DENSE_FP8) ||
        (out_type != DENSE_BF16 && out_type != DENSE_F32)) {
        set_error(MOE_E_ARG, "dense_linear_workspace_bytes: bad size or type");
        return 0;
    }
    return qdense::linear_workspace(n_tokens, R, K, x_type);
}

int32_t dense_linear(const dense_rows *x, const dense_matrix4 *w, const dense_rows *out, int32_t n_tokens, void *workspace,
                     size_t workspace_bytes, void *stream) {
    const char *call = "dense_linear";
    int32_t rc;
    if ((rc = check_matrix(w, call))) return rc;
    if (n_tokens < 0 || n_tokens > kMostTokens) return set_error(MOE_E_ARG, "%s: n_tokens must be 0..2^24", call);
    if (!x || !out) return set_error(MOE_E_ARG, "%s: x or out is null", call);
    if (x->type != DENSE_BF16 && x->type != DENSE_FP8) return set_error(MOE_E_ARG, "%s: x must be bf16 or fp8", call);
    if (out->type != DENSE_BF16 && out->type != DENSE_F32) return set_error(MOE_E_ARG, "%s: out must be bf16 or fp32", call);
    if (n_tokens == 0) return MOE_OK;
    if ((rc = check_rows(x, 1, call, "x"))) return rc;
    if (!out->data) return set_error(MOE_E_ARG, "%s: out is null", call);
    if (!aligned(out->data, (size_t)element_bytes(out->type))) return set_error(MOE_E_ARG, "%s: out is not aligned to its elements", call);
    if ((rc = check_apart(out, n_tokens, 1, w->rows, call, "out"))) return rc;
    if (out->data == x->data || (workspace && (workspace == x->data || workspace == out->data)))
        return set_error(MOE_E_ARG, "%s: out, x and the workspace overlap", call);
    if (workspace && !aligned(workspace, 16)) return set_error(MOE_E_WORKSPACE, "%s: workspace is not 16-byte aligned", call);
    const qdense::LinearArgs a{rows(x), rows(out), (const uint8_t *)w->codes, w->scales, n_tokens, w->rows, w->cols, x->type, out->type, 1, (float *)workspace};
    return hip_result(qdense::launch_linear(a, workspace ? workspace_bytes : 0, (hipStream_t)stream), call);
}

}  // extern "C"
