// Host side of the attention calls (include/qattn.h): argument checks, the rotary frequencies, launches.  No device code here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "qattn_internal.h"
#include "qmoe_internal.h"

using qmoe::set_error;

namespace {

int32_t hip_result(hipError_t e, const char *what) {
    return e == hipSuccess ? MOE_OK : set_error(MOE_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

constexpr float kLog2E = 1.44269504088896340736f;          // exponentials are powers of two in the kernels

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int32_t check_rows(const attn_rows *r, const char *call, const char *name) {
    if (!r || !r->data) return set_error(MOE_E_ARG, "%s: %s is null", call, name);
    if (!aligned(r->data, 16)) return set_error(MOE_E_ARG, "%s: %s is not 16-byte aligned", call, name);
    if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride % 8 || r->head_stride % 8)
        return set_error(MOE_E_ARG, "%s: strides of %s must be multiples of 8 elements and not negative", call, name);
    return MOE_OK;
}

qattn::Rows rows(const attn_rows *r) {
    return r ? qattn::Rows{(uint16_t *)r->data, (long)r->token_stride, (long)r->head_stride} : qattn::Rows{nullptr, 0, 0};
}

int32_t check_dim(int dim, const char *call) {
    if (dim < 16 || dim > qattn::kMaxDim || dim % 16) return set_error(MOE_E_ARG, "%s: dim must be a multiple of 16 from 16 to %d", call, qattn::kMaxDim);
    return MOE_OK;
}

int32_t check_heads(int Hq, int Hk, const char *call) {
    if (Hk < 1 || Hk > 1024 || Hq < Hk || Hq > 1024 || Hq % Hk)
        return set_error(MOE_E_ARG, "%s: heads_kv must be 1..1024 and heads_q a multiple of it, at most 1024", call);
    return MOE_OK;
}

int32_t check_cache(const attn_cache *c, const char *call) {
    if (!c || !c->k || !c->v) return set_error(MOE_E_ARG, "%s: the cache or its k or v is null", call);
    if (c->format != ATTN_BF16 && c->format != ATTN_FP8) return set_error(MOE_E_ARG, "%s: unknown cache format", call);
    if (c->format == ATTN_FP8 && (!c->k_scale || !c->v_scale)) return set_error(MOE_E_ARG, "%s: an fp8 cache needs k_scale and v_scale", call);
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || (c->format == ATTN_FP8 && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))))
        return set_error(MOE_E_ARG, "%s: k and v must be 16-byte, scales 4-byte aligned", call);
    if (c->n_pages < 1 || c->heads_kv < 1 || c->heads_kv > 1024) return set_error(MOE_E_ARG, "%s: n_pages must be positive, heads_kv 1..1024", call);
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
        return set_error(MOE_E_ARG, "%s: page_tokens must be 16, 32, 64, 128 or 256", call);
    return check_dim(c->dim, call);
}

qattn::Cache cache_of(const attn_cache *c) {
    return {(uint8_t *)c->k, (uint8_t *)c->v, c->k_scale, c->v_scale, c->n_pages, c->heads_kv, __builtin_ctz((unsigned)c->page_tokens), c->dim};
}

int32_t check_place(const attn_place *p, int n_tokens, const char *call) {
    if (n_tokens < 0) return set_error(MOE_E_ARG, "%s: n_tokens negative", call);
    if (n_tokens == 0) return MOE_OK;             // tensors without elements have no address
    if (!p || !p->pos || !p->pages) return set_error(MOE_E_ARG, "%s: the place or its pos or pages is null", call);
    if (p->n_seqs < 1 || p->seq_pages < 1) return set_error(MOE_E_ARG, "%s: n_seqs and seq_pages must be positive", call);
    return MOE_OK;
}

}  // namespace

extern "C" {

int32_t attn_rope_frequencies(int32_t dims, double base, int32_t scaling, double factor, double trained, double fast, double slow,
                              double *inv_freq, float *mscale) {
    const char *call = "attn_rope_frequencies";
    if (!inv_freq || !mscale) return set_error(MOE_E_ARG, "%s: null argument", call);
    if (dims < 2 || dims > qattn::kMaxDim || dims % 2) return set_error(MOE_E_ARG, "%s: dims must be even, 2..%d", call, qattn::kMaxDim);
    if (scaling < ATTN_SCALE_NONE || scaling > ATTN_SCALE_WAVES) return set_error(MOE_E_ARG, "%s: unknown scaling", call);
    if (!(base > 1.0) || !std::isfinite(base)) return set_error(MOE_E_ARG, "%s: base must be over 1", call);
    if (scaling != ATTN_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return set_error(MOE_E_ARG, "%s: factor must be 1 or more", call);
    if (scaling == ATTN_SCALE_BASE && dims < 4) return set_error(MOE_E_ARG, "%s: scaling the base needs 4 dims or more", call);
    if (scaling >= ATTN_SCALE_RAMP && (!(trained >= 1.0) || !std::isfinite(trained) || !(slow > 0.0) || !(fast > slow) || !std::isfinite(fast)))
        return set_error(MOE_E_ARG, "%s: needs trained >= 1 and fast > slow > 0", call);
    const double two_pi = 6.283185307179586476925286766559;
    if (scaling == ATTN_SCALE_BASE) base *= std::pow(factor, dims / (dims - 2.0));
    // the (fractional) pair that turns `turns` times within the trained positions
    const auto pair_at = [&](double turns) { return dims * std::log(trained / (turns * two_pi)) / (2.0 * std::log(base)); };
    double lo = 0.0, hi = 0.0;
    if (scaling == ATTN_SCALE_RAMP) {
        lo = std::fmax(0.0, std::floor(pair_at(fast)));
        hi = std::fmin(dims - 1.0, std::ceil(pair_at(slow)));
        hi = std::fmax(hi, lo + 1e-3);
    }
    for (int i = 0; i < dims / 2; ++i) {
        double f = std::pow(base, -2.0 * i / dims);
        if (scaling == ATTN_SCALE_LINEAR) {
            f /= factor;
        } else if (scaling == ATTN_SCALE_RAMP) {
            const double r = std::fmin(1.0, std::fmax(0.0, (i - lo) / (hi - lo)));
            f = f * (1.0 - r) + f / factor * r;
        } else if (scaling == ATTN_SCALE_WAVES) {
            const double turns = trained * f / two_pi;     // trained / wavelength
            const double t = std::fmin(1.0, std::fmax(0.0, (turns - slow) / (fast - slow)));
            f = (1.0 - t) * f / factor + t * f;
        }
        inv_freq[i] = f;
    }
    *mscale = scaling == ATTN_SCALE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return MOE_OK;
}

int32_t attn_append(const attn_cache *cache, const attn_rows *q, const attn_rows *k, const attn_rows *v, const attn_rows *q_out,
                    const attn_rows *k_out, int32_t heads_q, int32_t n_tokens, const attn_place *place, const attn_rope *rope,
                    int32_t *bad, void *stream) {
    const char *call = "attn_append";
    int32_t rc;
    if ((rc = check_cache(cache, call)) || (rc = check_place(place, n_tokens, call))) return rc;
    if ((q == nullptr) != (q_out == nullptr) || (q == nullptr) != (heads_q == 0)) return set_error(MOE_E_ARG, "%s: q, q_out and heads_q go together", call);
    if (q && ((rc = check_heads(heads_q, cache->heads_kv, call)))) return rc;
    if (rope && rope->dims != 0) {
        if (!rope->inv_freq) return set_error(MOE_E_ARG, "%s: inv_freq is null", call);
        if (rope->dims < 0 || rope->dims > cache->dim || rope->dims % 16) return set_error(MOE_E_ARG, "%s: rope dims must be a multiple of 16, at most dim", call);
        if (rope->layout != ATTN_ROPE_HALF && rope->layout != ATTN_ROPE_INTERLEAVED) return set_error(MOE_E_ARG, "%s: unknown rope layout", call);
        if (!std::isfinite(rope->mscale)) return set_error(MOE_E_ARG, "%s: mscale is not finite", call);
    }
    if (n_tokens == 0) return MOE_OK;
    if ((q && ((rc = check_rows(q, call, "q")) || (rc = check_rows(q_out, call, "q_out")))) || (rc = check_rows(k, call, "k")) || (rc = check_rows(v, call, "v")) ||
        (k_out && (rc = check_rows(k_out, call, "k_out"))))
        return rc;
    qattn::AppendArgs a{cache_of(cache), rows(q), rows(k), rows(v), rows(q_out), rows(k_out), place->seq, place->pos, place->pages,
                        rope ? rope->inv_freq : nullptr, bad, n_tokens, heads_q, place->n_seqs, place->seq_pages, rope ? rope->dims : 0,
                        rope && rope->layout == ATTN_ROPE_INTERLEAVED, cache->format == ATTN_FP8, rope ? rope->mscale : 1.f};
    return hip_result(qattn::launch_append(a, (hipStream_t)stream), call);
}

int32_t attn_read(const attn_cache *cache, const attn_place *place, int32_t n_tokens, const attn_rows *k_out, const attn_rows *v_out,
                  int32_t *bad, void *stream) {
    const char *call = "attn_read";
    int32_t rc;
    if ((rc = check_cache(cache, call)) || (rc = check_place(place, n_tokens, call))) return rc;
    if (n_tokens == 0) return MOE_OK;
    if ((rc = check_rows(k_out, call, "k_out")) || (rc = check_rows(v_out, call, "v_out"))) return rc;
    qattn::ReadArgs a{cache_of(cache), rows(k_out), rows(v_out), place->seq, place->pos, place->pages, bad, n_tokens, place->n_seqs,
                      place->seq_pages, cache->format == ATTN_FP8};
    return hip_result(qattn::launch_read(a, (hipStream_t)stream), call);
}

size_t attn_prompt_workspace_bytes(int32_t n_seqs, int32_t n_q, int32_t n_k, int32_t heads_q, int32_t heads_kv, int32_t dim) {
    const char *call = "attn_prompt_workspace_bytes";
    if (check_heads(heads_q, heads_kv, call) || check_dim(dim, call) || n_seqs < 1 || n_seqs > 1 << 20 || n_q < 1 || n_q > 1 << 30 || n_k < 1 || n_k > 1 << 30) return 0;
    const int parts = qattn::prompt_parts(n_seqs, n_q, n_k, heads_q, heads_kv, dim);
    return parts > 1 ? (size_t)parts * n_q * heads_q * (dim + 2) * 4 : 0;
}

int32_t attn_prompt(const attn_rows *q, const attn_rows *k, const attn_rows *v, const attn_rows *out, float *lse, const int32_t *cu_q,
                    const int32_t *cu_k, int32_t n_seqs, int32_t n_q, int32_t n_k, int32_t heads_q, int32_t heads_kv, int32_t dim,
                    float scale, int32_t causal, void *workspace, size_t workspace_bytes, void *stream) {
    const char *call = "attn_prompt";
    int32_t rc;
    if ((rc = check_heads(heads_q, heads_kv, call)) || (rc = check_dim(dim, call))) return rc;
    if (n_seqs < 0 || n_q < 0 || n_k < 0) return set_error(MOE_E_ARG, "%s: negative size", call);
    if (n_seqs > 1 << 20) return set_error(MOE_E_ARG, "%s: n_seqs must be at most 2^20", call);
    if (n_q > 1 << 30 || n_k > 1 << 30) return set_error(MOE_E_ARG, "%s: n_q and n_k must be at most 2^30", call);      // rows up to the end of a tile have 32 bits
    if (!(scale > 0.f) || !std::isfinite(scale * kLog2E)) return set_error(MOE_E_ARG, "%s: scale must be positive, and scale * log2(e) finite", call);
    if (n_seqs == 0 || n_q == 0) return MOE_OK;
    if (!cu_q || !cu_k) return set_error(MOE_E_ARG, "%s: cu_q or cu_k is null", call);
    if ((rc = check_rows(q, call, "q")) || (rc = check_rows(out, call, "out"))) return rc;
    if (n_k > 0 && ((rc = check_rows(k, call, "k")) || (rc = check_rows(v, call, "v")))) return rc;
    if (n_k > 0 && (k->token_stride > 1 << 24 || v->token_stride > 1 << 24)) return set_error(MOE_E_ARG, "%s: token strides of k and v must be at most 2^24", call);
    if (workspace && !aligned(workspace, 16)) return set_error(MOE_E_WORKSPACE, "%s: workspace is not 16-byte aligned", call);
    const size_t need = workspace ? attn_prompt_workspace_bytes(n_seqs, n_q, n_k, heads_q, heads_kv, dim) : 0;
    const int parts = need && workspace_bytes >= need ? qattn::prompt_parts(n_seqs, n_q, n_k, heads_q, heads_kv, dim) : 1;
    float *part_o = (float *)workspace, *part_ml = parts > 1 ? part_o + (size_t)parts * n_q * heads_q * dim : nullptr;
    qattn::PromptArgs a{rows(q), n_k ? rows(k) : qattn::Rows{nullptr, 0, 0}, n_k ? rows(v) : qattn::Rows{nullptr, 0, 0}, rows(out), lse,
                        cu_q, cu_k, n_seqs, n_q, n_k, heads_q, heads_kv, dim, causal != 0, scale * kLog2E, qattn::prompt_log_tile(n_seqs, n_q, heads_q, heads_kv, parts), parts, qattn::prompt_slots(dim), part_o, part_ml};
    return hip_result(qattn::launch_prompt(a, (hipStream_t)stream), call);
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// A decode workspace: the arrival counters, then the pieces' sums.  Where the sums begin follows from the workspace's size alone, a 256th of it behind its start: by a
// call's own counters they would begin where another call, of more sequences or heads, has its own, which every call must find zero.  A 256th is more than any
// call's counters: a head of a sequence has 4 bytes of them and 16 * 18 * 4 bytes of sums at least.
static size_t counter_room(size_t workspace_bytes) { return up256(workspace_bytes / 256); }
static size_t sums_bytes(int n_seqs, int Hq, int Hk, int dim) {
    return up256((size_t)qattn::decode_pieces(n_seqs, Hq, Hk) * Hk * qattn::group_tiles(Hq, Hk) * 16 * (dim + 2) * 4);
}
static bool decode_shape_ok(int n_seqs, int Hq, int Hk) { return n_seqs >= 0 && n_seqs <= 65535 && Hk >= 1 && Hk <= 1024 && Hq >= Hk && Hq <= 1024 && Hq % Hk == 0; }

size_t attn_decode_counter_bytes(int32_t n_seqs, int32_t heads_q, int32_t heads_kv) {
    if (!decode_shape_ok(n_seqs, heads_q, heads_kv)) {
        set_error(MOE_E_ARG, "attn_decode_counter_bytes: n_seqs must be 0..65535, heads_kv 1..1024, heads_q a multiple of it, at most 1024");
        return 0;
    }
    return up256((size_t)(n_seqs ? n_seqs : 1) * heads_kv * qattn::group_tiles(heads_q, heads_kv) * 4);
}

size_t attn_decode_workspace_bytes(int32_t n_seqs, int32_t heads_q, int32_t heads_kv, int32_t dim) {
    if (!attn_decode_counter_bytes(n_seqs, heads_q, heads_kv) || check_dim(dim, "attn_decode_workspace_bytes")) return 0;
    const size_t sums = sums_bytes(n_seqs, heads_q, heads_kv, dim);
    return sums + up256((sums + 254) / 255);      // the least n with n - counter_room(n) >= sums
}

int32_t attn_decode(const attn_cache *cache, const attn_rows *q, const attn_rows *out, float *lse, int32_t n_seqs, int32_t heads_q,
                    const int32_t *pages, int32_t seq_pages, const int32_t *lens, float scale, void *workspace, size_t workspace_bytes,
                    int32_t *bad, void *stream) {
    const char *call = "attn_decode";
    int32_t rc;
    if ((rc = check_cache(cache, call)) || (rc = check_heads(heads_q, cache->heads_kv, call))) return rc;
    if (n_seqs < 0 || n_seqs > 65535) return set_error(MOE_E_ARG, "%s: n_seqs must be 0..65535", call);
    if (n_seqs == 0) return MOE_OK;
    if (seq_pages < 1 || (int64_t)seq_pages * cache->page_tokens >= (int64_t)1 << 30) return set_error(MOE_E_ARG, "%s: seq_pages must be positive, and seq_pages * page_tokens below 2^30", call);
    if ((int64_t)n_seqs * seq_pages * cache->page_tokens >= (int64_t)1 << 38) return set_error(MOE_E_ARG, "%s: n_seqs * seq_pages * page_tokens must be below 2^38", call);
    if (!(scale > 0.f) || !std::isfinite(scale * kLog2E)) return set_error(MOE_E_ARG, "%s: scale must be positive, and scale * log2(e) finite", call);
    if (!pages || !lens) return set_error(MOE_E_ARG, "%s: pages or lens is null", call);
    if ((rc = check_rows(q, call, "q")) || (rc = check_rows(out, call, "out"))) return rc;
    const size_t need = attn_decode_workspace_bytes(n_seqs, heads_q, cache->heads_kv, cache->dim);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return set_error(MOE_E_WORKSPACE, "%s: workspace too small or not 256-byte aligned (%zu bytes needed)", call, need);
    uint8_t *w = (uint8_t *)workspace;
    const int64_t most = (int64_t)n_seqs * std::max<int64_t>(1, ((int64_t)seq_pages * cache->page_tokens + 255) / 256);      // a piece has 256 keys at least
    const int pieces = (int)std::min<int64_t>(most, qattn::decode_pieces(n_seqs, heads_q, cache->heads_kv));
    qattn::DecodeArgs a{cache_of(cache), rows(q), rows(out), lse, pages, lens, bad, (int32_t *)w,
                        (float *)(w + counter_room(workspace_bytes)), n_seqs, heads_q, seq_pages,
                        cache->format == ATTN_FP8, pieces, scale * kLog2E};
    return hip_result(qattn::launch_decode(a, (hipStream_t)stream), call);
}

}  // extern "C"
