/*
 * qattn — the attention block between two MoE layers of a served model, on AMD MI355X (gfx950).
 *
 * The serving system around the layer of qmoe.h runs two kinds of iterations (QLLM, arXiv 2503.09304, Sec. 2.1 and 3.2):
 * prefill, all tokens of a batch of prompts at once, and decode, one token a sequence on the keys and values kept from before.
 * Per layer that is
 *
 *     prefill:  attn_append -> attn_prompt          (a prompt's next chunk: attn_append -> attn_read -> attn_prompt)
 *     decode:   attn_append -> attn_decode
 *
 * between the projections to q, k, v and the output projection, which are plain matrix products and the caller's.
 *
 * Conventions that hold for every call
 *  - Pointers marked [device] are GPU global memory owned by the caller; the library allocates nothing, creates no stream, keeps
 *    no state between calls and never waits: calls enqueue on `stream` (a hipStream_t as void*, NULL = the default stream) and
 *    return, so they can be captured into a graph.  The current device is that of the pointers and of the stream.
 *  - Return value: MOE_OK or a negative moe_status (qmoe.h), with the text in moe_last_error().  On an error nothing was enqueued
 *    (MOE_E_HIP excepted).
 *  - Queries, keys, values and outputs are bfloat16.  Products are summed in fp32, the softmax is in fp32, its weights are
 *    rounded to bf16 once (they are a matrix operand), outputs are rounded to bf16 once.
 *  - Heads: query head h reads key/value head h / (heads_q / heads_kv).  A head has dim elements, a multiple of 16 from 16 to 128.
 *  - A call's results are the same bits every time.  A sequence's may differ in the last bits with the others of its call: in how many places its keys are
 *    cut, and so the order of its sums, goes by all lengths of the call (attn_decode, and attn_prompt with a workspace).  attn_prompt without a workspace
 *    cuts nothing: there a sequence's bits are the same whatever stands beside it.
 *  - Calls of no tokens (queries, sequences) do nothing and look at no pointer of theirs but the cache's.
 *  - Tokens that take part are assumed finite.  (A value that is not reaches, in a causal prompt, also queries of its sequence that stand
 *    fewer than 128 tokens before it: their weight for it is 0, and 0 times it is NaN.)  What lies beside them (slots of a page that
 *    no token was written to, rows between strides) may hold anything, NaN included, and reaches no output.
 *  - Numbers on the device (seq, pos, pages, lens, cu) cannot be checked by the host.  The kernels check them: what they do with
 *    one that is out of range is said at each call; nothing is read or written out of bounds, and *bad ([device] int32, may be NULL),
 *    which the caller has set to 0, counts them.
 */
#ifndef QATTN_H
#define QATTN_H

#include "qmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of heads: element d of head h of token t is data[t * token_stride + h * head_stride + d].  Strides in elements, multiples
 * of 8 and not negative; data 16-byte aligned.  So q, k and v may be slices of the rows of one product, or, with a stride of 0, one row
 * for all tokens or heads; the rows of an output are apart. */
typedef struct {
    void *data; /* [device] bf16 */
    int64_t token_stride;
    int64_t head_stride;
} attn_rows;

/* A cache of keys and values in pages.  Elements of one head in one page are dense:
 *     k, v              [n_pages, heads_kv, page_tokens, dim]
 *     k_scale, v_scale  [n_pages, heads_kv, page_tokens]       ATTN_FP8 only, else NULL
 * ATTN_BF16: bfloat16.  ATTN_FP8: e4m3 (OCP: largest 448), and for each token and head one scale byte e8m0 (2^(byte-127), as in the
 * 4-bit weights of qmoe.h): value = element * scale.  The scale is the smallest power of two, 2^-126 at least, for which no
 * element is over 448, so writing rounds each bf16 element once, to 4 significant bits and no finer than 2^-9 of the scale (one that would round to
 * 2^128 to 1.875 * 2^127), and a value read back is exactly a bf16, those below 2^-126 among them.
 * page_tokens: 16, 32, 64, 128 or 256.  k and v 16-byte aligned, scales 4-byte aligned. */
enum { ATTN_BF16 = 0, ATTN_FP8 = 1 };
typedef struct {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    int32_t n_pages, heads_kv, page_tokens, dim;
    int32_t format;
} attn_cache;

/* Where tokens stand: token t is at position pos[t] (from 0) of sequence seq[t] (seq NULL: of sequence t), that is in slot
 * pos % page_tokens of page pages[seq * seq_pages + pos / page_tokens].  A position below 0 marks a row of padding. */
typedef struct {
    const int32_t *seq;   /* [device] [n_tokens] or NULL      */
    const int32_t *pos;   /* [device] [n_tokens]              */
    const int32_t *pages; /* [device] [n_seqs, seq_pages]     */
    int32_t n_seqs, seq_pages;
} attn_place;

/* Rotary positions.  dims (a multiple of 16, 0..dim; 0 = none) elements of each head are rotated in pairs, pair i by the angle
 * pos * inv_freq[i]; the elements behind them stay.  ATTN_ROPE_HALF pairs (i, i + dims/2), ATTN_ROPE_INTERLEAVED (2i, 2i + 1).
 *     (a, b) -> (a c - b s, b c + a s),   c = mscale cos(angle), s = mscale sin(angle)
 * Angles are formed and reduced in 64 bits, so far positions keep their full precision. */
enum { ATTN_ROPE_HALF = 0, ATTN_ROPE_INTERLEAVED = 1 };
typedef struct {
    const double *inv_freq; /* [device] [dims/2]; see attn_rope_frequencies */
    int32_t dims, layout;
    float mscale;
} attn_rope;

/* Frequencies for attn_rope, on the host (no GPU is touched): dims/2 doubles into inv_freq ([host]), the factor on cos and sin into
 * *mscale ([host]).  With f_i = base^(-2i/dims):
 *   ATTN_SCALE_NONE    f_i                                                                                      mscale 1
 *   ATTN_SCALE_LINEAR  f_i / factor: positions squeezed into the trained range                                  mscale 1
 *   ATTN_SCALE_BASE    base * factor^(dims/(dims-2)) in place of base: the lowest frequency is divided by factor  mscale 1
 *   ATTN_SCALE_RAMP    (1 - r_i) f_i + r_i f_i / factor with r_i = clamp((i - lo) / (hi - lo), 0, 1), where pair `lo` (rounded down)
 *                      turns `fast` times and `hi` (rounded up) `slow` times within trained positions        mscale 0.1 ln factor + 1
 *   ATTN_SCALE_WAVES   by wavelength w = 2 pi / f_i: f_i where w < trained/fast, f_i / factor where w > trained/slow, between them
 *                      (1 - t) f_i / factor + t f_i with t = (trained/w - slow) / (fast - slow)                 mscale 1
 * dims even, 2..128 (BASE: 4 at least); base > 1, factor >= 1; RAMP and WAVES: trained >= 1, fast > slow > 0. */
enum { ATTN_SCALE_NONE = 0, ATTN_SCALE_LINEAR = 1, ATTN_SCALE_BASE = 2, ATTN_SCALE_RAMP = 3, ATTN_SCALE_WAVES = 4 };
int32_t attn_rope_frequencies(int32_t dims, double base, int32_t scaling, double factor, double trained, double fast, double slow,
                              double *inv_freq, float *mscale);

/* Rotates the queries and keys of n_tokens tokens and writes keys and values to the cache.  q [heads_q heads] -> q_out, k -> k_out
 * and cache, v -> cache; q_out and k_out are rounded to bf16 once, and the cache takes the rounded keys.  q and q_out may be NULL
 * (both, with heads_q 0), k_out may be NULL; q_out may be q and k_out may be k, otherwise outputs overlap no input.
 * A row of padding writes nothing.  A token whose sequence, page index or page is out of range is counted in *bad and not written
 * to the cache; its q_out and k_out are.  Tokens of a call have slots of their own: what a slot that two of them name holds afterwards is not
 * specified (it may be parts of both, or the elements of one under the scale of the other). */
int32_t attn_append(const attn_cache *cache, const attn_rows *q, const attn_rows *k, const attn_rows *v, const attn_rows *q_out,
                    const attn_rows *k_out, int32_t heads_q, int32_t n_tokens, const attn_place *place, const attn_rope *rope,
                    int32_t *bad, void *stream);

/* Keys and values of n_tokens tokens out of the cache, as bf16 (exactly what the cache holds).  Rows of padding, and tokens out of
 * range (counted in *bad), give zeros. */
int32_t attn_read(const attn_cache *cache, const attn_place *place, int32_t n_tokens, const attn_rows *k_out, const attn_rows *v_out,
                  int32_t *bad, void *stream);

/* Attention over whole prompts, packed: sequence b has queries cu_q[b] .. cu_q[b+1] - 1 out of n_q and keys cu_k[b] .. cu_k[b+1] - 1
 * out of n_k (cu [device] int32 [n_seqs + 1], ascending).  Its queries are its last tokens: with nq queries and nk keys, query i
 * sees keys 0 .. nk - nq + i (causal != 0) or all of them.
 *     out_i = sum_j p_ij v_j,   p_ij = exp(scale q_i.k_j) / sum_j' exp(scale q_i.k_j')
 * A query that sees no key gives zeros.  lse ([device] float [n_q, heads_q], may be NULL): ln of the sum of the exponentials,
 * -inf for a query without keys.  Rows of out that belong to no sequence are left untouched.  Entries of cu out of 0..n_q (n_k) or
 * descending are clamped to the range and to the entry before them.  scale > 0, at most 2^127.  out overlaps no input.  Token strides of k and v: at
 * most 2^24; n_seqs: at most 2^20; n_q and n_k: at most 2^30.
 * workspace ([device], 16-byte aligned, may be NULL; its contents before and after the call are of no account): where queries are so few that
 * they leave CUs idle, the keys of a query are cut into parts that run side by side, and a second launch joins them.
 * attn_prompt_workspace_bytes(...) is what that takes, 0 where nothing is cut; with less than that nothing is cut either. */
size_t attn_prompt_workspace_bytes(int32_t n_seqs, int32_t n_q, int32_t n_k, int32_t heads_q, int32_t heads_kv, int32_t dim);
int32_t attn_prompt(const attn_rows *q, const attn_rows *k, const attn_rows *v, const attn_rows *out, float *lse, const int32_t *cu_q,
                    const int32_t *cu_k, int32_t n_seqs, int32_t n_q, int32_t n_k, int32_t heads_q, int32_t heads_kv, int32_t dim,
                    float scale, int32_t causal, void *workspace, size_t workspace_bytes, void *stream);

/* Attention of one query a sequence over the cache: query b sees the first lens[b] tokens of sequence b (lens [device] int32
 * [n_seqs]), whose pages are pages[b * seq_pages ..].  The formula, lse ([device] float [n_seqs, heads_q], may be NULL) and the answer
 * without keys are those of attn_prompt.  lens out of 0 .. seq_pages * page_tokens are clamped, pages out of 0 .. n_pages - 1 hold no
 * keys; *bad counts each of both once.  n_seqs at most 65535, seq_pages * page_tokens below 2^30, n_seqs times that below 2^38.
 * Long sequences are cut into pieces that run side by side; the last piece of a sequence to finish joins them, in the order of the
 * pieces, so results do not depend on timing.  workspace [device], 256-byte aligned, attn_decode_workspace_bytes(...) long or longer: its first
 * attn_decode_counter_bytes(...) bytes have to be zero at the first call; every call leaves them zero.  Calls of different numbers of
 * sequences, heads and dim may share a workspace that is large enough for each of them, zeroed for the one with the most counter bytes, if all of them
 * state the same workspace_bytes (the place of the sums follows from it).  They are ordered by the caller (one stream, for instance). */
size_t attn_decode_workspace_bytes(int32_t n_seqs, int32_t heads_q, int32_t heads_kv, int32_t dim);
size_t attn_decode_counter_bytes(int32_t n_seqs, int32_t heads_q, int32_t heads_kv);
int32_t attn_decode(const attn_cache *cache, const attn_rows *q, const attn_rows *out, float *lse, int32_t n_seqs, int32_t heads_q,
                    const int32_t *pages, int32_t seq_pages, const int32_t *lens, float scale, void *workspace, size_t workspace_bytes,
                    int32_t *bad, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QATTN_H */
