// Internal declarations shared by the host side of the attention calls and their kernels (the public ABI is include/qattn.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qattn.h"

namespace qattn {

constexpr int kMaxDim = 128;

// Workgroups that a call's kernels are launched with: launch(first, n) for runs of all of them, in order.  A launch of 2^32 threads or more would lose the
// excess; 2^23 workgroups of 256 are half that.
constexpr long kMostLaunched = 1 << 23;
template <class F>
inline void in_launches(long all, F &&launch) {
    for (long at = 0; at < all; at += kMostLaunched) launch((int)at, (unsigned)(all - at < kMostLaunched ? all - at : kMostLaunched));
}

// Rows of heads as the kernels take them (bf16 elements).
struct Rows {
    uint16_t *p;
    long ts, hs;
};

// A cache as the kernels take it.
struct Cache {
    uint8_t *k, *v;               // bf16 or e4m3
    uint8_t *ks, *vs;             // scale bytes (e4m3)
    int n_pages, Hk, page_shift, D;
};

struct AppendArgs {
    Cache c;
    Rows q, k, v, qo, ko;         // q.p, qo.p, ko.p may be nullptr
    const int32_t *seq, *pos, *pages;
    const double *inv_freq;
    int32_t *bad;
    int n_tokens, Hq, n_seqs, seq_pages, rot, interleaved, fp8;
    float mscale;
};
hipError_t launch_append(const AppendArgs &a, hipStream_t s);

struct ReadArgs {
    Cache c;
    Rows ko, vo;
    const int32_t *seq, *pos, *pages;
    int32_t *bad;
    int n_tokens, n_seqs, seq_pages, fp8;
};
hipError_t launch_read(const ReadArgs &a, hipStream_t s);

struct PromptArgs {
    Rows q, k, v, o;
    float *lse;
    const int32_t *cu_q, *cu_k;
    int n_seqs, n_q, n_k, Hq, Hk, D, causal;
    float scale_log2;             // scale * log2(e)
    int log_tile;                 // of the queries that a workgroup has of a head
    int parts, slots;             // most parts of a query's keys; workgroups that the chip holds
    float *part_o;                // [part][n_q][Hq][D] sums, with parts > 1
    float *part_ml;               // [part][n_q][Hq][2] what they are relative to, in powers of two, and the sums of the weights
};
// Tiles and parts for a call: see attn_prompt.hip.
int prompt_slots(int D);
int prompt_log_tile(int n_seqs, int n_q, int Hq, int Hk, int parts);
int prompt_parts(int n_seqs, int n_q, int n_k, int Hq, int Hk, int D);
hipError_t launch_prompt(const PromptArgs &a, hipStream_t s);

struct DecodeArgs {
    Cache c;
    Rows q, o;
    float *lse;
    const int32_t *pages, *lens;
    int32_t *bad;
    int32_t *arrived;             // [n_seqs][Hk * group tiles], zero between calls
    float *part;                  // pieces: [piece][16][D + 2] fp32
    int n_seqs, Hq, seq_pages, fp8;
    int pieces;                   // most pieces of all sequences per (key/value head, group tile): the grid
    float scale_log2;
};
// A group tile is up to 16 query heads that share a key/value head.
__host__ __device__ inline int group_tiles(int Hq, int Hk) { return (Hq / Hk + 15) / 16; }
// Workgroups that a decode launch cuts the keys into, before the pieces of each sequence are rounded up: see attn_decode.hip.
constexpr int kFewestWgs = 256, kMostWgs = 1536;
// Most pieces of all sequences, per (key/value head, group tile): workgroups, and places in the workspace.  Ranges are 512 / heads workgroups, rounded up, with two
// places each.
inline int decode_pieces(int n_seqs, int Hq, int Hk) {
    const int heads = Hk * group_tiles(Hq, Hk);
    return n_seqs + (kMostWgs + heads - 1) / heads;
}
inline long decode_workgroups(const DecodeArgs &a) { return (long)a.pieces * a.c.Hk * group_tiles(a.Hq, a.c.Hk); }
hipError_t launch_decode(const DecodeArgs &a, hipStream_t s);

}  // namespace qattn
