// attn_prompt: attention over packed prompts, causal or not, heads grouped over shared keys.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup has 4 waves; a wave owns 32 * QB queries of one
// head and goes through the keys 64 at a time:
//     S^T[key, q] = K Q^T     v_mfma_f32_32x32x16_bf16, A = 32 keys x 16 d, B = 16 d x 32 queries
//     O^T[d, q]   = V^T P^T   A = 32 d x 16 keys,  B = 16 keys x 32 queries
// Transposed like this a lane holds 16 keys of one query per tile, so the maximum and the sum of a row are formed inside the lane (one
// exchange with lane ^ 32 at the end), and the weights are the second product's B operand as they stand: slot 8h + j of it
// (h = lane / 32) is key 8 (j / 4) + 4h + j % 4 of the 16, and V^T is read in that order.
// K and V tiles are staged in LDS, double-buffered, through registers (the loads of the next tile are in flight while one is worked on),
// their 16-byte pieces XOR-swizzled by row.  K rows are read as they are, V^T by ds_read_b64_tr_b16.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_pieces.h"
#include "qattn_internal.h"

namespace qattn {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kKeys = 64;                         // keys of a tile

__device__ __forceinline__ f32x16 mma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float other_half_max(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
// 4 keys of one d: lane i of 16 gets element i of the 4 rows that lanes 4r .. 4r + 3 point at, 8 bytes each.
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
__device__ __forceinline__ u32x2 read_transposed(const uint16_t *p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
}

// Slots of 16 bytes: piece c of row r of a tile stands at c ^ swz(r).
template <int DP>
__device__ __forceinline__ int swz_k(int r) { return DP == 128 ? (r & 15) : (r & 7); }
template <int DP>
__device__ __forceinline__ int swz_v(int r) { return DP == 128 ? 2 * (r & 7) : 2 * (r & 3); }

// An entry of cu, held to 0..n and to what the entry before it allows.
__device__ __forceinline__ int2 span(const int32_t *cu, int b, int n) {
    const int lo = min(max(cu[b], 0), n);
    return {lo, min(max(cu[b + 1], lo), n)};
}

template <int DP, int QB>
__global__ __launch_bounds__(kWaves * 64) void prompt_tile(const PromptArgs a, int tiles, int item0) {
    constexpr int QT = kWaves * 32 * QB;          // queries of a workgroup
    constexpr int CH = DP / 8;                    // 16-byte pieces of a row
    constexpr int KS = DP / 16;                   // MFMA steps of a score
    constexpr int DT = DP / 32;                   // 32-d tiles of the output
    constexpr int LD = kKeys * CH / (kWaves * 64);   // pieces of K (and V) that a thread moves per tile
    __shared__ __attribute__((aligned(16))) uint16_t s_k[2][kKeys * DP];
    __shared__ __attribute__((aligned(16))) uint16_t s_v[2][kKeys * DP];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, col = lane & 31;
    // Neighbouring workgroups run on different XCDs: those of one key/value head are Hk apart, so with 8 such heads
    // each XCD's L2 holds the keys of one.  Late tiles of a sequence see the most keys: they start first.
    const int G = a.Hq / a.Hk, num = blockIdx.x + item0;
    const int hk = num % a.Hk, rest = num / a.Hk, head = hk * G + rest % G, item = tiles - 1 - rest / G;
    const Piece at = find_piece(a.n_seqs, (uint32_t)item, [&](int b) { const int2 s = span(a.cu_q, b, a.n_q); return s.y - s.x; },
                                [](int n) { return (uint32_t)(n + QT - 1) / QT; });
    const int b = at.seq;
    if (b < 0) return;
    const int2 sq = span(a.cu_q, b, a.n_q), sk = span(a.cu_k, b, a.n_k);
    const int nq = __builtin_amdgcn_readfirstlane(sq.y - sq.x), nk = __builtin_amdgcn_readfirstlane(sk.y - sk.x);
    const int r0 = at.piece * QT;                 // first query of the tile, within the sequence
    const long q_row = __builtin_amdgcn_readfirstlane(sq.x), k_row = __builtin_amdgcn_readfirstlane(sk.x);
    const int w0 = r0 + wave * 32 * QB;                                        // first query of the wave
    // keys that the tile's last query sees, and those that all queries of the wave see / any of them sees
    const int shift = nk - nq;
    const int tile_keys = a.causal ? min(nk, max(0, shift + min(nq, r0 + QT))) : nk;
    const int wave_all = a.causal ? max(0, shift + w0 + 1) : nk;
    const int wave_any = w0 >= nq ? 0 : a.causal ? min(nk, max(0, shift + min(nq, w0 + 32 * QB))) : nk;
    const int n_tiles = (tile_keys + kKeys - 1) / kKeys;

    u32x4 qf[QB][KS];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int r = w0 + 32 * i + col;
        const uint16_t *p = a.q.p + (q_row + min(r, nq - 1)) * a.q.ts + (long)head * a.q.hs;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[i][s] = 16 * s < a.D ? *reinterpret_cast<const u32x4 *>(p + 16 * s + 8 * h) : u32x4{0, 0, 0, 0};
    }
    f32x16 o[QB][DT];
    float m[QB], l[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][d][r] = 0.f;
    }

    // the pieces that this thread moves: rows tr + i * (256 / CH), piece tc
    const int tr = tid / CH, tc = tid % CH;
    const uint16_t *kp = a.k.p + k_row * a.k.ts + (long)hk * a.k.hs + tc * 8;
    const uint16_t *vp = a.v.p + k_row * a.v.ts + (long)hk * a.v.hs + tc * 8;
    const bool has_d = tc * 8 < a.D;
    u32x4 kr[LD], vr[LD];
    const auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            const int key = t * kKeys + tr + i * (kWaves * 64 / CH);
            const bool in = has_d && key < nk;
            kr[i] = in ? *reinterpret_cast<const u32x4 *>(kp + (long)key * a.k.ts) : u32x4{0, 0, 0, 0};
            vr[i] = in ? *reinterpret_cast<const u32x4 *>(vp + (long)key * a.v.ts) : u32x4{0, 0, 0, 0};
        }
    };
    const auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            const int r = tr + i * (kWaves * 64 / CH);
            *reinterpret_cast<u32x4 *>(&s_k[buf][r * DP + (tc ^ swz_k<DP>(r)) * 8]) = kr[i];
            *reinterpret_cast<u32x4 *>(&s_v[buf][r * DP + (tc ^ swz_v<DP>(r)) * 8]) = vr[i];
        }
    };

    if (n_tiles > 0) {
        fetch(0);
        store(0);
    }
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int buf = t & 1;
        if (t + 1 < n_tiles) fetch(t + 1);
        if (t * kKeys < wave_any) {
            f32x16 s[QB][2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int i = 0; i < QB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[i][n][r] = 0.f;
                const int row = 32 * n + col;
#pragma unroll
                for (int st = 0; st < KS; ++st) {
                    const u32x4 kf = *reinterpret_cast<const u32x4 *>(&s_k[buf][row * DP + ((2 * st + h) ^ swz_k<DP>(row)) * 8]);
#pragma unroll
                    for (int i = 0; i < QB; ++i) s[i][n] = mma(kf, qf[i][st], s[i][n]);
                }
            }
            if ((t + 1) * kKeys > wave_all || (t + 1) * kKeys > nk) {
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    const int last = min(nk - 1, a.causal ? shift + w0 + 32 * i + col : nk - 1) - t * kKeys;      // last key of the query, in the tile
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (32 * n + 8 * (r / 4) + 4 * h + r % 4 > last) s[i][n][r] = -INFINITY;
                }
            }
            u32x4 pf[QB][4];
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                float top = s[i][0][0];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][n][r]);
                top = other_half_max(top);
                // The sums may stand relative to any value: they are taken over to a new maximum only where it is 2^8 above the old.
                if (__any((top - m[i]) * a.scale_log2 > 8.f)) {
                    const float next = fmaxf(m[i], top), f = __builtin_amdgcn_exp2f((m[i] - (next == -INFINITY ? 0.f : next)) * a.scale_log2);
                    m[i] = next;
                    l[i] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[i][d][r] *= f;
                }
                const float base = (m[i] == -INFINITY ? 0.f : m[i]) * a.scale_log2;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[i][n][r] = __builtin_amdgcn_exp2f(fmaf(s[i][n][r], a.scale_log2, -base));
                        l[i] += s[i][n][r];
                    }
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) pf[i][c][j] = pack_bf16(s[i][c / 2][8 * (c & 1) + 2 * j], s[i][c / 2][8 * (c & 1) + 2 * j + 1]);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int row = 16 * c + 4 * h + (lane & 15) / 4;
                    const int piece = 4 * d + 2 * ((lane >> 4) & 1) + (lane & 3) / 2, at8 = (lane & 1) * 4;
                    const u32x2 v0 = read_transposed(&s_v[buf][row * DP + (piece ^ swz_v<DP>(row)) * 8 + at8]);
                    const u32x2 v1 = read_transposed(&s_v[buf][(row + 8) * DP + (piece ^ swz_v<DP>(row + 8)) * 8 + at8]);
                    const u32x4 vf = {v0[0], v0[1], v1[0], v1[1]};
#pragma unroll
                    for (int i = 0; i < QB; ++i) o[i][d] = mma(vf, pf[i][c], o[i][d]);
                }
        }
        if (t + 1 < n_tiles) store(buf ^ 1);
        __syncthreads();
    }

#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const float sum = other_half_sum(l[i]), inv = sum > 0.f ? 1.f / sum : 0.f;
        const int r = w0 + 32 * i + col;
        if (r >= nq) continue;
        uint16_t *to = a.o.p + (q_row + r) * a.o.ts + (long)head * a.o.hs;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = 32 * d + 8 * j + 4 * h;
                const u32x2 x = {pack_bf16(o[i][d][4 * j] * inv, o[i][d][4 * j + 1] * inv), pack_bf16(o[i][d][4 * j + 2] * inv, o[i][d][4 * j + 3] * inv)};
                if (e < a.D) *reinterpret_cast<u32x2 *>(to + e) = x;
            }
        if (a.lse != nullptr && h == 0)
            a.lse[(q_row + r) * a.Hq + head] = sum > 0.f ? (m[i] * a.scale_log2 + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    }
}

template <int DP, int QB>
void prompt_n(const PromptArgs &a, hipStream_t s) {
    const long tiles = (a.n_q + (long)kWaves * 32 * QB - 1) / (kWaves * 32 * QB) + a.n_seqs, all = tiles * a.Hq;
    // a launch of 2^32 threads or more would lose the excess
    for (long at = 0; at < all; at += 1 << 23)
        prompt_tile<DP, QB><<<dim3((unsigned)std::min<long>(all - at, 1 << 23)), dim3(kWaves * 64), 0, s>>>(a, (int)tiles, (int)at);
}

}  // namespace

hipError_t launch_prompt(const PromptArgs &a, hipStream_t s) {
    if (a.D <= 64) prompt_n<64, 1>(a, s);
    else prompt_n<128, 1>(a, s);
    return hipGetLastError();
}

}  // namespace qattn
