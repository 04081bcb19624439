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
#include <type_traits>
#include <utility>

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
__device__ __forceinline__ f32x16 zero16() { return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ float other_half_max(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F &&f) {
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}
#ifndef NPRE
#define NPRE 4
#endif
#ifndef NVAL
#define NVAL 80
#endif
#ifndef SCHED
#define SCHED 1
#endif
// An offset of 32 bits that is widened where it is used: widened in front of the loop it would become part of a 64-bit address in vector registers.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}
// 4 keys of one d: lane i of 16 gets element i of the 4 rows that lanes 4r .. 4r + 3 point at, 8 bytes each.
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
__device__ __forceinline__ u32x2 read_transposed(const uint8_t *p) {
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
__global__ __launch_bounds__(kWaves * 64, DP * QB > 128 ? 1 : 2) void prompt_tile(const PromptArgs a, int tiles, int item0) {
    constexpr int QT = kWaves * 32 * QB;          // queries of a workgroup
    constexpr int CH = DP / 8;                    // 16-byte pieces of a row
    constexpr int KS = DP / 16;                   // MFMA steps of a score
    constexpr int DT = DP / 32;                   // 32-d tiles of the output
    constexpr int LD = kKeys * CH / (kWaves * 64);   // pieces of K (and V) that a thread moves per tile
    constexpr int ROW = DP * 2, TILE = kKeys * ROW, VT = 2 * TILE;       // bytes
    __shared__ __attribute__((aligned(16))) uint8_t s_kv[4 * TILE];      // two tiles of K, two of V

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
    // tiles of keys that the tile's last query sees, and those that its first query sees whole
    const int shift = nk - nq;
    const int n_tiles = ((a.causal ? min(nk, max(0, shift + min(nq, r0 + QT))) : nk) + kKeys - 1) / kKeys;
    const int whole_tiles = min(nk, a.causal ? max(0, shift + r0 + 1) : nk) / kKeys;

    u32x4 qf[QB][KS];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int r = w0 + 32 * i + col;
        const uint16_t *p = a.q.p + (q_row + min(r, nq - 1)) * a.q.ts + (long)head * a.q.hs;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[i][s] = *reinterpret_cast<const u32x4 *>(p + min(16 * s, a.D - 16) + 8 * h);
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (16 * s >= a.D) qf[i][s] = u32x4{0, 0, 0, 0};
    }
    f32x16 o[QB][DT];
    float m[QB], l[QB];                           // what a row's sums are relative to, the sum of its weights (of the lane's half of the keys)
    float base[QB], limit[QB];                    // m in powers of two, 0 before there is one; the largest score that needs no other m
    const float slack = 8.f / a.scale_log2;
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        m[i] = limit[i] = -INFINITY;
        base[i] = 0.f;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[i][d] = zero16();
    }

    // The 16-byte pieces that this thread moves: rows tr + i * (256 / CH) of a tile, piece tc.  Rows behind the last key are that key again
    // (their weights are 0), pieces behind the end of a head its last one (the queries are 0 there, those outputs are not stored).
    const int tr = tid / CH, tc = tid % CH, dc = min(tc * 8, a.D - 8);
    const uint16_t *kp = a.k.p + k_row * a.k.ts + (long)hk * a.k.hs;
    const uint16_t *vp = a.v.p + k_row * a.v.ts + (long)hk * a.v.hs;
    u32x4 moved[LD];
    uint32_t kat[LD], vat[LD];                    // bytes from the tile's first row
    const auto rows_at = [&](uint32_t (&at)[LD], long stride, int t) {
#pragma unroll
        for (int i = 0; i < LD; ++i) at[i] = 2u * (uint32_t)(max(0, min(tr + i * (kWaves * 64 / CH), nk - 1 - t * kKeys)) * (int)stride + dc);
    };
    const auto fetch = [&](const uint16_t *p, const uint32_t (&at)[LD], long stride, int t) {
        const char *tile = (const char *)(p + min(t, (nk - 1) / kKeys) * kKeys * stride);
#pragma unroll
        for (int i = 0; i < LD; ++i) moved[i] = *reinterpret_cast<const u32x4 *>(tile + here(at[i]));
    };
    // Places in LDS (bytes; 16-byte pieces are XOR-swizzled by row, in the same way for rows that are 16 apart (K), 8 apart (V)), so that what is
    // read and written differs from these by constants.
    int k_to, v_to, k_from[KS], v_from[DT];
    k_to = tr * ROW + (tc ^ swz_k<DP>(tr)) * 16;
    v_to = VT + tr * ROW + (tc ^ swz_v<DP>(tr)) * 16;
#pragma unroll
    for (int st = 0; st < KS; ++st) k_from[st] = col * ROW + ((2 * st + h) ^ swz_k<DP>(col)) * 16;
    const int v_row = 4 * h + (lane & 15) / 4;
#pragma unroll
    for (int d = 0; d < DT; ++d) v_from[d] = VT + v_row * ROW + ((4 * d + 2 * ((lane >> 4) & 1) + (lane & 3) / 2) ^ swz_v<DP>(v_row)) * 16 + (lane & 1) * 8;
    const auto store = [&](int to) {
#pragma unroll
        for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4 *>(&s_kv[to + i * (kWaves * 64 / CH) * ROW]) = moved[i];
    };
    // Scores of keys 32 n .. of a tile.
    const auto scores = [&](f32x16 (&s)[QB], auto n) {
#pragma unroll
        for (int i = 0; i < QB; ++i) s[i] = zero16();
#pragma unroll
        for (int st = 0; st < KS; ++st) {
            const u32x4 kf = *reinterpret_cast<const u32x4 *>(&s_kv[k_from[st] + 32 * n * ROW]);
#pragma unroll
            for (int i = 0; i < QB; ++i) s[i] = mma(kf, qf[i][st], s[i]);
        }
    };
    // o += V^T P^T for keys 32 n .. of a tile.
    const auto values = [&](const u32x4 (&p)[QB][2], auto n) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const u32x2 v0 = read_transposed(&s_kv[v_from[d] + (32 * n + 16 * c) * ROW]);
                const u32x2 v1 = read_transposed(&s_kv[v_from[d] + (32 * n + 16 * c + 8) * ROW]);
                const u32x4 vf = {v0[0], v0[1], v1[0], v1[1]};
#pragma unroll
                for (int i = 0; i < QB; ++i) o[i][d] = mma(vf, p[i][c], o[i][d]);
            }
    };
    const auto other_k = [&]() {
        k_to ^= TILE;
#pragma unroll
        for (int st = 0; st < KS; ++st) k_from[st] ^= TILE;
    };
    const auto other_v = [&]() {
        v_to ^= TILE;
#pragma unroll
        for (int d = 0; d < DT; ++d) v_from[d] ^= TILE;
    };
    // Largest of the lane's scores of each row (its other half is in lane ^ 32), keys `key0` ..; masked: those that a row does not see are
    // taken out first.
    const auto maxima = [&](f32x16 (&s)[QB], float (&top)[QB], int key0, auto masked) {
#pragma unroll
        for (int i = 0; i < QB; ++i) {
            if constexpr (masked) {
                const int last = min(nk - 1, a.causal ? shift + w0 + 32 * i + col : nk - 1) - key0;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[i][r] = 8 * (r / 4) + 4 * h + r % 4 > last ? -INFINITY : s[i][r];
            }
            top[i] = s[i][0];
#pragma unroll
            for (int r = 1; r < 16; ++r) top[i] = fmaxf(top[i], s[i][r]);
        }
    };
    // Weights of scores, relative to m, and their sum (before they are rounded: lse is as exact as fp32).
    const auto weights = [&](f32x16 (&s)[QB], u32x4 (&p)[QB][2]) {
#pragma unroll
        for (int i = 0; i < QB; ++i) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[i][r] = __builtin_amdgcn_exp2f(fmaf(s[i][r], a.scale_log2, -base[i]));
                l[i] += s[i][r];
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) p[i][c][j] = pack_bf16(s[i][8 * c + 2 * j], s[i][8 * c + 2 * j + 1]);
        }
    };

    // Half a tile (32 keys) at a time: the scores of the next half, the weights of this one and the sums of the one before depend on nothing
    // of each other, so the matrix unit works on the first and third while the vector unit forms the second.
    f32x16 sa[QB], sb[QB];
    u32x4 pa[QB][2], pb[QB][2];
    float top[QB];
    // The sums may stand relative to any value: they go over to a new maximum only where that is 2^8 above the old.  The weights p of the half
    // before are still relative to the old one, so their sums (half n of the tile at v_from) are taken first.
    const auto grow = [&](u32x4 (&p)[QB][2], auto n) {
        bool over = false;
#pragma unroll
        for (int i = 0; i < QB; ++i) over |= top[i] > limit[i];
        if (__any(over)) {
            values(p, n);
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                p[i][0] = p[i][1] = u32x4{0, 0, 0, 0};
                const float most = other_half_max(top[i]), next = most > limit[i] ? most : m[i];
                const float f = next == m[i] ? 1.f : __builtin_amdgcn_exp2f((m[i] - next) * a.scale_log2);
                m[i] = next;
                base[i] = next == -INFINITY ? 0.f : next * a.scale_log2;
                limit[i] = next + slack;
                l[i] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[i][d][r] *= f;
            }
        }
    };
    // The order of such a half: matrix instructions with LDS reads for the ones behind them and VALU instructions between them.
    const auto interleave = [&](auto masked) {
        constexpr int M = (KS + 2 * DT) * QB, R = KS + 4 * DT, V = (masked ? 120 : NVAL) * QB / M + 1;
        __builtin_amdgcn_sched_group_barrier(0x100, NPRE, 0);
        static_for<M>([&](auto i) {
            constexpr int reads = (i + 1) * (R - NPRE) / M - i * (R - NPRE) / M;
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
        });
    };
    // Tile t + 1 of K and tile t of V go to LDS meanwhile, each into the place of the one two before it, whose last reader is behind a barrier.
    const int last_tile = (nk - 1) / kKeys;
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
    const auto tile = [&](int t, auto masked) {
        if (t + 1 == last_tile) {
            rows_at(kat, a.k.ts, last_tile);
            rows_at(vat, a.v.ts, last_tile);
        }
        fetch(kp, kat, a.k.ts, t + 1);
        grow(pb, One{});
        scores(sb, One{});
        weights(sa, pa);
        values(pb, One{});                         // the half before: tile t - 1's second
        maxima(sb, top, t * kKeys + 32, masked);
        other_k();
        other_v();
        store(k_to);
        if constexpr (SCHED) interleave(masked);
        __syncthreads();
        fetch(vp, vat, a.v.ts, t + 1);
        grow(pa, Zero{});
        scores(sa, Zero{});                        // tile t + 1
        weights(sb, pb);
        values(pa, Zero{});
        maxima(sa, top, (t + 1) * kKeys, masked);
        store(v_to);
        if constexpr (SCHED) interleave(masked);
    };
    if (n_tiles > 0) {
        rows_at(kat, a.k.ts, 0);
        rows_at(vat, a.v.ts, 0);
        fetch(kp, kat, a.k.ts, 0);
        store(k_to);
        fetch(vp, vat, a.v.ts, 0);
        store(v_to);
#pragma unroll
        for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4 *>(&s_kv[VT + TILE + (tid + i * kWaves * 64) * 16]) = u32x4{0, 0, 0, 0};       // values of the half before the first
#pragma unroll
        for (int i = 0; i < QB; ++i) pb[i][0] = pb[i][1] = u32x4{0, 0, 0, 0};
        __syncthreads();
        scores(sa, Zero{});
        maxima(sa, top, 0, std::true_type{});
#pragma unroll
        for (int d = 0; d < DT; ++d) v_from[d] ^= TILE;
        int t = 0;
        for (; t + 1 < whole_tiles; ++t) tile(t, std::false_type{});
        for (; t < n_tiles; ++t) tile(t, std::true_type{});
        values(pb, One{});
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

#ifndef QBSEL
#define QBSEL 1
#endif
hipError_t launch_prompt(const PromptArgs &a, hipStream_t s) {
    if (a.D <= 64) prompt_n<64, QBSEL>(a, s);
    else prompt_n<128, QBSEL>(a, s);
    return hipGetLastError();
}

}  // namespace qattn
