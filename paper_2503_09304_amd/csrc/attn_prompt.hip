// attn_prompt: attention over packed prompts, causal or not, heads grouped over shared keys.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup has 4 waves; a wave owns 32 queries of one
// head (of as many heads of a key/value head as share a tile, see prompt_log_tile) and goes through the keys 64 at a time:
//     S^T[key, q] = K Q^T     v_mfma_f32_16x16x32_bf16, A = 16 keys x 32 d, B = 32 d x 16 queries
//     O^T[d, q]   = V^T P^T   A = 16 d x 32 keys, B = 32 keys x 16 queries
// Transposed like this a lane holds 8 of 32 keys of each of its two queries, so maxima and sums are formed inside the lane (an exchange between
// the 4 lanes of a query is needed only where a maximum grows, and at the end), and the weights are the second product's B operand as they
// stand: slot 8g + 4t + r of it (g = lane / 16) is key 16t + 4g + r, and V^T is read in that order.
// K and V tiles are staged in LDS, double-buffered, through registers, each requested a whole tile before it is stored there, in 16-byte pieces
// XOR-swizzled by row.  K rows are read as they are, V^T by ds_read_b64_tr_b16.
//
// What bounds it.  Per 32 keys and 32 queries of 128 elements a wave has 32 matrix instructions (512 clocks of its SIMD), 24 LDS reads and
// 84 vector instructions, 16 of them exponentials (400 clocks).  Two workgroups share a CU: 2 waves on a SIMD.  On zeros the kernel runs at 1.27
// PFLOP/s, on random values at 1.1, at 2.0 GHz instead of 2.4: the power limit, as for this library's other large products (a large product of the vendor's
// library 1.19).  So what counts is clocks and energy: scores, weights and sums of three successive half tiles side by side (below), a maximum
// that stays needs no rescaling (2^8 of room), 16x16x32 instructions (2.5 % over 32x32x16).  Steps from the first kernel, 16384 tokens, 32 heads on 8, us, each on its day's box: 3864;
// side by side 2494; no rescaling 2141; maxima behind the scores 2077; 16x16x32 2039; loads a tile ahead 2005; ends by wave 1979.
// Kept out: two blocks of 32 queries a wave (LDS read half as often, but one wave a SIMD: 2300 at the time), rows padded instead of swizzled (2083, bank
// conflicts), the sums' instructions in assembly into their own registers (2083), rescaling the sums half a tile later (2088).
//
// Measured (us, TFLOP/s; boxes differ by 3 %): 16384 tokens, 32 heads of 128 on 8, 2000 to 2050, 1100 to 1072; 4096 147, 937; 3584 in 8 prompts 46 to 48; 16 heads of 64
// on as many 608 to 622, 904; 17 tokens 6.9.
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
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kKeys = 64;                         // keys of a tile

__device__ __forceinline__ f32x4 mma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
// Over the 4 lanes that hold one row, in each of them.
template <class F>
__device__ __forceinline__ float row_all(float v, F &&f) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F &&f) {
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}
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

// Slots of 16 bytes: piece c of row r of a tile stands at c ^ swz(r), so that what a read takes in at once, 256 bytes, comes from all banks: one piece
// of 16 rows (K), two of 8 rows (V).
template <int DP>
__device__ __forceinline__ int swz_k(int r) { return DP == 128 ? r & 15 : (r >> 1) & 7; }
template <int DP>
__device__ __forceinline__ int swz_v(int r) { return DP == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }

constexpr int kTileRows = kWaves * 32;             // rows of a workgroup: a tile of queries (1 << a.log_tile of them) for each of the heads that it has

// The keys of a tile of queries are cut into parts where they are many and the queries few: as many as have about a share each, one at least and
// a.parts at most.  A share is what a workgroup has if the chip is full and all have the same, kPartTiles tiles of keys at least: joining costs 5 us and 8 bytes an
// element.  Us with 8, 6 and 4 tiles at least, 32 heads on 8: 16 queries on 2016 keys 22.9, 22.9, 19.8 (uncut 41); 128 on 1128 28.4, 26.2, 26.3 (29); 200 on 1200 31, 29, 32 (30); four
// times 16 on 500 to 8000 31, 31, 32 (59); 64 on 8064 35 each (79); 512 on 4096 57 each (72); six times 50 to 300 on 100 to 3000, 16 heads of 64, 32, 35, 35 (47).
constexpr uint32_t kPartTiles = 4;
// Lengths here are in steps of as many keys as a tile has queries; w: the work of a tile.
__host__ __device__ inline int head_groups(const PromptArgs &a) { return a.Hq * (1 << a.log_tile) / kTileRows; }          // workgroups of a tile
struct Cut {
    uint32_t share, most;
    __device__ __forceinline__ uint32_t parts(uint32_t w) const { return most == 1 ? 1u : min(max((w + share / 2) / share, 1u), most); }
    // parts(0) + ... + parts(w - 1)
    __device__ __forceinline__ uint32_t sum(uint32_t w) const {
        if (most == 1) return w;
        const uint32_t x = w + share / 2, capped = min(x, (most + 1) * share), k = capped / share;
        return min(w, share - share / 2) + share * (k * (k - 1) / 2) + (capped - k * share) * k + (x - capped) * most;
    }
};
__device__ __forceinline__ int2 tiles_of(const PromptArgs &a, const Span &s) {
    return {(s.nq + (1 << a.log_tile) - 1) >> a.log_tile, max(0, a.causal ? s.nk - s.nq : s.nk) >> a.log_tile};
}
__device__ __forceinline__ Sequences sequences(const PromptArgs &a) { return {a.cu_q, a.cu_k, a.n_seqs, a.n_q, a.n_k, [&](const Span &s) { return tiles_of(a, s); }}; }
__device__ __forceinline__ Cut cut_of(const PromptArgs &a, const Sequences &seqs) {
    if (a.parts == 1) return {1, 1};
    uint32_t work = 0;                            // of all tiles, a step more of each sequence's at most
    Reached reached;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        const int2 t = tiles_of(a, seqs.at(b0, reached));
        work += t.x * (t.y + (t.x + 1) / 2);
    }
    work = last_lane(wave_scan(work));
    return {max(kPartTiles * kKeys >> a.log_tile, (uint32_t)min((unsigned long long)work * head_groups(a) / a.slots + 1, 1ull << 26)), (uint32_t)a.parts};
}
// The tile of queries and the part of its keys with this number; the tiles of keys that the tile's last query sees.
__device__ __forceinline__ Tile tile_of(const PromptArgs &a, const Sequences &seqs, const Cut &cut, uint32_t number, bool whole) {
    const Tile at = find_heaviest(seqs, number, [&](const Span &s) { return tiles_of(a, s); },
        [&](uint32_t w) { return whole ? 1u : cut.parts(w); }, [&](uint32_t w) { return whole ? w : cut.sum(w); });
    const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };          // the same in all lanes, and to be known as such
    return {scalar(at.piece), scalar(at.part), scalar(at.work), {scalar(at.span.q0), scalar(at.span.nq), scalar(at.span.k0), scalar(at.span.nk)}};
}
__device__ __forceinline__ int key_tiles(const PromptArgs &a, const Span &s, int q_end) {
    return ((a.causal ? min(s.nk, max(0, s.nk - s.nq + min(s.nq, q_end))) : s.nk) + kKeys - 1) / kKeys;
}

template <int DP>
__global__ __launch_bounds__(kWaves * 64, 2) void prompt_tile(const PromptArgs a, int item0) {
    const int QT = 1 << a.log_tile, wg_heads = kTileRows >> a.log_tile;
    constexpr int CH = DP / 8;                    // 16-byte pieces of a row
    constexpr int KS = DP / 32;                   // MFMA steps of a score
    constexpr int DT = DP / 16;                   // 16-d tiles of the output
    constexpr int LD = kKeys * CH / (kWaves * 64);   // pieces of K (and V) that a thread moves per tile
    constexpr int ROW = DP * 2, TILE = kKeys * ROW, VT = 2 * TILE;       // bytes
    __shared__ __attribute__((aligned(16))) uint8_t s_kv[4 * TILE];      // two tiles of K, two of V

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    // Neighbouring workgroups run on different XCDs: those of one key/value head are Hk apart, so with 8 such heads
    // each XCD's L2 holds the keys of one.  Tiles that see the most keys start first.
    const int G = a.Hq / a.Hk, groups = G / wg_heads, num = blockIdx.x + item0;
    const int hk = num % a.Hk, rest = num / a.Hk, head = hk * G + rest % groups * wg_heads + wave % wg_heads;
    const Sequences seqs = sequences(a);
    const Cut cut = cut_of(a, seqs);
    const Tile at = tile_of(a, seqs, cut, (uint32_t)(rest / groups), false);
    if (at.piece < 0) return;
    const int nq = at.span.nq, r0 = at.piece * QT;                       // first query of the tile, within the sequence
    const long q_row = at.span.q0;
    const int w0 = r0 + wave / wg_heads * 32;                // first query of the wave
    // Keys of the part: a query r sees those before shift + r + 1.
    const int all_tiles = key_tiles(a, at.span, r0 + QT), parts = (int)cut.parts(at.work), part = at.part;
    const int first_key = (int)((long)all_tiles * part / parts) * kKeys, end_key = (int)((long)all_tiles * (part + 1) / parts) * kKeys;
    const long k_row = at.span.k0 + first_key;
    const int nk = min(at.span.nk, end_key) - first_key, shift = at.span.nk - nq - first_key;
    // tiles of keys that the tile's last query sees; that the wave's last query sees, and its first query sees whole
    const auto tiles_to = [&](int r) { return ((a.causal ? min(nk, max(0, shift + min(nq, r))) : nk) + kKeys - 1) / kKeys; };
    const int n_tiles = tiles_to(r0 + QT), wave_tiles = w0 < nq ? tiles_to(w0 + 32) : 0;
    const int whole_tiles = min(wave_tiles, min(nk, a.causal ? max(0, shift + w0 + 1) : nk) / kKeys);

    f32x4 o[DT][2];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][0] = o[d][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    // What a row's sums are relative to, in powers of two too (0 before there is one), and the largest score that needs no other; the sum of
    // its weights, and the largest score of the half tile that is next (both of the lane's keys: the others are 16, 32 and 48 lanes away).
    const float slack = 8.f / a.scale_log2;
    float m[2] = {-INFINITY, -INFINITY}, base[2] = {0.f, 0.f}, limit[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, top[2];

    // The 16-byte pieces that this thread moves: rows tr + i * (256 / CH) of a tile, piece tc.  Rows behind the last key are that key again
    // (their weights are 0), pieces behind the end of a head its last one (the queries are 0 there, those outputs are not stored).
    const int tr = tid / CH, tc = tid % CH, dc = min(tc * 8, a.D - 8);
    const uint16_t *kp = a.k.p + k_row * a.k.ts + (long)hk * a.k.hs;
    const uint16_t *vp = a.v.p + k_row * a.v.ts + (long)hk * a.v.hs;
    u32x4 k_moved[LD], v_moved[LD];               // on their way
    uint32_t kat[LD], vat[LD];                    // bytes from the tile's first row
    const auto rows_at = [&](uint32_t (&at)[LD], long stride, int t) {
#pragma unroll
        for (int i = 0; i < LD; ++i) at[i] = 2u * (uint32_t)(max(0, min(tr + i * (kWaves * 64 / CH), nk - 1 - t * kKeys)) * (int)stride + dc);
    };
    const auto fetch = [&](u32x4 (&moved)[LD], const uint16_t *p, const uint32_t (&at)[LD], long stride, int t) {
        const char *tile = (const char *)(p + min(t, (nk - 1) / kKeys) * kKeys * stride);
#pragma unroll
        for (int i = 0; i < LD; ++i) moved[i] = *reinterpret_cast<const u32x4 *>(tile + here(at[i]));
    };
    const int last_tile = (nk - 1) / kKeys;
    if (n_tiles > 0) {
        rows_at(kat, a.k.ts, 0);
        rows_at(vat, a.v.ts, 0);
        fetch(k_moved, kp, kat, a.k.ts, 0);
        fetch(v_moved, vp, vat, a.v.ts, 0);
    }
    u32x4 qf[2][KS];                              // queries w0 + col, w0 + 16 + col
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint16_t *p = a.q.p + (q_row + min(w0 + 16 * q + col, nq - 1)) * a.q.ts + (long)head * a.q.hs;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[q][s] = *reinterpret_cast<const u32x4 *>(p + min(32 * s + 8 * g, a.D - 8));
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (32 * s + 8 * g >= a.D) qf[q][s] = u32x4{0, 0, 0, 0};
    }
    // Places in LDS (bytes; 16-byte pieces are XOR-swizzled by row, in the same way for rows that are 16 apart (K), 8 apart (V)), so that what is
    // read and written differs from these by constants.
    int k_to, v_to, k_from[KS], v_from[DT];
    k_to = tr * ROW + (tc ^ swz_k<DP>(tr)) * 16;
    v_to = VT + tr * ROW + (tc ^ swz_v<DP>(tr)) * 16;
#pragma unroll
    for (int st = 0; st < KS; ++st) k_from[st] = col * ROW + ((4 * st + g) ^ swz_k<DP>(col)) * 16;
    const int v_row = 4 * g + col / 4;
#pragma unroll
    for (int d = 0; d < DT; ++d) v_from[d] = VT + v_row * ROW + ((2 * d + (lane & 3) / 2) ^ swz_v<DP>(v_row)) * 16 + (lane & 1) * 8;
    const auto store = [&](const u32x4 (&moved)[LD], int to) {
#pragma unroll
        for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4 *>(&s_kv[to + i * (kWaves * 64 / CH) * ROW]) = moved[i];
    };
    // A operands: keys 32 n + 16 t .. of the tile at k_from, elements 32 st ..; values of keys 32 n .., elements 16 d ...
    const auto k_frag = [&](int n, int t, int st) { return *reinterpret_cast<const u32x4 *>(&s_kv[k_from[st] + (32 * n + 16 * t) * ROW]); };
    const auto v_frag = [&](int n, int d) {
        const u32x2 v0 = read_transposed(&s_kv[v_from[d] + 32 * n * ROW]), v1 = read_transposed(&s_kv[v_from[d] + (32 * n + 16) * ROW]);
        return u32x4{v0[0], v0[1], v1[0], v1[1]};
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
    // o += V^T P^T for keys 32 n .. of the tile at v_from.
    const auto add_values = [&](const u32x4 &v, const u32x4 (&p)[2], int d) {
#pragma unroll
        for (int q = 0; q < 2; ++q) o[d][q] = mma(v, p[q], o[d][q]);
    };
    // Scores: [query tile][key tile], a lane's element r is key 16 t + 4 g + r of query 16 q + col.
    typedef f32x4 Scores[2][2];
    const auto add_scores = [&](const u32x4 &k, Scores &s, int t, int st) {
#pragma unroll
        for (int q = 0; q < 2; ++q) s[q][t] = mma(k, qf[q][st], st == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[q][t]);
    };
    // The largest of the lane's scores s of keys `key0` ..; masked: those that the row does not see are taken out first.
    const auto maximum = [&](Scores &s, int key0, auto masked) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if constexpr (masked) {
                const int last = min(nk - 1, a.causal ? shift + w0 + 16 * q + col : nk - 1) - key0 - 4 * g;
#pragma unroll
                for (int r = 0; r < 8; ++r) s[q][r / 4][r % 4] = 16 * (r / 4) + r % 4 > last ? -INFINITY : s[q][r / 4][r % 4];
            }
            top[q] = s[q][0][0];
#pragma unroll
            for (int r = 1; r < 8; ++r) top[q] = fmaxf(top[q], s[q][r / 4][r % 4]);
        }
    };
    // The sums may stand relative to any value: they go over to a new maximum only where that is 2^8 above the old.  The weights p of the half
    // before are still relative to the old one, so their sums (half n of the tile at v_from) are taken first.
    const auto grow = [&](u32x4 (&p)[2], auto n) {
        if (__any(top[0] > limit[0] || top[1] > limit[1])) {
            static_for<DT>([&](auto d) { add_values(v_frag(n, d), p, d); });
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                p[q] = u32x4{0, 0, 0, 0};
                const float most = row_all(top[q], [](float x, float y) { return fmaxf(x, y); }), next = most > limit[q] ? most : m[q];
                const float f = next == m[q] ? 1.f : __builtin_amdgcn_exp2f((m[q] - next) * a.scale_log2);
                m[q] = next;
                base[q] = next == -INFINITY ? 0.f : next * a.scale_log2;
                limit[q] = next + slack;
                l[q] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d][q] *= f;
            }
        }
    };
    // Half a tile (32 keys) at a time: the scores of the next half, the weights of this one and the sums of the one before depend on nothing
    // of each other, so the matrix unit works on the first and third while the vector unit forms the second.
    // Step by step: a matrix instruction, the LDS read of the one LA steps behind it, and a share of the vector work.  Left to the
    // compiler the reads stand right in front of their use, and each waits out LDS.
    // Scores of half n_k of the tile at k_from -> next (and their maxima -> top), weights of cur -> p_cur, sums of half n_v with p_old.
    constexpr int LA = 4;                         // steps that LDS is read ahead (3, 6 and 8: the same within 1 %)
    const auto half = [&](Scores &next, auto n_k, Scores &cur, u32x4 (&p_cur)[2], const u32x4 (&p_old)[2], auto n_v, int key0, auto masked) {
        constexpr int N = 2 * KS, M = 2 * N;          // score steps (and as many steps for the sums), steps in all
        // Scores and sums in turn, so that no step waits for the one before; the last scores a little earlier, their maxima are last.
        constexpr auto is_score = [](int i) { return i < M - 4 ? i % 2 == 0 : i < M - 2; };
        constexpr auto index = [](int i) { return i < M - 4 ? i / 2 : N - 2 + i % 2; };
        u32x4 frag[M];
        const auto read = [&](auto i) {
            constexpr int j = index(i);
            if constexpr (is_score(i)) frag[i] = k_frag(n_k, j / KS, j % KS);
            else frag[i] = v_frag(n_v, j);
        };
        const auto weight = [&](int i) {
            const int q = i / 8, t = i % 8 / 4, r = i % 4;
            cur[q][t][r] = __builtin_amdgcn_exp2f(fmaf(cur[q][t][r], a.scale_log2, -base[q]));
            l[q] += cur[q][t][r];
            // To bf16, as the values beside them in the product are: half a step, and errors against 64 bits 1.3 times those of fp32 weights (16384 tokens:
            // 2.1e-3 of the outputs' size to 1.6e-3, which is what rounding the outputs alone leaves).  A product with what the rounding leaves would be half
            // as many matrix instructions again where these are the bound.
            if (r & 1) p_cur[q][2 * t + r / 2] = pack_bf16(cur[q][t][r - 1], cur[q][t][r]);
        };
        static_for<LA>(read);
        __builtin_amdgcn_s_setprio(1);                // before the CU's other waves, while those are between halves: 16384 tokens 1 %, 4096 5 %
        __builtin_amdgcn_sched_barrier(0);
        static_for<M>([&](auto i) {
            constexpr int j = index(i);
            if constexpr (is_score(i)) add_scores(frag[i], next, j / KS, j % KS);
            else add_values(frag[i], p_old, j);
            if constexpr (i + LA < M) read(std::integral_constant<int, i + LA>{});
            static_for<16 / M>([&](auto r) { weight(i * (16 / M) + r); });
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
        maximum(next, key0, masked);
    };
    Scores sa, sb;
    u32x4 pa[2], pb[2];
    // Tile t + 1 of K goes to LDS at the end of the first half, of V at the end of the second, each into the place of the one two before it, whose
    // last reader is behind a barrier; each was requested a whole tile earlier.
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
    const auto tile = [&](int t, auto masked) {
        if (t + 1 == last_tile) rows_at(vat, a.v.ts, last_tile);
        if (t + 2 == last_tile) rows_at(kat, a.k.ts, last_tile);
        fetch(v_moved, vp, vat, a.v.ts, t + 1);
        grow(pb, One{});
        half(sb, One{}, sa, pa, pb, One{}, t * kKeys + 32, masked);      // the half before: tile t - 1's second
        other_k();
        other_v();
        store(k_moved, k_to);
        __syncthreads();
        fetch(k_moved, kp, kat, a.k.ts, t + 2);
        grow(pa, Zero{});
        half(sa, Zero{}, sb, pb, pa, Zero{}, (t + 1) * kKeys, masked);   // the next: tile t + 1's first
        store(v_moved, v_to);
    };
    if (n_tiles > 0) {
#pragma unroll
        for (int i = 0; i < LD; ++i) *reinterpret_cast<u32x4 *>(&s_kv[VT + TILE + (tid + i * kWaves * 64) * 16]) = u32x4{0, 0, 0, 0};       // values of the half before the first
#pragma unroll
        for (int i = 0; i < 2; ++i) pb[i] = u32x4{0, 0, 0, 0};
        store(k_moved, k_to);
        if (last_tile == 1) rows_at(kat, a.k.ts, 1);
        fetch(k_moved, kp, kat, a.k.ts, 1);
        store(v_moved, v_to);
        __syncthreads();
        static_for<2 * KS>([&](auto i) { add_scores(k_frag(0, i / KS, i % KS), sa, i / KS, i % KS); });
        maximum(sa, 0, std::true_type{});
#pragma unroll
        for (int d = 0; d < DT; ++d) v_from[d] ^= TILE;
        int t = 0;
        for (; t + 1 < whole_tiles; ++t) tile(t, std::false_type{});
        for (; t < wave_tiles; ++t) tile(t, std::true_type{});
        static_for<DT>([&](auto d) { add_values(v_frag(1, d), pb, d); });
        for (; t < n_tiles; ++t) {                 // for the other waves: what tile() moves, and its barrier
            if (t + 1 == last_tile) rows_at(vat, a.v.ts, last_tile);
            if (t + 2 == last_tile) rows_at(kat, a.k.ts, last_tile);
            fetch(v_moved, vp, vat, a.v.ts, t + 1);
            k_to ^= TILE;
            v_to ^= TILE;
            store(k_moved, k_to);
            __syncthreads();
            fetch(k_moved, kp, kat, a.k.ts, t + 2);
            store(v_moved, v_to);
        }
    }

    if (parts > 1) {                              // join_parts' to finish
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float sum = row_all(l[q], [](float x, float y) { return x + y; });
            const int r = w0 + 16 * q + col;
            if (r >= nq) continue;
            const long at_row = ((long)part * a.n_q + q_row + r) * a.Hq + head;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (16 * d < a.D) *reinterpret_cast<f32x4 *>(a.part_o + at_row * a.D + 16 * d + 4 * g) = o[d][q];
            if (g == 0) *reinterpret_cast<float2 *>(a.part_ml + at_row * 2) = float2{m[q] * a.scale_log2, sum};
        }
        return;
    }
    // Out through LDS, for stores of whole rows: a lane's elements are 8 bytes of each 32 (32 sequences of 128 tokens, 32 heads: 3900 of a workgroup's 25000 clocks).
    constexpr int O_ROW = DP * 2 + 16;
    __syncthreads();                              // the other waves' last reads of K and V
    uint8_t *s_o = &s_kv[wave * 32 * O_ROW];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float sum = row_all(l[q], [](float x, float y) { return x + y; }), inv = sum != 0.f ? 1.f / sum : 0.f;
        const int r = w0 + 16 * q + col;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const f32x4 x = o[d][q] * inv;
            *reinterpret_cast<u32x2 *>(s_o + (16 * q + col) * O_ROW + 32 * d + 8 * g) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        }
        if (a.lse != nullptr && g == 0 && r < nq)
            a.lse[(q_row + r) * a.Hq + head] = sum != 0.f ? (m[q] * a.scale_log2 + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    }
    uint16_t *to = a.o.p + q_row * a.o.ts + (long)head * a.o.hs;
#pragma unroll
    for (int i = 0; i < 32 * CH / 64; ++i) {
        const int row = (i * 64 + lane) / CH, c = lane % CH;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(s_o + row * O_ROW + c * 16);
        if (w0 + row < nq && c * 8 < a.D) *reinterpret_cast<u32x4 *>(to + (w0 + row) * a.o.ts + c * 8) = x;
    }
}

// The parts of 32 queries of one head joined, in their order.
constexpr int kJoinQ = 32;
__global__ __launch_bounds__(256) void join_parts(const PromptArgs a, int item0) {
    const int num = blockIdx.x + item0, head = num % a.Hq, rest = num / a.Hq, joins = (1 << a.log_tile) / kJoinQ;
    const Sequences seqs = sequences(a);
    const Cut cut = cut_of(a, seqs);
    const Tile at = tile_of(a, seqs, cut, (uint32_t)(rest / joins), true);
    if (at.piece < 0) return;
    const int r0 = (at.piece << a.log_tile) + rest % joins * kJoinQ, parts = (int)cut.parts(at.work);
    if (parts == 1) return;
    const int rows = min(kJoinQ, at.span.nq - r0), c = a.D / 4;
    const long stride = (long)a.n_q * a.Hq;
    for (int i = threadIdx.x; i < rows * c; i += 256) {
        const int r = i / c, d = (i - r * c) * 4;
        const long row = at.span.q0 + r0 + r, at_row = row * a.Hq + head;
        float top = -INFINITY, sum = 0.f;
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
        constexpr int U = 4;                      // parts requested before the first is used
        for (int p0 = 0; p0 < parts; p0 += U) {
            float2 ml[U];
            f32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long x = min(p0 + u, parts - 1) * stride + at_row;
                ml[u] = *reinterpret_cast<const float2 *>(a.part_ml + x * 2);
                v[u] = *reinterpret_cast<const f32x4 *>(a.part_o + x * a.D + d);
            }
            float next = top;
#pragma unroll
            for (int u = 0; u < U; ++u) next = fmaxf(next, ml[u].x);
            const float base = next == -INFINITY ? 0.f : next, keep = __builtin_amdgcn_exp2f(top - base);
            top = next;
            sum *= keep;
            acc *= keep;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float f = p0 + u < parts ? __builtin_amdgcn_exp2f(ml[u].x - base) : 0.f;
                sum += f * ml[u].y;
                acc += v[u] * f;
            }
        }
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        *reinterpret_cast<u32x2 *>(a.o.p + row * a.o.ts + (long)head * a.o.hs + d) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
        if (a.lse != nullptr && d == 0) a.lse[at_row] = sum != 0.f ? (top + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    }
}

template <int DP>
void prompt_n(const PromptArgs &a, hipStream_t s) {
    const long tiles = ((a.n_q + (1l << a.log_tile) - 1) >> a.log_tile) + a.n_seqs, groups = head_groups(a);
    // With parts(w) <= 1 + w / share and a share of all work * groups / slots or more, cutting adds slots / groups parts at most.
    const long all = (a.parts == 1 ? tiles : std::min(tiles * a.parts, tiles + a.slots / groups + 1)) * groups;
    in_launches(all, [&](int at, unsigned n) { prompt_tile<DP><<<dim3(n), dim3(kWaves * 64), 0, s>>>(a, at); });
    const long joins = a.parts > 1 ? tiles * a.Hq * ((1 << a.log_tile) / kJoinQ) : 0;
    in_launches(joins, [&](int at, unsigned n) { join_parts<<<dim3(n), dim3(256), 0, s>>>(a, at); });
}

}  // namespace

int prompt_slots(int D) { return D <= 64 ? 768 : 512; }

// Queries of a tile where several heads share a key/value head: 32 of four heads or 64 of two, all waves with the same keys and fewer idle in a sequence's last tile. Us with 32 / 128:
// 3584 tokens in 8 prompts 50 / 54, 16 times 8 queries on 1500 keys 35 / 43, five chunks of 1 to 500 on 30 226 keys 56 / 61; 16384 tokens 2016 / 2018.
static int most_heads(int Hq, int Hk) { return Hq / Hk % 4 == 0 ? 4 : Hq / Hk % 2 == 0 ? 2 : 1; }
static long tiles_about(int n_seqs, int n_q, int queries) { return std::max((n_q + (long)queries - 1) / queries + (n_seqs - 1) / 2, (long)n_seqs); }
// Where every workgroup of 128 queries has a CU of its own, idle waves cost nothing, and fewer busy ones are faster: 17 tokens 6.6 / 7.2, 2 times 300 13.3 / 14.2.
int prompt_log_tile(int n_seqs, int n_q, int Hq, int Hk, int parts) {
    if (parts == 1 && tiles_about(n_seqs, n_q, kTileRows) * Hq <= 256) return 7;
    return most_heads(Hq, Hk) == 4 ? 5 : most_heads(Hq, Hk) == 2 ? 6 : 7;
}

// Most parts for a call; which tiles are cut into how many the kernels decide.  The host knows the totals only, and rules out where nothing can be gained for the 5 us:
// where most CUs have work as it is.  A second workgroup on a CU adds half to what it does, so one sequence is cut where it fills a third of the chip or less (us uncut / cut: 1024
// queries on 2048 keys, 32 heads 48 / 58, 512 on 4096 72 / 56; 2048 on as many, 8 heads 48 / 36); several may be uneven, their longest twice the average: two thirds
// (700 and 900 queries on 3700 and 2900 keys, 32 heads 95 / 102; 2434 of six on 16 649, 16 heads of 64 72 / 63), whole prompts half.  And short sequences: 16 tiles
// of keys (1024 on as many, 8 heads) 26 / 29, 18 (128 on 1128, 32 heads) 29 / 26.  16 parts at most (with 8: four times 16 on 500 to 8000 keys 36 us instead of 31; 32: the same).
int prompt_parts(int n_seqs, int n_q, int n_k, int Hq, int Hk, int D) {
    const int heads = most_heads(Hq, Hk), queries = kTileRows / heads;
    const long slots = prompt_slots(D), tiles = (n_q + (long)queries - 1) / queries, each = (long)n_k / n_seqs / kKeys;
    const long wgs = tiles_about(n_seqs, n_q, queries) * Hq / heads, f = n_seqs == 1 ? 1 : 2;
    if (3 * wgs > f * slots || (n_k < 2l * n_q && 2 * wgs >= slots) || f * each <= 16) return 1;
    if ((tiles + n_seqs) * ((long)n_k / queries + tiles + 2) >= 1l << 31) return 1;                // the kernels' sums of work have 32 bits
    const long share = std::max((long)kPartTiles, each * wgs / slots);
    return (int)std::max(1l, std::min((f * each + share / 2) / share, 16l));
}

// Heads between run as the next of 64 and 128, their missing elements as zeros that are multiplied too: 16384 tokens, 32 heads on 8, 2010 us with heads of 128, 1971 of 96,
// 1957 of 80.  No configuration of this library has others, and kernels of their own were not built for them.
hipError_t launch_prompt(const PromptArgs &a, hipStream_t s) {
    if (a.D <= 64) prompt_n<64>(a, s);
    else prompt_n<128>(a, s);
    return hipGetLastError();
}

}  // namespace qattn
