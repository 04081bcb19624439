// attn_decode: one query a sequence over the paged cache.
//
// Every key and value is read once and used for the G query heads that share it (4 G flop for 2 elements), so the bound is HBM.
// The queries of a key/value head are the 16 columns of v_mfma_f32_16x16x32_bf16 (G up to 16, further ones in another group tile):
//     S^T[key, q] = K Q^T     A = 16 keys x 32 d: a lane holds 16 bytes of one key's row, straight from the page
//     O^T[d, q]   = V^T P^T   A = 16 d x 32 keys
// A lane of S^T holds 4 keys of one column per tile, so with slot 8g + 4t + r of the second product standing for key 16t + 4g + r
// (g = lane / 16, t = 0, 1) the weights are its B operand as they are.  V^T needs 8 keys of one d in a lane: a lane loads 8 bytes
// (fp8: 4 or 8) of each of its 8 keys and sorts them by v_perm, one per two elements, so nothing passes through LDS.
// An fp8 element becomes bf16 exactly; the power of two of a key's row goes onto its score, a value's onto its weight.
//
// Work: a workgroup's 4 waves take blocks of 32 keys in turn, each with its own running maximum and sum, and are joined in LDS.  Sequences are cut into pieces
// of equal size that share all keys out evenly; where lengths do not let them come out even, each workgroup has a range of all keys instead, as long as
// the others', which may begin and end inside sequences and hold several.  Each workgroup finds what is its own from the lengths (attn_pieces.h).  What a sequence has
// in several workgroups goes to the workspace as fp32 sums, and the last of them to arrive joins all in the order of the pieces.
// Us, pieces for 256 / 512 / 1024 workgroups, 8 key/value heads of 128, bf16 unless it says fp8: one sequence of 131071 keys 89 / 94 / 101, fp8 50 / 54 / 61, of 16384
// 19.8 / 23.5 / 23.4.  Pieces for 1024 or 1536 / ranges: 64 of 33 to 16384 keys, fp8, 86 / 79, bf16 154 / 142; 16 of 33 to 30000 71 / 62; 300 of 1 to 2000, 4 heads, 61 / 53; 100000 keys
// beside three short sequences 88 / 80.
//
// Measured (us, TB/s): 131071 keys 86, 6.2; the same in fp8 50, 5.5; 128 sequences of 3000 keys 242, 6.5; 64 of 33 to 16384, fp8, 77, 4.9; of one key 4.5.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_pieces.h"
#include "qattn_internal.h"

namespace qattn {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kBlock = 32;                       // keys of a wave's step
// Steps of a sequence that is not cut: joining its pieces would take longer.  Us uncut / in pieces of two steps at least, 8 key/value heads of 128: 257 keys
// 7.1 / 9.2, 512 9.3 / 9.3, 700 11.3 / 9.5, 1000 14.5 / 9.9; 32 sequences of 512 keys, 4 heads, 11.9 / 12.1; of 600 13.4 / 14.0; of 1 to 1000 17.1 / 11.0.
constexpr uint32_t kWholeSteps = 4;
// Ranges: workgroups of a launch, two on a CU (384 90 us, 448 84, 512 79, 768 80 for 64 sequences of 33 to 16384 keys, fp8), and the fewest steps of one (3, 4, 6: the same).
// A sequence counts as a step more than it has, for its start and end (as two: 0 to 12 % slower).
constexpr uint32_t kRangeWgs = 512, kFewestRange = 6;

__device__ __forceinline__ f32x4 mma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w, bool hi) {
    return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}
__device__ __forceinline__ float power(uint32_t bytes, int i) { return __uint_as_float(((bytes >> (8 * i)) & 0xFFu) << 23); }

// Largest over the 4 lanes that hold one column, in each of them.
__device__ __forceinline__ float column_max(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// An offset of 32 bits that is widened where it is used: widened in front of the loop it would become part of a 64-bit address in vector registers.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Two floats that workgroups of other XCDs write and read.
__device__ __forceinline__ void put(float *p, float a, float b) {
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), __builtin_bit_cast(unsigned long long, f32x2{a, b}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get(const float *p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// m where it stands for something, 0 for a row that has seen no key: x - finite(m) is then -inf, and its exponential 0.
__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }

// A wave's step of 32 keys as it is loaded: two tiles of 16.
template <int DP, bool FP8>
struct Step {
    static constexpr int KL = FP8 ? DP / 64 : DP / 32;       // 16-byte loads of a key's row by its 4 lanes
    static constexpr int VE = FP8 ? DP / 16 : 4;             // elements of a value load: d = VE * (lane % 16) + 0 .. VE - 1 (+ 64 u)
    static constexpr int VU = DP / 16 / VE;                  // value loads of a row
    static constexpr int VW = FP8 ? VE / 4 : VE / 2;         // words of one
    typedef uint32_t V __attribute__((ext_vector_type(VW)));
    long row[2];                                             // first rows (of the cache) of the tiles
    int keys[2];                                             // keys of the tiles: the first so many, 16 or more for all, 0 or less for none
    u32x4 k[2][KL];
    V v[2][4][VU];
    uint32_t ks[2], vs[2];                                   // scale bytes of keys 4g .. 4g + 3
};

// WHOLE: dim is DP, so that offsets within a tile are constants.  RANGES: there may be ranges instead of pieces.
template <int DP, bool FP8, bool WHOLE, bool RANGES>
__global__ __launch_bounds__(kWaves * 64, 3) void decode_piece(const DecodeArgs a, int first_wg) {
    constexpr int KS = DP / 32;                       // MFMA steps of a score
    constexpr int DT = DP / 16;                       // d tiles of the output
    constexpr int ESZ = FP8 ? 1 : 2;
    constexpr int KL = Step<DP, FP8>::KL, VE = Step<DP, FP8>::VE, VU = Step<DP, FP8>::VU, VW = Step<DP, FP8>::VW;
    __shared__ float s_o[kWaves][16][DP + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int GT = group_tiles(a.Hq, a.c.Hk), G = a.Hq / a.c.Hk;
    const uint32_t wg = blockIdx.x + first_wg;
    const int hk = wg % a.c.Hk, gt = (wg / a.c.Hk) % GT, item = wg / (a.c.Hk * GT);
    const int P = 1 << a.c.page_shift, most = a.seq_pages << a.c.page_shift;
    const auto len_of = [&](int b) { return min(max(a.lens[b], 0), most); };

    // Pieces are whole steps of the workgroup (4 x 32 keys), two at least, as many steps as make `wgs` workgroups of all keys.  Sequences of up to four
    // are not cut, those without keys have a piece too, for its zeros.  The fewest workgroups that come out about even are taken: 256 (one a CU) or 512 for one
    // sequence or several of a length; where these do not, ranges, or, with little to do, pieces for 1024 or 1536.
    const int step = kWaves * kBlock, heads = a.c.Hk * GT;
    const auto steps_of = [&](int len) { return (uint32_t)(len + step - 1) / step; };
    uint32_t total = 0;
    for (int i = 0; i < a.n_seqs; i += 64) total = __builtin_elementwise_add_sat(total, i + lane < a.n_seqs ? steps_of(len_of(i + lane)) : 0u);
    total = last_lane(wave_scan(total));
    uint32_t piece_steps = 0;
    const auto pieces_of = [&](int len) { return steps_of(len) <= kWholeSteps ? 1u : (steps_of(len) + piece_steps - 1) / piece_steps; };
    uint32_t range = 0;                           // steps of a workgroup, 0: it has a piece
    for (uint32_t wgs = kFewestWgs; ; wgs = wgs < 1024 ? 2 * wgs : kMostWgs) {
        const uint32_t shares = (wgs + heads - 1) / heads;
        piece_steps = max(2u, (total + shares - 1) / shares);
        if (wgs == kMostWgs) break;
        uint32_t n = 0;
        for (int i = 0; i < a.n_seqs; i += 64) n += i + lane < a.n_seqs ? pieces_of(len_of(i + lane)) : 0u;
        if (last_lane(wave_scan(n)) * heads <= wgs) break;
        if constexpr (RANGES) {
            const uint32_t all = total + (uint32_t)a.n_seqs, r = (uint32_t)(((unsigned long long)all * heads + kRangeWgs - 1) / kRangeWgs);
            if (wgs == kRangeWgs && r >= kFewestRange && total < 1u << 28) {
                if ((uint32_t)item > (all - 1) / r) return;
                range = r;
                break;
            }
        }
    }
    const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };      // the same in all lanes, and to be known as such
    const int hg = gt * a.c.Hk + hk, D = WHOLE ? DP : a.c.D;
    const long piece_size = 16 * (D + 2);         // of a piece in the workspace: [16][D] sums, [16] pairs of maximum and total

    // Keys k0 .. k1 - 1 of sequence b, its piece `piece` of n_pieces; part_at(i): where piece i stands in the workspace.
    const auto run = [&](int b, int len, int piece, int n_pieces, int k0, int k1, auto part_at) {
        const int32_t *pages = a.pages + (long)b * a.seq_pages;
        if (a.bad != nullptr && hk == 0 && gt == 0 && piece == 0) {
            int bad = tid == 0 && a.lens[b] != len;
            for (int i = tid; i < (len + P - 1) >> a.c.page_shift; i += kWaves * 64) bad += (uint32_t)pages[i] >= (uint32_t)a.c.n_pages;
            if (bad != 0) atomicAdd(a.bad, bad);
        }

        // queries of this group tile: column `col`, elements by the order in which a lane holds those of a key
        const int head = hk * G + gt * 16 + col;
        const bool has_q = gt * 16 + col < G;
        u32x4 qf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = FP8 ? (s / 2) * 64 + 16 * g + (s & 1) * 8 : 32 * s + 8 * g;
            qf[s] = has_q && d < a.c.D ? *reinterpret_cast<const u32x4 *>(a.q.p + (long)b * a.q.ts + (long)head * a.q.hs + d) : u32x4{0, 0, 0, 0};
        }

        f32x4 o[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;

        // Offsets of the lane's pieces within a tile of 16 rows.  Where a head has fewer than DP elements the pieces behind its end
        // are its last one again: the queries are zero there, and those outputs are not stored.
        const uint32_t row_bytes = (WHOLE ? DP : a.c.D) * ESZ;
        uint32_t k_at[KL], v_at[VU];                  // 32 bits, added to scalar addresses: 64 bits a load do not leave registers for two steps
#pragma unroll
        for (int i = 0; i < KL; ++i) k_at[i] = col * row_bytes + (WHOLE ? 64 * i + 16 * g : min(64u * i + 16 * g, row_bytes - 16));
#pragma unroll
        for (int u = 0; u < VU; ++u) v_at[u] = 4 * g * row_bytes + (WHOLE ? (64 * u + VE * col) * ESZ : min((64u * u + VE * col) * ESZ, row_bytes - VE * ESZ));

        Step<DP, FP8> st;
        int page[2];                                  // of the step that is fetched next: requested a step before, or its loads would wait for it
        const auto fetch_pages = [&](int k) {
#pragma unroll
            for (int t = 0; t < 2; ++t) page[t] = pages[min(k + 16 * t, k1 - 1) >> a.c.page_shift];
        };
        // Keys of the step at k, then its values: loads come back in the order in which they are issued.
        const auto fetch_keys = [&](int k) {
            int now[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) now[t] = scalar(page[t]);                // addresses are a scalar and an offset
            fetch_pages(k + step);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = k + 16 * t;
                st.keys[t] = (uint32_t)now[t] < (uint32_t)a.c.n_pages ? k1 - key : 0;
                st.row[t] = (((long)(st.keys[t] > 0 ? now[t] : 0) * a.c.Hk + hk) << a.c.page_shift) + (key & (P - 1));
                const uint8_t *kp = a.c.k + st.row[t] * row_bytes;
#pragma unroll
                for (int i = 0; i < KL; ++i) st.k[t][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + here(k_at[i])));
                if constexpr (FP8) st.ks[t] = *reinterpret_cast<const uint32_t *>(a.c.ks + st.row[t] + here(4u * g));
            }
        };
        const auto fetch_values = [&]() {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint8_t *vp = a.c.v + st.row[t] * row_bytes;
                if constexpr (FP8) st.vs[t] = *reinterpret_cast<const uint32_t *>(a.c.vs + st.row[t] + here(4u * g));
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int u = 0; u < VU; ++u)
                        st.v[t][r][u] = __builtin_nontemporal_load(reinterpret_cast<const typename Step<DP, FP8>::V *>(vp + r * row_bytes + here(v_at[u])));
            }
        };
        // Scores of 2 x 4 keys of this lane's column, from the keys.
        const auto score = [&](float (&s)[8]) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KL; ++i) {
                    if constexpr (FP8) {
                        const u32x4 w = st.k[t][i];
                        c = mma(u32x4{fp8_pair(w[0], false), fp8_pair(w[0], true), fp8_pair(w[1], false), fp8_pair(w[1], true)}, qf[2 * i], c);
                        c = mma(u32x4{fp8_pair(w[2], false), fp8_pair(w[2], true), fp8_pair(w[3], false), fp8_pair(w[3], true)}, qf[2 * i + 1], c);
                    } else {
                        c = mma(st.k[t][i], qf[i], c);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * t + r] = FP8 ? c[r] * power(st.ks[t], r) * a.scale_log2 : c[r] * a.scale_log2;
            }
        };
        // Softmax of the scores and their part of the output, from the values; keys[t]: keys of tile t.
        const auto attend = [&](float (&s)[8], const int (&keys)[2]) {
            const bool some = min(keys[0], keys[1]) < 16;
            if (some) {                                       // keys that are none: no score
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = 4 * g + i % 4 >= keys[i / 4] ? -INFINITY : s[i];
            }
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
            top = column_max(top);
            // The sums may stand relative to any value: they are taken over to a new maximum only where it is 2^8 above the old.
            if (__any(top - m > 8.f)) {
                const float next = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - finite(next));
                m = next;
                l *= keep;
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] *= keep;
            }
            const float base = finite(m);
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(s[i] - base);
                l += p[i];
            }
            if (some) {                                       // and zeros for whatever their values hold
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool none = 4 * g + r >= keys[t];
                        if (FP8 && none) st.vs[t] &= ~(0xFFu << (8 * r));
#pragma unroll
                        for (int u = 0; u < VU; ++u)
#pragma unroll
                            for (int i = 0; i < VW; ++i) st.v[t][r][u][i] = none ? 0u : st.v[t][r][u][i];
                    }
                }
            }
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= power(st.vs[i / 4], i % 4);
            }
            // Weights to bf16, as the values beside them in the product are: half a step, and errors against 64 bits 1.1 to 1.4 times those of fp32 weights (131071 keys:
            // 2.3e-3 of the outputs' size to 1.7e-3, which is what rounding the outputs alone leaves).  A second product with what the rounding leaves would hide
            // behind the loads; attn_prompt's weights have none, and a token is to see its context the same way in both.
            const u32x4 pf = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
            // tile (u, e): d = 64 u + VE * (lane % 16) + e
#pragma unroll
            for (int u = 0; u < VU; ++u) {
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    if constexpr (FP8) {
                        // elements 4w .. 4w + 3: bytes of two keys side by side, then two at a time to bf16
                        uint32_t lo[4], hi[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t a0 = st.v[j / 2][2 * (j & 1)][u][w], a1 = st.v[j / 2][2 * (j & 1) + 1][u][w];
                            lo[j] = __builtin_amdgcn_perm(a1, a0, 0x05010400u);
                            hi[j] = __builtin_amdgcn_perm(a1, a0, 0x07030602u);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t *src = e < 2 ? lo : hi;
                            const u32x4 vf = {fp8_pair(src[0], e & 1), fp8_pair(src[1], e & 1), fp8_pair(src[2], e & 1), fp8_pair(src[3], e & 1)};
                            o[VE * u + 4 * w + e] = mma(vf, pf, o[VE * u + 4 * w + e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            u32x4 vf;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                vf[j] = __builtin_amdgcn_perm(st.v[j / 2][2 * (j & 1) + 1][u][w], st.v[j / 2][2 * (j & 1)][u][w], e ? 0x07060302u : 0x05040100u);
                            o[VE * u + 2 * w + e] = mma(vf, pf, o[VE * u + 2 * w + e]);
                        }
                    }
                }
            }
        };
        // The next step's keys are requested as soon as this one's scores are formed, its values as soon as this one's are used, into the same
        // registers.  (A second set of registers for them: 256 and 100 bytes of scratch for bf16 heads of 128, 134 us instead of 94 on 131071 keys, which half the prefetched
        // steps waited for.)
        int k = k0 + wave * kBlock;
        if (k < k1) {
            fetch_pages(k);
            fetch_keys(k);
            fetch_values();
            float s[8];
            for (; k + step < k1; k += step) {
                const int keys[2] = {st.keys[0], st.keys[1]};
                score(s);
                fetch_keys(k + step);
                attend(s, keys);
                fetch_values();
            }
            score(s);
            attend(s, st.keys);
        }
        l = column_sum(l);
        // o[VE u + e][r]: d = 64 u + VE * (4 g + r) + e of column col
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < VE; ++e) s_o[wave][col][64 * u + VE * (4 * g + r) + e] = o[VE * u + e][r];
        if (g == 0) {
            s_m[wave][col] = m;
            s_l[wave][col] = l;
        }
        __syncthreads();

        // the four waves' sums joined: thread (q, x) has elements EX x .. EX x + EX - 1 of query q
        constexpr int EX = DP / 16;
        const int q = tid >> 4, x = tid & 15;
        const int n_q = min(16, G - gt * 16);                        // queries of the tile
        float top = s_m[0][q];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][q]);
        float sum = 0.f, acc[EX] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][q] - finite(top));
            sum += f * s_l[w][q];
#pragma unroll
            for (int i = 0; i < EX; ++i) acc[i] += f * s_o[w][q][EX * x + i];
        }
        const auto finish = [&](int q, int x, float top, float sum, const float (&acc)[EX]) {
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            const int head_q = hk * G + gt * 16 + q;
            uint16_t *to = a.o.p + (long)b * a.o.ts + (long)head_q * a.o.hs + EX * x;
            if (EX * x < D) {
#pragma unroll
                for (int i = 0; i < EX; i += 4)
                    *reinterpret_cast<u32x2 *>(to + i) = u32x2{pack_bf16(acc[i] * inv, acc[i + 1] * inv), pack_bf16(acc[i + 2] * inv, acc[i + 3] * inv)};
            }
            if (a.lse != nullptr && x == 0) a.lse[(long)b * a.Hq + head_q] = sum != 0.f ? (top + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
        };
        if (n_pieces == 1) {
            if (q < n_q) finish(q, x, top, sum, acc);
            return;
        }
        float *part = part_at(piece);
        // Stores of a piece go through to where the other XCDs see them, and have arrived there before the workgroup is counted.  (A
        // release by the counting thread writes back all of its XCD's L2 instead: 0.4 us each, one after the other.)
        if (q < n_q) {
            if (EX * x < D) {
#pragma unroll
                for (int i = 0; i < EX; i += 2) put(part + q * D + EX * x + i, acc[i], acc[i + 1]);
            }
            if (x == 0) put(part + 16 * D + 2 * q, top, sum);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            int32_t *count = a.arrived + (long)b * heads + hg;
            const int n = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = n == n_pieces - 1;
            if (n == n_pieces - 1) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!s_last) return;
        // Groups of 16 threads for each of the queries (n_q rounded up to a power of two), as many to a query as there are: each takes a run of the
        // pieces, and the runs are joined in LDS, in order.
        const int qs = n_q <= 1 ? 1 : n_q <= 2 ? 2 : n_q <= 4 ? 4 : n_q <= 8 ? 8 : 16, runs = 16 / qs;
        const int jq = q % qs, run = q / qs, per = (n_pieces + runs - 1) / runs;
        const int i0 = min(n_pieces, run * per), i1 = min(n_pieces, i0 + per);
        const int jx = min(EX * x, D - EX);
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < EX; ++i) acc[i] = 0.f;
        if (jq < n_q) {
            constexpr int U = 8;                                     // pieces requested before the first is used
            for (int i = i0; i < i1; i += U) {
                f32x2 pm[U], v[U][EX / 2];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float *p = part_at(min(i + u, i1 - 1));
                    pm[u] = get(p + 16 * D + 2 * jq);
#pragma unroll
                    for (int e = 0; e < EX / 2; ++e) v[u][e] = get(p + jq * D + jx + 2 * e);
                }
                float next = top;
#pragma unroll
                for (int u = 0; u < U; ++u) next = fmaxf(next, pm[u][0]);
                const float keep = __builtin_amdgcn_exp2f(top - finite(next));
                top = next;
                sum *= keep;
#pragma unroll
                for (int e = 0; e < EX; ++e) acc[e] *= keep;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float f = i + u < i1 ? __builtin_amdgcn_exp2f(pm[u][0] - finite(top)) : 0.f;
                    sum += f * pm[u][1];
#pragma unroll
                    for (int e = 0; e < EX; ++e) acc[e] += f * v[u][e / 2][e % 2];
                }
            }
        }
        __syncthreads();
        float *s_run = &s_o[0][0][0];                                // [16][DP]
#pragma unroll
        for (int e = 0; e < EX; ++e) s_run[q * DP + EX * x + e] = acc[e];
        if (x == 0) {
            s_m[0][q] = top;
            s_l[0][q] = sum;
        }
        __syncthreads();
        if (q >= n_q) return;
        top = -INFINITY;
        for (int r = 0; r < runs; ++r) top = fmaxf(top, s_m[0][q + r * qs]);
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < EX; ++e) acc[e] = 0.f;
        for (int r = 0; r < runs; ++r) {
            const float f = __builtin_amdgcn_exp2f(s_m[0][q + r * qs] - finite(top));
            sum += f * s_l[0][q + r * qs];
#pragma unroll
            for (int e = 0; e < EX; ++e) acc[e] += f * s_run[(q + r * qs) * DP + EX * x + e];
        }
        finish(q, x, top, sum, acc);
    };

    if (!RANGES || range == 0) {
        const Piece at = find_piece(a.n_seqs, (uint32_t)item, len_of, pieces_of);
        if (at.seq < 0) return;
        const int piece = scalar(at.piece), len = scalar(at.size), n_pieces = scalar((int)pieces_of(len));
        const int piece_keys = scalar((int)((steps_of(len) + n_pieces - 1) / n_pieces) * step);        // pieces of a sequence are of a size
        const int k0 = min(len, piece * piece_keys), k1 = min(len, k0 + piece_keys);
        float *first = a.part + ((item - piece) * (long)heads + hg) * piece_size;
        run(scalar(at.seq), len, piece, n_pieces, k0, k1, [&](int i) { return first + i * (heads * piece_size); });
        return;
    }
    if constexpr (RANGES) {
        const Piece at = find_piece(a.n_seqs, (uint32_t)item * range, len_of, [&](int len) { return steps_of(len) + 1; });
        int b = scalar(at.seq), len = scalar(at.size), from = scalar(at.piece), left = (int)range, r = (int)range;
        for (;;) {
            const int steps = scalar((int)steps_of(len) + 1), to = min(steps, from + left), start = item * r + (r - left) - from;
            const int w0 = start / r, w1 = (start + steps - 1) / r;          // first and last of the workgroups that have some of the sequence
            float *first = a.part + (2 * w0 * (long)heads + hg) * piece_size;
            run(b, len, item - w0, w1 - w0 + 1, min(len, max(0, from - 1) * step), min(len, (to - 1) * step),
                [&](int i) { return first + (2 * i + (i == 0)) * (heads * piece_size); });
            left -= to - from;
            if (left == 0 || ++b >= a.n_seqs) return;
            from = 0;
            len = scalar(len_of(b));
            __syncthreads();                      // LDS of the piece before
        }
    }
}

}  // namespace

hipError_t launch_decode(const DecodeArgs &a, hipStream_t s) {
    // Whether the lengths that the table of pages has room for are enough for ranges.  Heads between 16 and 128 run as the next of 64 and 128, in pieces only: no
    // configuration of this library has them, and more kernels were not built for them.  64 sequences of 33 to 16384 keys, bf16, heads of 128 134 us, 5.6 TB/s; of 112 158, 4.2;
    // of 96 135, 4.2; of 80 132, 3.6; of 64 68, 5.6.
    const long steps = (((long)a.seq_pages << a.c.page_shift) + kWaves * kBlock - 1) / (kWaves * kBlock) + 1, heads = (long)a.c.Hk * group_tiles(a.Hq, a.c.Hk);
    const bool ranges = a.n_seqs > 1 && a.n_seqs * steps * heads > kRangeWgs * (kFewestRange - 1);
    const auto run = [&](auto dp, auto fp8) {
        in_launches(decode_workgroups(a), [&](int at, unsigned n) {
            const dim3 grid(n), block(kWaves * 64);
            if (a.c.D == dp && ranges) decode_piece<dp, fp8, true, true><<<grid, block, 0, s>>>(a, at);
            else if (a.c.D == dp) decode_piece<dp, fp8, true, false><<<grid, block, 0, s>>>(a, at);
            else decode_piece<dp, fp8, false, false><<<grid, block, 0, s>>>(a, at);
        });
    };
    typedef std::integral_constant<int, 64> D64;
    typedef std::integral_constant<int, 128> D128;
    if (a.c.D <= 64 && a.fp8) run(D64{}, std::true_type{});
    else if (a.c.D <= 64) run(D64{}, std::false_type{});
    else if (a.fp8) run(D128{}, std::true_type{});
    else run(D128{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace qattn
