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
// Work: sequences are cut into pieces of equal size so that about kDecodeWgs workgroups share all keys, whatever the lengths (each finds
// its piece from the lengths, attn_pieces.h).  A workgroup's 4 waves take its blocks of 32 keys in turn, each with its own
// running maximum and sum, and are joined in LDS; pieces of a sequence leave fp32 sums in the workspace and the last of
// them to arrive joins all in the order of the pieces.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_pieces.h"
#include "qattn_internal.h"

namespace qattn {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kBlock = 32;                       // keys of a wave's step

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

// m where it stands for something, 0 for a row that has seen no key: x - finite(m) is then -inf, and its exponential 0.
__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }

template <int DP, bool FP8>
__global__ __launch_bounds__(kWaves * 64) void decode_piece(const DecodeArgs a) {
    constexpr int KS = DP / 32;                       // MFMA steps of a score
    constexpr int DT = DP / 16;                       // d tiles of the output
    constexpr int VE = FP8 ? DP / 16 : 4;             // elements of a value load: d = VE * (lane % 16) + 0 .. VE - 1 (+ 64 u)
    constexpr int VU = DT / VE;                       // value loads of a key's row
    __shared__ float s_o[kWaves][16][DP + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int GT = group_tiles(a.Hq, a.c.Hk), G = a.Hq / a.c.Hk;
    const int hk = blockIdx.x % a.c.Hk, gt = (blockIdx.x / a.c.Hk) % GT, item = blockIdx.x / (a.c.Hk * GT);
    const int P = 1 << a.c.page_shift, most = a.seq_pages << a.c.page_shift;
    const auto len_of = [&](int b) { return min(max(a.lens[b], 0), most); };

    // keys of a piece: what makes kDecodeWgs of them in all, in whole steps of the workgroup
    long total = 0;
    for (int b = lane; b < a.n_seqs; b += 64) total += len_of(b);
    total = wave_sum(total);
    const int shares = a.pieces - a.n_seqs;
    const long share = min((total + shares - 1) / shares, 1l << 30);
    const int step = kWaves * kBlock;
    const int piece_keys = (int)max((long)2 * step, (share + step - 1) / step * step);
    // a sequence without keys still has a piece: its zeros are somebody's to write
    const int2 at = find_piece(a.n_seqs, item, [&](int b) { return max(1, (len_of(b) + piece_keys - 1) / piece_keys); });
    const int b = __builtin_amdgcn_readfirstlane(at.x), piece = __builtin_amdgcn_readfirstlane(at.y);
    if (b < 0) return;
    const int len = len_of(b), n_pieces = max(1, (len + piece_keys - 1) / piece_keys);
    const int k0 = piece * piece_keys, k1 = min(len, k0 + piece_keys);
    const int32_t *pages = a.pages + (long)b * a.seq_pages;
    if (a.bad != nullptr && tid == 0 && hk == 0 && gt == 0 && piece == 0 && a.lens[b] != len) atomicAdd(a.bad, 1);

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
    const int esz = FP8 ? 1 : 2;

    for (int k = k0 + wave * kBlock; k < k1; k += step) {
        // rows (of the cache) of the first keys of the two tiles of 16; -1: no keys
        long row[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = k + 16 * t;
            int page = -1;
            if (key < k1) {
                page = pages[key >> a.c.page_shift];
                if (page < 0 || page >= a.c.n_pages) {
                    page = -1;
                    if (a.bad != nullptr && lane == 0 && gt == 0) atomicAdd(a.bad, 1);
                }
            }
            row[t] = page < 0 ? -1 : (((long)page * a.c.Hk + hk) << a.c.page_shift) + (key & (P - 1));
        }
        const bool whole = k + kBlock <= k1 && row[0] >= 0 && row[1] >= 0;
        u32x4 kf[2][KS];
        uint32_t vr[2][4][VU][VE / 4 * (FP8 ? 1 : 2)];
        uint32_t ksc[2], vsc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const long at_row = row[t] < 0 ? 0 : row[t];
            const uint8_t *kp = a.c.k + (at_row + col) * a.c.D * esz;
#pragma unroll
            for (int s = 0; s < (FP8 ? KS / 2 : KS); ++s) {
                const int byte = 64 * s + 16 * g;
                const u32x4 x = byte < a.c.D * esz ? *reinterpret_cast<const u32x4 *>(kp + byte) : u32x4{0, 0, 0, 0};
                if constexpr (FP8) {
                    kf[t][2 * s] = u32x4{fp8_pair(x[0], false), fp8_pair(x[0], true), fp8_pair(x[1], false), fp8_pair(x[1], true)};
                    kf[t][2 * s + 1] = u32x4{fp8_pair(x[2], false), fp8_pair(x[2], true), fp8_pair(x[3], false), fp8_pair(x[3], true)};
                } else {
                    kf[t][s] = x;
                }
            }
            if constexpr (FP8) {
                ksc[t] = *reinterpret_cast<const uint32_t *>(a.c.ks + at_row + 4 * g);
                vsc[t] = *reinterpret_cast<const uint32_t *>(a.c.vs + at_row + 4 * g);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const long at_row = row[t] < 0 ? 0 : row[t];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint8_t *vp = a.c.v + (at_row + 4 * g + r) * a.c.D * esz;
#pragma unroll
                for (int u = 0; u < VU; ++u) {
                    const int d = 64 * u + VE * col;
                    if constexpr (FP8 && VE == 4) {
                        vr[t][r][u][0] = d < a.c.D ? *reinterpret_cast<const uint32_t *>(vp + d) : 0u;
                    } else {
                        const u32x2 x = d < a.c.D ? *reinterpret_cast<const u32x2 *>(vp + d * esz) : u32x2{0, 0};
                        vr[t][r][u][0] = x[0];
                        vr[t][r][u][1] = x[1];
                    }
                }
            }
        }
        // scores of 2 x 4 keys of this lane's column
        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) c = mma(kf[t][i], qf[i], c);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * t + r] = FP8 ? c[r] * power(ksc[t], r) * a.scale_log2 : c[r] * a.scale_log2;
        }
        if (!whole) {                                     // keys that are none: no score, and zeros for whatever their values hold
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool none = row[t] < 0 || k + 16 * t + 4 * g + r >= k1;
                    s[4 * t + r] = none ? -INFINITY : s[4 * t + r];
                    if (FP8 && none) vsc[t] &= ~(0xFFu << (8 * r));
#pragma unroll
                    for (int u = 0; u < VU; ++u)
#pragma unroll
                        for (int i = 0; i < VE / 4 * (FP8 ? 1 : 2); ++i) vr[t][r][u][i] = none ? 0u : vr[t][r][u][i];
                }
            }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(m, column_max(top));
        const float base = finite(top), keep = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= keep;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(s[i] - base);
            l += p[i];
            if constexpr (FP8) p[i] *= power(vsc[i / 4], i % 4);
        }
        const u32x4 pf = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
        // tile (u, e): d = 64 u + VE * (lane % 16) + e
#pragma unroll
        for (int u = 0; u < VU; ++u) {
#pragma unroll
            for (int w = 0; w < VE / 4 * (FP8 ? 1 : 2); ++w) {
                if constexpr (FP8) {
                    // elements 4w .. 4w + 3: bytes of two keys side by side, then two at a time to bf16
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t x = vr[j / 2][2 * (j & 1)][u][w], y = vr[j / 2][2 * (j & 1) + 1][u][w];
                        lo[j] = __builtin_amdgcn_perm(y, x, 0x05010400u);
                        hi[j] = __builtin_amdgcn_perm(y, x, 0x07030602u);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t *src = e < 2 ? lo : hi;
                        const u32x4 vf = {fp8_pair(src[0], e & 1), fp8_pair(src[1], e & 1), fp8_pair(src[2], e & 1), fp8_pair(src[3], e & 1)};
                        f32x4 &acc = o[VE * u + 4 * w + e];
                        acc = mma(vf, pf, acc * keep);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        u32x4 vf;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            vf[j] = __builtin_amdgcn_perm(vr[j / 2][2 * (j & 1) + 1][u][w], vr[j / 2][2 * (j & 1)][u][w], e ? 0x07060302u : 0x05040100u);
                        f32x4 &acc = o[VE * u + 2 * w + e];
                        acc = mma(vf, pf, acc * keep);
                    }
                }
            }
        }
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

    // the four waves' sums joined: thread (q, x) has DP / 16 elements of query q
    const int q = tid >> 4, x = tid & 15;
    const int D = a.c.D;
    float top = s_m[0][q];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][q]);
    float sum = 0.f, acc[DT] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][q] - finite(top));
        sum += f * s_l[w][q];
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] += f * s_o[w][q][x + 16 * i];
    }
    const int head_q = hk * G + gt * 16 + q;
    const bool mine = gt * 16 + q < G;
    if (n_pieces > 1) {
        const int heads = a.c.Hk * GT, hg = gt * a.c.Hk + hk;
        float *part = a.part + ((long)item * heads + hg) * 16 * (D + 2);
        if (mine) {
            float *to = part + q * (D + 2);
#pragma unroll
            for (int i = 0; i < DT; ++i)
                if (x + 16 * i < D) to[x + 16 * i] = acc[i];
            if (x == 0) {
                to[D] = top;
                to[D + 1] = sum;
            }
        }
        __threadfence();                                  // the piece is visible to the device before it is counted
        __syncthreads();
        if (tid == 0) {
            int32_t *count = a.arrived + (long)b * heads + hg;
            const int n = __hip_atomic_fetch_add(count, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
            s_last = n == n_pieces - 1;
            if (n == n_pieces - 1) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!s_last) return;
        __threadfence();
        if (!mine) return;
        const long stride = (long)heads * 16 * (D + 2);
        const float *from = part - piece * stride + q * (D + 2);      // the sequence's first piece
        top = -INFINITY;
        for (int i = 0; i < n_pieces; ++i) top = fmaxf(top, from[i * stride + D]);
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = 0.f;
        for (int i = 0; i < n_pieces; ++i) {
            const float *p = from + i * stride;
            const float f = __builtin_amdgcn_exp2f(p[D] - finite(top));
            sum += f * p[D + 1];
#pragma unroll
            for (int j = 0; j < DT; ++j)
                if (x + 16 * j < D) acc[j] += f * p[x + 16 * j];
        }
    }
    if (!mine) return;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    uint16_t *to = a.o.p + (long)b * a.o.ts + (long)head_q * a.o.hs;
#pragma unroll
    for (int i = 0; i < DT; ++i)
        if (x + 16 * i < D) to[x + 16 * i] = __builtin_bit_cast(uint16_t, (__bf16)(acc[i] * inv));
    if (a.lse != nullptr && x == 0) a.lse[(long)b * a.Hq + head_q] = sum > 0.f ? (top + __log2f(sum)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace

hipError_t launch_decode(const DecodeArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.pieces * a.c.Hk * group_tiles(a.Hq, a.c.Hk))), block(kWaves * 64);
    if (a.c.D <= 64) {
        if (a.fp8) decode_piece<64, true><<<grid, block, 0, s>>>(a);
        else decode_piece<64, false><<<grid, block, 0, s>>>(a);
    } else {
        if (a.fp8) decode_piece<128, true><<<grid, block, 0, s>>>(a);
        else decode_piece<128, false><<<grid, block, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace qattn
