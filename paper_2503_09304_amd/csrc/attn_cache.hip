// attn_append and attn_read: rotary positions and the paged cache of keys and values.
//
// Both move rows of heads: nothing is used twice, so the bound is HBM.  A row (one head of one token) belongs to 4 or 8 lanes
// (dim up to 64, 128), 16 elements a lane in two 16-byte pieces, chosen so that a lane holds both elements of each of its pairs:
// pieces 2p and 2p + 1, or, where pairs are half a rotation apart, pieces p and p + rot/16.  So rotation is inside the lane, and the
// largest element of a row, which its 8-bit scale follows, is 2 or 3 exchanges between neighbouring lanes away.
//
// Angles: pos * f in units of half turns in 64 bits, taken to the nearest quarter turn there, the rest (at most a quarter of a
// half turn, exact to 2^-27) in fp32 sincospi.  Positions of 2^20 keep 33 bits of their angle this way; in fp32 they would
// keep 4.  One thread per (token, pair) forms them, all heads of the token read them from LDS.
//
// Rows go past the caches (non-temporal loads and stores where nothing is read twice: 9826 tokens 55.7 -> 52.1 us).  Measured: 9826 tokens of 32 + 8 + 8 heads
// of 128 into a bf16 cache 51 us, 4.7 TB/s (a copy of 4 GiB by the vendor's library 4.9), into an fp8 cache and read back 64, 4.4; one token 4.0 us; 40276 fp8 tokens read 54 us, 4.6 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "qattn_internal.h"

namespace qattn {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// cos and sin of pos * f.
__device__ __forceinline__ float2 angle(int pos, double f, float mscale) {
    const double t = (double)pos * (f * 0.31830988618379067154);       // half turns
    const double q = rint(t * 2.0);
    const float r = (float)(t - q * 0.5);
    float s, c;
    sincospif(r, &s, &c);
    const int n = (int)((long long)q & 3);
    const float c1 = n & 1 ? s : c, s1 = n & 1 ? c : s;
    return {((n + 1) & 2 ? -c1 : c1) * mscale, (n & 2 ? -s1 : s1) * mscale};
}

// Page of token `pos` of sequence `seq`, or -1.
__device__ __forceinline__ int page_of(const Cache &c, const int32_t *pages, int n_seqs, int seq_pages, int seq, int pos) {
    if (seq < 0 || seq >= n_seqs || pos < 0 || (pos >> c.page_shift) >= seq_pages) return -1;
    const int p = pages[(long)seq * seq_pages + (pos >> c.page_shift)];
    return p >= 0 && p < c.n_pages ? p : -1;
}

// Row of head h of a slot, in rows of the cache.
__device__ __forceinline__ long cache_row(const Cache &c, int page, int h, int pos) {
    return (((long)page * c.Hk + h) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// Scale byte of a row whose largest element has the bits `m` (sign cleared): 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(uint32_t m) {
    const int b = (int)(m >> 23) - 8 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b < 1 ? 1 : b;
}

template <int LPR>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
    return m;
}

// 8 bf16 elements as e4m3 codes of element * 2^(127 - byte), at most `most`.
__device__ __forceinline__ u32x2 to_fp8(const u32x4 &x, float inv, float most) {
    const auto one = [&](float v) { return __builtin_amdgcn_fmed3f(v * inv, -most, most); };
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(one(lo_f(x[2 * i])), one(hi_f(x[2 * i])), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(one(lo_f(x[2 * i + 1])), one(hi_f(x[2 * i + 1])), w, true);
        r[i] = (uint32_t)w;
    }
    return r;
}

// 8 e4m3 codes as bf16: exact.
__device__ __forceinline__ u32x4 from_fp8(const u32x2 &x, float scale) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false));
        r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true));
    }
    return r;
}

constexpr int kThreads = 256;

// The rows of a workgroup's tokens, LPR lanes each, dealt out to its threads: thread `tid` has rows tid / LPR, that + 256 / LPR, ...
template <int LPR>
struct RowWalk {
    int tt, r;                        // token of the workgroup, row of it
    int rows;
    __device__ __forceinline__ RowWalk(int tid, int rows_) : tt(0), r(tid / LPR), rows(rows_) { wrap(); }
    __device__ __forceinline__ void next() {
        r += kThreads / LPR;
        wrap();
    }
    __device__ __forceinline__ void wrap() {
        while (r >= rows) {
            r -= rows;
            ++tt;
        }
    }
};

// TOK tokens a workgroup.
template <int LPR, int TOK>
__global__ __launch_bounds__(kThreads) void append_rows(const AppendArgs a) {
    __shared__ float2 cs[TOK][kMaxDim / 2];
    __shared__ long slot[TOK];                    // first key/value head's row of the token in the cache; -1: it is not written there
    __shared__ int padding[TOK];
    const int tid = threadIdx.x, p = tid % LPR;
    const int D = a.c.D, Hk = a.c.Hk, rows = a.Hq + 2 * Hk, half = a.rot / 2;
    const bool turned = p < a.rot / 16, in = p < D / 16;
    // the lane's two pieces of 8 elements
    const int c0 = (a.interleaved || !turned ? 2 * p : p) * 8, c1 = !a.interleaved && turned ? (p + a.rot / 16) * 8 : c0 + 8;
    for (long t0 = (long)blockIdx.x * TOK; t0 < a.n_tokens; t0 += (long)gridDim.x * TOK) {
        const int nt = (int)min((long)TOK, a.n_tokens - t0);
        // Loads of the first rows do not wait for the angles.
        constexpr int U = 2;                      // rows that are requested before the first is used (three: 9826 tokens 61.7 us instead of 55.7)
        RowWalk<LPR> walk(tid, rows);
        u32x4 x0[U], x1[U];
        int tt[U], r[U];
        const auto request = [&]() {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                tt[u] = walk.tt;
                r[u] = walk.r;
                walk.next();
                const int t = min(tt[u], nt - 1), kind = (r[u] >= a.Hq) + (r[u] >= a.Hq + Hk);        // q, k, v
                const int h = r[u] - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + Hk);
                const Rows &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
                const uint16_t *from = src.p + (t0 + t) * src.ts + h * src.hs;
                x0[u] = *reinterpret_cast<const u32x4 *>(from + (in ? c0 : 0));
                x1[u] = *reinterpret_cast<const u32x4 *>(from + (in ? c1 : 0));
            }
        };
        request();
        __syncthreads();                                                  // cs and slot of the tokens before
        if (tid < nt) {
            const long t = t0 + tid;
            const int pos = a.pos[t];
            const int page = page_of(a.c, a.pages, a.n_seqs, a.seq_pages, a.seq ? a.seq[t] : (int)t, pos);
            padding[tid] = pos < 0;
            slot[tid] = page < 0 ? -1 : cache_row(a.c, page, 0, pos);
            if (page < 0 && pos >= 0 && a.bad != nullptr) atomicAdd(a.bad, 1);
        }
        for (int i = tid; i < nt * half; i += kThreads) {
            const int t = i / half, q = i - t * half;
            cs[t][q] = angle(a.pos[t0 + t], a.inv_freq[q], a.mscale);
        }
        __syncthreads();
        // Whole waves go round, for the exchange between the lanes of a row.
        for (int first = 0; first < nt * rows; first += U * (kThreads / LPR)) {
            if (first > 0) request();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool active = in && tt[u] < nt && !padding[min(tt[u], nt - 1)];
                const int t = min(tt[u], nt - 1), kind = (r[u] >= a.Hq) + (r[u] >= a.Hq + Hk);
                const int h = r[u] - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + Hk);
                u32x4 y0 = x0[u], y1 = x1[u];
                if (kind != 2 && turned) {
                    const float2 *w = &cs[t][8 * p];
                    if (a.interleaved) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 e = w[i], f = w[i + 4];
                            y0[i] = pack_bf16(lo_f(y0[i]) * e.x - hi_f(y0[i]) * e.y, hi_f(y0[i]) * e.x + lo_f(y0[i]) * e.y);
                            y1[i] = pack_bf16(lo_f(y1[i]) * f.x - hi_f(y1[i]) * f.y, hi_f(y1[i]) * f.x + lo_f(y1[i]) * f.y);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 e = w[2 * i], f = w[2 * i + 1];
                            const float al = lo_f(y0[i]), ah = hi_f(y0[i]), bl = lo_f(y1[i]), bh = hi_f(y1[i]);
                            y0[i] = pack_bf16(al * e.x - bl * e.y, ah * f.x - bh * f.y);
                            y1[i] = pack_bf16(bl * e.x + al * e.y, bh * f.x + ah * f.y);
                        }
                    }
                }
                const Rows &dst = kind == 0 ? a.qo : a.ko;
                if (active && kind != 2 && dst.p != nullptr) {
                    uint16_t *to = dst.p + (t0 + t) * dst.ts + h * dst.hs;
                    __builtin_nontemporal_store(y0, reinterpret_cast<u32x4 *>(to + c0));
                    __builtin_nontemporal_store(y1, reinterpret_cast<u32x4 *>(to + c1));
                }
                const long at = slot[t];
                const bool kept = active && kind != 0 && at >= 0;
                const long row = at + ((long)h << a.c.page_shift);
                if (a.fp8) {
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        m = max(m, max(y0[i] & 0x7FFF0000u, (y0[i] << 16) & 0x7FFF0000u));
                        m = max(m, max(y1[i] & 0x7FFF0000u, (y1[i] << 16) & 0x7FFF0000u));
                    }
                    const int byte = scale_byte(row_max<LPR>(in ? m : 0u));
                    if (kept) {
                        uint8_t *to = (kind == 1 ? a.c.k : a.c.v) + row * D;
                        const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
                        const float most = byte == 247 ? 240.f : 448.f;       // 256 * 2^(247 - 127) would be over the largest bf16
                        *reinterpret_cast<u32x2 *>(to + c0) = to_fp8(y0, inv, most);
                        *reinterpret_cast<u32x2 *>(to + c1) = to_fp8(y1, inv, most);
                        if (p == 0) (kind == 1 ? a.c.ks : a.c.vs)[row] = (uint8_t)byte;
                    }
                } else if (kept) {
                    uint16_t *to = (uint16_t *)(kind == 1 ? a.c.k : a.c.v) + row * D;
                    __builtin_nontemporal_store(y0, reinterpret_cast<u32x4 *>(to + c0));
                    __builtin_nontemporal_store(y1, reinterpret_cast<u32x4 *>(to + c1));
                }
            }
        }
    }
}

// Rows of the tokens from `first` on, n in all, LPR lanes each, U a thread, requested before the first is used.  Every lane finds its token's slot for
// itself (through LDS, a workgroup's tokens at a time, all wait for the slots before they ask for a row: 40276 fp8 tokens 62 us instead of 55).
template <int LPR, int U>
__global__ __launch_bounds__(kThreads) void read_rows(const ReadArgs a, long first, uint32_t n) {
    const int D = a.c.D, Hk = a.c.Hk, p = threadIdx.x % LPR;
    const uint32_t row0 = blockIdx.x * (U * kThreads / LPR) + threadIdx.x / LPR;
    if (p >= D / 16) return;
    u32x4 x0[U], x1[U];
    float scale[U];
    bool none[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t row = min(row0 + u * (kThreads / LPR), n - 1), tt = row / (2 * Hk), r = row - tt * (2 * Hk);
        const long t = first + tt;
        const int kind = r >= (uint32_t)Hk, h = kind ? r - Hk : r, pos = a.pos[t];
        const int page = page_of(a.c, a.pages, a.n_seqs, a.seq_pages, a.seq ? a.seq[t] : (int)t, pos);
        none[u] = page < 0;
        if (page < 0 && pos >= 0 && r == 0 && p == 0 && a.bad != nullptr && row0 + u * (kThreads / LPR) < n) atomicAdd(a.bad, 1);
        const long at = page < 0 ? 0 : cache_row(a.c, page, h, pos);
        const uint8_t *pool = kind ? a.c.v : a.c.k;
        if (a.fp8) {
            x0[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(pool + at * D + p * 16));
            scale[u] = __uint_as_float((uint32_t)(kind ? a.c.vs : a.c.ks)[at] << 23);
        } else {
            const u32x4 *from = reinterpret_cast<const u32x4 *>((const uint16_t *)pool + at * D + p * 16);
            x0[u] = __builtin_nontemporal_load(from);
            x1[u] = __builtin_nontemporal_load(from + 1);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t row = row0 + u * (kThreads / LPR);
        if (row >= n) return;
        const uint32_t tt = row / (2 * Hk), r = row - tt * (2 * Hk);
        const int kind = r >= (uint32_t)Hk, h = kind ? r - Hk : r;
        u32x4 y0 = x0[u], y1 = x1[u];
        if (a.fp8) {
            y1 = from_fp8(u32x2{y0[2], y0[3]}, scale[u]);
            y0 = from_fp8(u32x2{y0[0], y0[1]}, scale[u]);
        }
        if (none[u]) y0 = y1 = u32x4{0, 0, 0, 0};
        const Rows &dst = kind ? a.vo : a.ko;
        u32x4 *to = reinterpret_cast<u32x4 *>(dst.p + (first + tt) * dst.ts + h * dst.hs + p * 16);
        __builtin_nontemporal_store(y0, to);
        __builtin_nontemporal_store(y1, to + 1);
    }
}

// Tokens a workgroup: one where that is what spreads them over the chip, else four (9826 tokens of 48 heads of 128: two 60 us, four 55.7, eight 56.7; 2000
// tokens 12.9, 13.2, 18.2).
constexpr long kFewTokens = 1024, kMostWgs = 1 << 20;
template <class F>
void by_tokens(int n_tokens, F &&launch) {
    if (n_tokens <= kFewTokens) launch(std::integral_constant<int, 1>{}, dim3((unsigned)n_tokens));
    else launch(std::integral_constant<int, 4>{}, dim3((unsigned)std::min<long>(((long)n_tokens + 3) / 4, kMostWgs)));
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t s) {
    by_tokens(a.n_tokens, [&](auto tok, dim3 grid) {
        if (a.c.D <= 64) append_rows<4, tok><<<grid, dim3(kThreads), 0, s>>>(a);
        else append_rows<8, tok><<<grid, dim3(kThreads), 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, hipStream_t s) {
    const int lpr = a.c.D <= 64 ? 4 : 8, per = kThreads / lpr, rows = 2 * a.c.Hk;
    const long most = (1l << 23) / rows;          // tokens of a launch, so that its rows and threads stay within 32 bits
    for (long t = 0; t < a.n_tokens; t += most) {
        const uint32_t n = (uint32_t)(std::min(most, a.n_tokens - t) * rows), wgs = (n + per - 1) / per;
        // Two rows a thread where one would take more than 8 workgroups a CU (40276 fp8 tokens 55 us, one row 58, three 57; 509 bf16 tokens of 16 heads of 64,
        // 254 workgroups, 3.6 and with one row 3.2).
        const auto run = [&](auto l, auto u) { read_rows<l, u><<<dim3((wgs + u - 1) / u), dim3(kThreads), 0, s>>>(a, t, n); };
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        typedef std::integral_constant<int, 4> Four;
        typedef std::integral_constant<int, 8> Eight;
        if (lpr == 4 && wgs <= 2048) run(Four{}, One{});
        else if (lpr == 4) run(Four{}, Two{});
        else if (wgs <= 2048) run(Eight{}, One{});
        else run(Eight{}, Two{});
    }
    return hipGetLastError();
}

}  // namespace qattn
