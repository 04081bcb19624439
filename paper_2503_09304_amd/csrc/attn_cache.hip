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
#include <hip/hip_runtime.h>

#include <algorithm>

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

// TOK tokens a workgroup.
template <int LPR, int TOK>
__global__ __launch_bounds__(kThreads) void append_rows(const AppendArgs a) {
    __shared__ float2 cs[TOK][kMaxDim / 2];
    const int tid = threadIdx.x;
    const int pairs = a.c.D / 16, rows = a.Hq + 2 * a.c.Hk, half = a.rot / 2;
    for (long t0 = (long)blockIdx.x * TOK; t0 < a.n_tokens; t0 += (long)gridDim.x * TOK) {
        const int nt = (int)min((long)TOK, a.n_tokens - t0);
        __syncthreads();                                                  // cs of the tokens before
        for (int i = tid; i < nt * half; i += kThreads) {
            const int t = i / half, p = i - t * half;
            cs[t][p] = angle(a.pos[t0 + t], a.inv_freq[p], a.mscale);
        }
        __syncthreads();
        const int items = nt * rows * LPR;
        for (int it = tid; it < (items + 63) / 64 * 64; it += kThreads) {       // whole waves, for the exchange
            const int row = min(it / LPR, nt * rows - 1), p = it % LPR;
            const int tt = row / rows, r = row - tt * rows;
            const long t = t0 + tt;
            const int pos = a.pos[t];
            const bool active = it < items && p < pairs && pos >= 0;
            const int kind = r < a.Hq ? 0 : r < a.Hq + a.c.Hk ? 1 : 2;        // q, k, v
            const int h = kind == 0 ? r : kind == 1 ? r - a.Hq : r - a.Hq - a.c.Hk;
            const bool turn = kind != 2 && p < a.rot / 16;
            // the lane's two pieces of 8 elements
            const int c0 = a.interleaved || p >= a.rot / 16 ? 2 * p : p, c1 = !a.interleaved && p < a.rot / 16 ? p + a.rot / 16 : c0 + 1;
            u32x4 x0{0, 0, 0, 0}, x1{0, 0, 0, 0};
            if (active) {
                const Rows &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
                const uint16_t *from = src.p + t * src.ts + h * src.hs;
                x0 = *reinterpret_cast<const u32x4 *>(from + c0 * 8);
                x1 = *reinterpret_cast<const u32x4 *>(from + c1 * 8);
                if (turn) {
                    const float2 *w = &cs[tt][8 * p];
                    if (a.interleaved) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 u = w[i], v = w[i + 4];
                            x0[i] = pack_bf16(lo_f(x0[i]) * u.x - hi_f(x0[i]) * u.y, hi_f(x0[i]) * u.x + lo_f(x0[i]) * u.y);
                            x1[i] = pack_bf16(lo_f(x1[i]) * v.x - hi_f(x1[i]) * v.y, hi_f(x1[i]) * v.x + lo_f(x1[i]) * v.y);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 u = w[2 * i], v = w[2 * i + 1];
                            const float al = lo_f(x0[i]), ah = hi_f(x0[i]), bl = lo_f(x1[i]), bh = hi_f(x1[i]);
                            x0[i] = pack_bf16(al * u.x - bl * u.y, ah * v.x - bh * v.y);
                            x1[i] = pack_bf16(bl * u.x + al * u.y, bh * v.x + ah * v.y);
                        }
                    }
                }
                const Rows &dst = kind == 0 ? a.qo : a.ko;
                if (kind != 2 && dst.p != nullptr) {
                    uint16_t *to = dst.p + t * dst.ts + h * dst.hs;
                    *reinterpret_cast<u32x4 *>(to + c0 * 8) = x0;
                    *reinterpret_cast<u32x4 *>(to + c1 * 8) = x1;
                }
            }
            int page = -1;
            if (it < items && kind != 0 && pos >= 0) {
                page = page_of(a.c, a.pages, a.n_seqs, a.seq_pages, a.seq ? a.seq[t] : (int)t, pos);
                if (page < 0 && kind == 1 && h == 0 && p == 0 && a.bad != nullptr) atomicAdd(a.bad, 1);
            }
            if (a.fp8) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m = max(m, max(x0[i] & 0x7FFF0000u, (x0[i] << 16) & 0x7FFF0000u));
                    m = max(m, max(x1[i] & 0x7FFF0000u, (x1[i] << 16) & 0x7FFF0000u));
                }
                const int byte = scale_byte(row_max<LPR>(m));
                if (page >= 0 && active) {
                    const long row_at = cache_row(a.c, page, h, pos);
                    uint8_t *to = (kind == 1 ? a.c.k : a.c.v) + row_at * a.c.D;
                    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
                    const float most = byte == 247 ? 240.f : 448.f;       // 256 * 2^(247 - 127) would be over the largest bf16
                    *reinterpret_cast<u32x2 *>(to + c0 * 8) = to_fp8(x0, inv, most);
                    *reinterpret_cast<u32x2 *>(to + c1 * 8) = to_fp8(x1, inv, most);
                    if (p == 0) (kind == 1 ? a.c.ks : a.c.vs)[row_at] = (uint8_t)byte;
                }
            } else if (page >= 0 && active) {
                uint16_t *to = (uint16_t *)(kind == 1 ? a.c.k : a.c.v) + cache_row(a.c, page, h, pos) * a.c.D;
                *reinterpret_cast<u32x4 *>(to + c0 * 8) = x0;
                *reinterpret_cast<u32x4 *>(to + c1 * 8) = x1;
            }
        }
    }
}

template <int LPR>
__global__ __launch_bounds__(kThreads) void read_rows(const ReadArgs a, long items) {
    const int pairs = a.c.D / 16, rows = 2 * a.c.Hk;
    for (long it = (long)blockIdx.x * kThreads + threadIdx.x; it < items; it += (long)gridDim.x * kThreads) {
        const long row = it / LPR;
        const int p = (int)(it % LPR);
        if (p >= pairs) continue;
        const long t = row / rows;
        const int r = (int)(row - t * rows), kind = r >= a.c.Hk, h = kind ? r - a.c.Hk : r;
        const int pos = a.pos[t];
        const int page = page_of(a.c, a.pages, a.n_seqs, a.seq_pages, a.seq ? a.seq[t] : (int)t, pos);
        u32x4 x0{0, 0, 0, 0}, x1{0, 0, 0, 0};
        if (page >= 0) {
            const long row_at = cache_row(a.c, page, h, pos);
            const uint8_t *pool = kind ? a.c.v : a.c.k;
            if (a.fp8) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(pool + row_at * a.c.D + p * 16);
                const float scale = __uint_as_float((uint32_t)(kind ? a.c.vs : a.c.ks)[row_at] << 23);
                x0 = from_fp8(u32x2{w[0], w[1]}, scale);
                x1 = from_fp8(u32x2{w[2], w[3]}, scale);
            } else {
                const u32x4 *from = reinterpret_cast<const u32x4 *>((const uint16_t *)pool + row_at * a.c.D + p * 16);
                x0 = from[0];
                x1 = from[1];
            }
        } else if (pos >= 0 && r == 0 && p == 0 && a.bad != nullptr) {
            atomicAdd(a.bad, 1);
        }
        const Rows &dst = kind ? a.vo : a.ko;
        u32x4 *to = reinterpret_cast<u32x4 *>(dst.p + t * dst.ts + h * dst.hs + p * 16);
        to[0] = x0;
        to[1] = x1;
    }
}

template <int LPR>
void append_n(const AppendArgs &a, hipStream_t s) {
    const long most = 1 << 20;                    // workgroups; beyond that they take several turns
    if (a.n_tokens <= 1024) {
        append_rows<LPR, 1><<<dim3((unsigned)a.n_tokens), dim3(kThreads), 0, s>>>(a);
    } else {
        append_rows<LPR, 4><<<dim3((unsigned)std::min<long>(((long)a.n_tokens + 3) / 4, most)), dim3(kThreads), 0, s>>>(a);
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t s) {
    if (a.c.D <= 64) append_n<4>(a, s);
    else append_n<8>(a, s);
    return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, hipStream_t s) {
    const int lpr = a.c.D <= 64 ? 4 : 8;
    const long items = (long)a.n_tokens * 2 * a.c.Hk * lpr;
    const unsigned grid = (unsigned)std::min<long>((items + kThreads - 1) / kThreads, 1 << 20);
    if (lpr == 4) read_rows<4><<<dim3(grid), dim3(kThreads), 0, s>>>(a, items);
    else read_rows<8><<<dim3(grid), dim3(kThreads), 0, s>>>(a, items);
    return hipGetLastError();
}

}  // namespace qattn
