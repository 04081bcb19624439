// dense_norm: residual's addition and root-mean-square norm of rows, out in bf16 or in e4m3 with a scale byte for every 32 elements.
//
//     r = x + add,   out = r * rsqrt(mean(r^2) + eps) * (weight + shift)
//
// A row stays in registers from its first read to its last write: CH pieces of 8 elements in each of TPR lanes, all requested at
// once, so every byte moves once.  Bound by memory (8192 rows of 4096 with a residual of bf16: 43.8 us, 6.1 TB/s; of fp32 71 us, 5.6 TB/s), one row by the way to
// memory and back (2.4 us of one call in a graph of them, where an empty kernel takes 2).  Loads and the total's stores pass the caches by, as nothing of them is read
// again before they would be overwritten; out goes through them: the product behind it reads it.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "qdense_internal.h"

namespace qdense {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// 8 elements of 16 or 32 bytes.
template <bool F32>
struct Eight {
    u32x4 w[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const char *p, long at) {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(p + at * (F32 ? 4 : 2));
        w[0] = __builtin_nontemporal_load(from);
        if constexpr (F32) w[1] = __builtin_nontemporal_load(from + 1);
    }
    __device__ __forceinline__ void store(char *p, long at) const {
        u32x4 *to = reinterpret_cast<u32x4 *>(p + at * (F32 ? 4 : 2));
        __builtin_nontemporal_store(w[0], to);
        if constexpr (F32) __builtin_nontemporal_store(w[1], to + 1);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (F32) return __uint_as_float(w[i / 4][i % 4]);
        else return i % 2 ? hi_f(w[0][i / 2]) : lo_f(w[0][i / 2]);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (F32) w[i / 4][i % 4] = __float_as_uint(v[i]);
            else if (i % 2) w[0][i / 2] = pack_bf16(v[i - 1], v[i]);
        }
    }
};

// Scale byte of 32 elements whose largest has the bits `m` (sign cleared): 448 = 1.75 * 2^8.  255: one of them is not finite.
__device__ __forceinline__ int scale_byte(uint32_t m) {
    const int b = (int)(m >> 23) - 8 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return m >= 0x7F800000u ? 255 : b < 1 ? 1 : b;
}

// 8 elements as e4m3 codes of element * 2^(127 - byte).
__device__ __forceinline__ u32x2 to_fp8(const float (&v)[8], int byte) {
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23), most = byte == 247 ? 240.f : 448.f;       // 256 * 2^(247 - 127) would be over the largest fp32
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = __builtin_amdgcn_fmed3f(v[4 * i + j] * inv, -most, most);
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
        r[i] = byte == 255 ? 0x7F7F7F7Fu : (uint32_t)w;
    }
    return r;
}

constexpr int kThreads = 256;

// A row has TPR lanes: some of a wave (several rows a wave), or whole waves of a workgroup.  ADD: 0 none, 1 bf16, 2 fp32.
template <int TPR, int CH, int ADD, bool FP8>
__global__ __launch_bounds__(TPR > 64 ? TPR : kThreads) void norm_rows(const NormArgs a, long first) {
    constexpr int WG = TPR > 64 ? TPR : kThreads, RPW = WG / TPR, WAVES = TPR > 64 ? TPR / 64 : 1;
    const int lane = threadIdx.x % TPR;
    const long row = first + (long)blockIdx.x * RPW + threadIdx.x / TPR;
    if (TPR <= 64 && row >= a.rows) return;              // whole rows of lanes leave; none of them is asked by an exchange of another row
    const uint32_t t = a.heads == 1 ? (uint32_t)row : (uint32_t)row / (uint32_t)a.heads, h = (uint32_t)row - t * (uint32_t)a.heads;
    const long xo = t * a.x.ts + h * a.x.hs, ao = t * a.add.ts + h * a.add.hs;
    Eight<false> x[CH];
    Eight<ADD == 2> r[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + lane) * 8;
        if (e < a.dim) {
            x[c].load(a.x.p, xo + e);
            if constexpr (ADD != 0) r[c].load(a.add.p, ao + e);
        }
    }
    // The weights are asked for before the sum where registers are there for them: one way to memory less (a row of 4096 alone).
    constexpr bool EARLY = CH <= 2;
    float g[EARLY ? CH : 1][8];
    const auto weights = [&](float (&to)[8], int e) {
        if (a.weight == nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = 1.f;
        } else if (a.weight_type == DENSE_F32) {
            const f32x4 *w = reinterpret_cast<const f32x4 *>((const float *)a.weight + e);
            const f32x4 w0 = w[0], w1 = w[1];
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = (i < 4 ? w0[i] : w1[i - 4]) + a.shift;
        } else {
            const u32x4 w = *reinterpret_cast<const u32x4 *>((const uint16_t *)a.weight + e);
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = (i % 2 ? hi_f(w[i / 2]) : lo_f(w[i / 2])) + a.shift;
        }
    };
    if constexpr (EARLY) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if ((c * TPR + lane) * 8 < a.dim) weights(g[c], (c * TPR + lane) * 8);
    }
    // <128, 4> and <512, 1> have rows of the same sizes, by how many there are: a row has the same sums in both, added in the same order, of each piece's lanes by waves.
    constexpr int SUMS = TPR == 128 && CH == 4 ? CH : 1;
    float sums[SUMS];
#pragma unroll
    for (int c = 0; c < SUMS; ++c) sums[c] = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + lane) * 8;
        float &sum = sums[c % SUMS];
        if (e < a.dim) {
            if constexpr (ADD != 0) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = x[c].get(i) + r[c].get(i);
                r[c].set(v);
                if (a.total.p != nullptr) r[c].store(a.total.p, t * a.total.ts + h * a.total.hs + e);
            } else {
                r[c].w[0] = x[c].w[0];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(r[c].get(i), r[c].get(i), sum);
        }
    }
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d <<= 1)
#pragma unroll
        for (int c = 0; c < SUMS; ++c) sums[c] += __shfl_xor(sums[c], d, 64);
    float sum = sums[0];
    if constexpr (WAVES > 1) {
        __shared__ float part[SUMS * WAVES];
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int c = 0; c < SUMS; ++c) part[c * WAVES + threadIdx.x / 64] = sums[c];
        __syncthreads();
        sum = part[0];
#pragma unroll
        for (int w = 1; w < SUMS * WAVES; ++w) sum += part[w];
    }
    const float inv = rsqrtf(sum / (float)a.dim + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + lane) * 8;
        if (e >= a.dim) continue;                        // dim is a multiple of 32 where four lanes share a scale: they stay or go together
        if constexpr (!EARLY) weights(g[0], e);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r[c].get(i) * inv * g[EARLY ? c : 0][i];
        if constexpr (FP8) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            m = max(m, (uint32_t)__shfl_xor((int)m, 1, 64));
            m = max(m, (uint32_t)__shfl_xor((int)m, 2, 64));
            const int byte = scale_byte(m);
            *reinterpret_cast<u32x2 *>(a.out.p + t * a.out.ts + h * a.out.hs + e) = to_fp8(v, byte);
            if (lane % 4 == 0) a.out.scale[row * (a.dim / 32) + e / 32] = (uint8_t)byte;
        } else {
            Eight<false> y;
            y.set(v);
            *reinterpret_cast<u32x4 *>(a.out.p + 2 * (t * a.out.ts + h * a.out.hs + e)) = y.w[0];
        }
    }
}

template <int TPR, int CH>
void run(const NormArgs &a, hipStream_t s) {
    constexpr int WG = TPR > 64 ? TPR : kThreads, RPW = WG / TPR;
    const auto go = [&](auto add, auto fp8) {
        constexpr long most = (1l << 31) / WG * RPW;     // a launch of 2^32 threads or more would lose the excess
        for (long r = 0; r < a.rows; r += most) {
            const long n = a.rows - r < most ? a.rows - r : most;
            norm_rows<TPR, CH, decltype(add)::value, decltype(fp8)::value><<<dim3((unsigned)((n + RPW - 1) / RPW)), dim3(WG), 0, s>>>(a, r);
        }
    };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, 1> Bf16;
    typedef std::integral_constant<int, 2> F32;
    const auto by_out = [&](auto add) { a.out_type == DENSE_FP8 ? go(add, std::true_type{}) : go(add, std::false_type{}); };
    if (a.add.p == nullptr) by_out(None{});
    else if (a.add_type == DENSE_F32) by_out(F32{});
    else by_out(Bf16{});
}

}  // namespace

// Up to 512 elements a row is within a wave: no barrier, and several rows a wave (8192 * 16 heads of 128: 24.9 us, 44 by a wave each).  Longer ones have the fewest lanes
// that hold them a piece each: rows wait for nothing but their own loads, and their workgroups come and go side by side.  Us of rows of 1024 / 2048 / 4096 with a bf16
// residual, 8192 of them: that many lanes 14.9 / 24.5 / 43.8, always 512 18.5 / 24.5 / 43.8, always a wave 13.5 / 24.0 / 50; 1024 of them: 3.4 / 4.7 / 7.7, 3.8 / 4.8 / 7.7,
// 4.2 / 5.9 / 9.6.  Without a residual a lane's one load leaves much of the way unused: where rows are many, four pieces a lane (4096 rows of 4096 12.7 us instead of 15.6,
// 4096 of 2816 10.3 instead of 13.1; 256 of 4096 4.0 instead of 3.2), each piece's squares summed by themselves as <512, 1> has them, so that a row's bits do not go by
// the number of rows (with one sum a lane 12.7 and 10.0).
hipError_t launch_norm(const NormArgs &a, hipStream_t s) {
    const int pieces = (a.dim + 7) / 8;
    if (pieces <= 8) run<8, 1>(a, s);
    else if (pieces <= 16) run<16, 1>(a, s);
    else if (pieces <= 32) run<32, 1>(a, s);
    else if (pieces <= 64) run<64, 1>(a, s);
    else if (pieces <= 128) run<128, 1>(a, s);
    else if (pieces <= 256) run<256, 1>(a, s);
    else if (pieces <= 512 && a.rows > 1024 && a.add.p == nullptr) run<128, 4>(a, s);
    else if (pieces <= 512) run<512, 1>(a, s);
    else if (pieces <= 1024) run<512, 2>(a, s);
    else if (pieces <= 2048) run<512, 4>(a, s);
    else run<512, 8>(a, s);
    return hipGetLastError();
}

}  // namespace qdense
