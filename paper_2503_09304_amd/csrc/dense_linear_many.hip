// dense_linear for many tokens: a tile of 256 rows by 128 tokens a workgroup.
//
// Each of four waves has 64 rows and all of the tile's tokens: weights come straight into its registers, a block of 128 columns ahead, and are widened there, a step before
// their products; the tokens' columns are brought to LDS while the block before is multiplied, and read by all waves, some products before they are needed (left to the
// compiler, which asks for two at a time and waits for them: 8192 tokens by 4096 x 4096 in bf16 214 us, 203 so).  Bound by the matrix units and the tokens' way to LDS
// (with the latter left out 174 us, with nothing but products 164), at a clock that power holds at 2.0 to 2.1 GHz: 198 us, 1.39 PFLOP/s; 4093 tokens by 28672 x 4096 in 8 bits 455 us,
// 2.1 PFLOP/s.  (Tokens and weights both through LDS, one workgroup a CU, two blocks ahead: 241 and 516.)
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dense_linear.h"

namespace qdense {
namespace {

constexpr int kXcds = 8, kGroup = 8;
constexpr int kWaves = 4, kRowTiles = 4, NT = 8;         // a wave's tiles of 16 rows, a workgroup's of 16 tokens

template <int XT>
__global__ __launch_bounds__(64 * kWaves, XT == X_WIDE ? 1 : 2) void linear_many(const LinearArgs a, long first_wg) {
    constexpr int PIECES = XT == X_BF16 ? 16 : 8;        // of 16 bytes, in a token's 128 columns
    constexpr int TOK = NT * 16, BLOCK = TOK * PIECES * 16, LOADS = BLOCK / 1024 / kWaves;
    static_assert(LOADS >= 1 && (TOK / LOADS) % 16 == 0, "the order of pieces goes by the token's place in 16");
    __shared__ __align__(16) char xs[2][BLOCK];
    __shared__ uint32_t xb[2][TOK];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, g = l >> 4, t16 = l & 15;
    const int blocks = (a.K + 127) / 128, sets = (a.K + 511) / 512, row_tiles = (a.R + 15) / 16;
    const int row_wgs = (row_tiles + kRowTiles * kWaves - 1) / (kRowTiles * kWaves);
    // Workgroups go to the XCDs in turn.  Each XCD has tiles that lie together, kGroup of them along the rows before the next tokens: its L2 holds what they share (tiles dealt to
    // the XCDs in turn / kGroup 4 / 8 / 16, us: 8192 tokens by 2816 x 2048 91 / 81 / 82 / 80, 3584 by 6144 x 4096 150 / 146 / 142 / 143).
    const long token_wgs = (a.n_tokens + TOK - 1) / TOK, all = row_wgs * token_wgs, per_xcd = (all + kXcds - 1) / kXcds;
    const long at = first_wg + blockIdx.x, wg = at % kXcds * per_xcd + at / kXcds;
    if (at / kXcds >= per_xcd || wg >= all) return;
    const int group = (int)(wg / (kGroup * token_wgs)), in_group = min(kGroup, row_wgs - group * kGroup);
    const long part = wg - group * kGroup * token_wgs;
    const int rt = (group * kGroup + (int)(part % in_group)) * (kRowTiles * kWaves) + w * kRowTiles, t0 = (int)(part / in_group) * TOK;
    const uint8_t *codes[kRowTiles], *scales[kRowTiles];
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) {
        const long tile = min(rt + r, row_tiles - 1);
        codes[r] = a.codes + tile * blocks * 1024;
        scales[r] = a.scales + tile * sets * 256;
    }
    // The pieces that this lane brings to LDS, and in which order a token's stand there: so that the lanes of one read use all banks.  It brings `here` tokens,
    // each STEP behind the one before, and the first again in the place of those behind the last.
    constexpr int PER = 64 / PIECES, STEP = kWaves * PER;        // tokens of a wave's load, of the workgroup's
    const int mine = w * PER + l / PIECES, p = l % PIECES, q = XT == X_BF16 ? p ^ (mine & 15) : p ^ (mine >> 1 & 7);
    const int first_piece = XT == X_BF16 ? 4 * (q & 3) + (q >> 2) : XT == X_FP8 ? q : 2 * (q & 3) + (q >> 2);
    const int here = (a.n_tokens - t0 - mine + STEP - 1) / STEP;
    const char *const src = a.x.p + (long)min(t0 + mine, a.n_tokens - 1) * a.x.ts * (XT == X_BF16 ? 2 : 1);
    const long step = STEP * a.x.ts * (XT == X_BF16 ? 2 : 1);
    const int k_bytes = a.K * (XT == X_BF16 ? 2 : 1);
    const uint8_t *xscale = XT == X_BF16 ? nullptr : a.x.scale + (long)min(t0 + tid % TOK, a.n_tokens - 1) * (a.K / 32);
    uint32_t next_xb[4] = {0, 0, 0, 0};
    u32x4 c[kRowTiles];
    uint32_t sc[kRowTiles];
    constexpr int ASKS = LOADS + kRowTiles + (XT == X_BF16 ? 0 : 1);
    const auto ask = [&](int i, int b, int buf) {        // the i-th part of what block b needs
        if (i < LOADS) {
            const int at = (b * PIECES + first_piece) * 16, off = at < k_bytes ? at : 0;    // behind the last column: weights are zero there
            to_lds(src + off + (i < here ? i * step : 0l), &xs[buf][(w + kWaves * i) * 1024]);
        } else if (i < LOADS + kRowTiles) {
            const int r = i - LOADS;
            c[r] = *reinterpret_cast<const u32x4 *>(codes[r] + (long)b * 1024 + l * 16);
            sc[r] = *reinterpret_cast<const uint32_t *>(scales[r] + (b >> 2) * 256 + l * 4);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) next_xb[j] = xscale[min(4 * b + j, a.K / 32 - 1)];
        }
    };
    f32x4 acc[kRowTiles][NT];
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ASKS; ++i) ask(i, 0, 0);
    const auto block = [&](int b, auto more) {
        const int buf = b & 1;
        if constexpr (XT != X_BF16)
            if (tid < TOK) xb[buf][tid] = next_xb[0] | next_xb[1] << 8 | next_xb[2] << 16 | next_xb[3] << 24;
        u32x4 cc[kRowTiles];
        uint32_t cs[kRowTiles];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // this wave's pieces are in LDS
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            cc[r] = c[r];
            cs[r] = sc[r] >> 8 * (b & 3) & 255;
        }
        products<XT, kRowTiles, NT>(acc, cc, cs, xs[buf], xb[buf], g, t16, [&](int i, int n) {
            if constexpr (decltype(more)::value) {
                constexpr int EARLY = 2;                 // in the first half: they have the second to come
#pragma unroll
                for (int k = 0; k < ASKS; ++k)
                    if (k * n / EARLY / ASKS == i) ask(k, b + 1, buf ^ 1);
            }
        });
    };
    for (int b = 0; b + 1 < blocks; ++b) block(b, std::true_type{});
    block(blocks - 1, std::false_type{});
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int t = t0 + n * 16 + t16;
        if (t >= a.n_tokens) continue;
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            const int o = (rt + r) * 16 + g * 4;
            if (o >= a.R) continue;
            store4(a, t, o, acc[r][n]);
        }
    }
}

}  // namespace

hipError_t launch_linear_many(const LinearArgs &a, hipStream_t s) {
    const long row_wgs = ((a.R + 15) / 16 + kRowTiles * kWaves - 1) / (kRowTiles * kWaves), all = (row_wgs * ((a.n_tokens + NT * 16 - 1) / (NT * 16)) + kXcds - 1) / kXcds * kXcds;
    constexpr long kMost = 1 << 23;                      // workgroups of 256 threads that a launch may have
    for (long at = 0; at < all; at += kMost) {
        const dim3 grid((unsigned)(all - at < kMost ? all - at : kMost)), block(64 * kWaves);
        if (a.x_type == DENSE_BF16) linear_many<X_BF16><<<grid, block, 0, s>>>(a, at);
        else if (a.out_type == DENSE_BF16) linear_many<X_FP8><<<grid, block, 0, s>>>(a, at);
        else linear_many<X_WIDE><<<grid, block, 0, s>>>(a, at);
    }
    return hipGetLastError();
}

}  // namespace qdense
