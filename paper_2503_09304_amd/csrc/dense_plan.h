// The rule by which dense_linear picks a kernel, its tiles and its ranges of columns.  Host code without HIP: a test runs it by itself.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>

namespace qdense {

constexpr int kFewWaves = 8, kFewTokens = 16;              // of a workgroup of linear_few
constexpr size_t kMostLds = 128 * 1024;
constexpr size_t kMostWorkspace = (size_t)1 << 28;
// Blocks of 128 columns whose tokens' scales linear_some has in LDS at once.  Ranges are no longer where they can be more (and nowhere where waves have tokens of their own:
// they do not wait for each other); one that is stops for the next scales (61 tokens in 8 bits by 4096 x 14336 without a workspace 19 us, by linear_many 105).
constexpr int kSomeBlocks = 64;

// How a call is cut into workgroups.
struct Plan {
    int tiles, rows;              // linear_some: of 16 tokens a workgroup, of 16 rows a wave; tiles 8: linear_many
    int ks;                       // waves that share rows, or, times four, rows and tokens of four waves
    int share;                    // linear_some: waves that share tokens, 4 or 1; linear_few: 0
    int ranges, range_blocks;     // of 128 columns
    size_t lds;                   // linear_few
};
inline void cut(Plan &p, int blocks, int ranges) {
    p.range_blocks = (blocks + ranges - 1) / ranges;
    p.ranges = (blocks + p.range_blocks - 1) / p.range_blocks;
}
inline Plan few_of(int n_tokens, int R, int K, bool bf16, int ranges) {
    const int blocks = (K + 127) / 128, row_tiles = (R + 15) / 16, token_tiles = (n_tokens + kFewTokens - 1) / kFewTokens;
    Plan p{1, 1, 1, 0, 1, 1, 0};
    const size_t per_block = (size_t)std::min(n_tokens, kFewTokens) * (bf16 ? 256 : 132);
    const int most = (int)std::min<size_t>(blocks, kMostLds / per_block);
    cut(p, blocks, std::max(ranges, (blocks + most - 1) / most));
    const long units = (long)row_tiles * token_tiles * p.ranges;
    while (p.ks < 8 && units * p.ks < 2048 && p.range_blocks >= 2 * p.ks) p.ks *= 2;
    p.lds = std::max<size_t>((size_t)p.range_blocks * per_block + 1024, (size_t)(p.ks > 1 ? kFewWaves * 1024 : 0));
    return p;
}
inline Plan some_of(int K, int tiles, int rows, int ks, int ranges, int share = 4) {
    Plan p{tiles, rows, ks, share, 1, 1, 0};
    cut(p, (K + 127) / 128, ranges);
    return p;
}
// Each variant where it is best, us, x in bf16, with its best number of ranges: 1 token by 6144 x 4096 linear_few 5.9, linear_some with tiles of 1x1 (16
// tokens by 16 rows of a wave) and KS 4 7.3, with 2x1 8.9; by 28672 x 4096 15.1 and, 1x1 with KS 2, 12.5; 16 by 6144 x 4096 9.3, KS 2 8.1, KS 4 7.4, 2x1 9.2; 8 by 32000 x 2048 11.3, 8.7; 64 by 1024 x 1024
// waves with tokens of their own 4.4, 2x1 4.9; 64 by 6144 x 4096 2x1 with KS 1 12.9 and with 2 10.0, 2x2 12.4, 4x2 14.3, 4x4 17.5, linear_many 42; 128
// 16.1, 15.8, 13.0, 17.1; 256 by 6144 x 4096 4x2 with KS 2 18.1, with 1 20.5, 4x4 24.2; 1024 53 with 4x2, 56 with 4x4 and linear_many; 4096 184, 168, 149.  Ranges: 61 by 4096 x 14336 in tiles
// of 4x2 with 8 of them 16.5, with 2 33.
// Us that a plan takes, fitted to what was measured (420 shapes of 64 to 16384 columns, 16 to 32000 rows, 1 to 8192 tokens, both types of x, every plan): a launch and the
// first bytes; for every block of 128 columns of the workgroups that a CU has what one takes alone, or among others; linear_few what a CU takes in; ranges a launch and
// their sums' way to memory and back; outputs their way to memory.  On 200 shapes drawn anew its choice takes 2.5 % more than the best plan of a shape in the mean, 49 % at most.
inline float us_of(const Plan &p, int n_tokens, int R, int K, bool bf16) {
    const int row_tiles = (R + 15) / 16, token_tiles = (n_tokens + p.tiles * 16 - 1) / (p.tiles * 16);
    const float sums = (float)n_tokens * R, ends = (p.ranges == 1 ? 0.f : 2.36f + sums * p.ranges * 1.86e-06f) + sums * 1.22e-06f;
    if (p.share == 0) {
        const int per = kFewWaves / p.ks;
        const long wgs = (long)((row_tiles + per - 1) / per) * token_tiles * p.ranges, on_cu = (wgs + 255) / 256;
        const float x = (float)std::min(n_tokens, kFewTokens) * (bf16 ? 256.f : 132.f) * p.range_blocks, w = (float)per * p.range_blocks * 1088.f;
        return 3.6f + (float)on_cu * (x + w) / 47.9e3f + ends;
    }
    const int per = p.tiles == 8 ? 16 : p.share * p.rows, rounds = (p.range_blocks + p.ks - 1) / p.ks;
    const long wgs = (long)((row_tiles + per - 1) / per) * token_tiles * p.ranges, on_cu = (wgs + 255) / 256;
    if (p.share == 1) return 3.33f + (float)on_cu * rounds * .474f + ends;
    // [x in bf16][tokens by rows of a wave: 4x2, 2x1, 2x2 tiles with KS 2; 2x1, 4x2, 4x4 with KS 1; linear_many; 1x1 with KS 2, 4]
    static const float alone[2][9] = {{.902f, .356f, .555f, .213f, .467f, .616f, 1.11f, .316f, .529f}, {.991f, .353f, .552f, .235f, .549f, .772f, 1.21f, .261f, .482f}},
                       among[2][9] = {{.778f, .33f, .7f, .151f, .341f, .475f, .71f, .234f, 1.14f}, {.997f, .388f, .799f, .181f, .403f, .676f, 1.01f, .195f, 1.25f}};
    const int kind = p.tiles == 8 ? 6 : p.tiles == 1 ? p.ks == 2 ? 7 : 8 : p.ks == 2 ? p.tiles == 4 ? 0 : p.rows : p.tiles == 2 ? 3 : p.rows == 2 ? 4 : 5;
    return 3.33f + (float)rounds * (on_cu > 1 ? (float)on_cu * among[bf16][kind] : alone[bf16][kind]) + ends;
}
inline size_t workspace_of(const Plan &p, int n_tokens, int R) { return p.ranges > 1 ? (size_t)p.ranges * n_tokens * (((size_t)R + 15) / 16 * 16) * 4 : 0; }
// The best plan whose ranges' sums fit `most` bytes.
inline Plan plan_of(int n_tokens, int R, int K, bool bf16, size_t most) {
    const int blocks = (K + 127) / 128;
    Plan best{8, 4, 1, 4, 1, blocks, 0};
    float least = n_tokens > 64 ? us_of(best, n_tokens, R, K, bf16) : INFINITY;
    const auto look = [&](const Plan &p) {
        if (p.ranges > 1 && workspace_of(p, n_tokens, R) > most) return;
        const float us = us_of(p, n_tokens, R, K, bf16);
        if (us < least) {
            best = p;
            least = us;
        }
    };
    const int whole = bf16 ? 1 : (blocks + kSomeBlocks - 1) / kSomeBlocks;       // ranges whose scales are in LDS at once
    int in_vain = 0;
    for (const int z : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (z > blocks || in_vain == 2) break;           // two more ranges without a gain: the host's time counts too
        const float before = least;
        const int cuts = std::max(z, most == 0 ? 1 : whole);
        if (n_tokens <= kFewTokens) look(few_of(n_tokens, R, K, bf16, z));
        if (n_tokens <= 64) {
            look(some_of(K, 1, 1, 2, cuts));
            look(some_of(K, 1, 1, 4, cuts));
        }
        if (n_tokens <= 1024) look(some_of(K, 2, 1, 4, std::max(z, whole), 1));
        if (n_tokens <= 4096) {
            look(some_of(K, 2, 1, 1, cuts));
            look(some_of(K, 4, 2, 2, cuts));
        }
        if (n_tokens <= 2048) {
            look(some_of(K, 2, 1, 2, cuts));
            look(some_of(K, 2, 2, 2, cuts));
        }
        if (n_tokens > 32) {
            look(some_of(K, 4, 2, 1, cuts));
            look(some_of(K, 4, 4, 1, cuts));
        }
        in_vain = least < before ? 0 : in_vain + 1;
    }
    return best;
}
// The plan of a call with `bytes` of workspace: the one that linear_workspace counted where there is enough, so that more changes nothing; else the best without ranges.
inline Plan plan_with(int n_tokens, int R, int K, bool bf16, size_t bytes) {
    const Plan p = plan_of(n_tokens, R, K, bf16, kMostWorkspace);
    return workspace_of(p, n_tokens, R) <= bytes ? p : plan_of(n_tokens, R, K, bf16, 0);
}

}  // namespace qdense
