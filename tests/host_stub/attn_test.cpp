// Checks of the attention calls' host side (qattn_api.hip) on the CPU: the kernels' launchers are recording stubs, nothing is computed.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "qattn_internal.h"

static int g_fail = 0;
#define CHECK(c) do { if (!(c)) { std::printf("FAILED line %d: %s\n", __LINE__, #c); ++g_fail; } } while (0)

namespace qmoe {
int32_t set_error(int32_t code, const char *fmt, ...) {
    va_list v;
    va_start(v, fmt);
    std::vprintf(fmt, v);
    va_end(v);
    std::printf("\n");
    return code;
}
}  // namespace qmoe

static std::vector<qattn::DecodeArgs> g_decode;

namespace qattn {
hipError_t launch_append(const AppendArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_read(const ReadArgs &, hipStream_t) { return hipSuccess; }
int prompt_slots(int) { return 512; }
int prompt_log_tile(int, int, int, int, int) { return 7; }
int prompt_parts(int, int, int, int, int, int) { return 1; }
hipError_t launch_prompt(const PromptArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode(const DecodeArgs &a, hipStream_t) {
    g_decode.push_back(a);
    return hipSuccess;
}
}  // namespace qattn

static uint8_t *const kBase = (uint8_t *)(1ull << 40);        // addresses that nothing looks at

// Bytes of a decode call's workspace: [0, counters) and [sums, end).
struct Used {
    size_t counters, sums, end;
};
static Used decode(int n, int Hq, int Hk, int D, size_t bytes) {
    const attn_cache c{kBase, kBase, nullptr, nullptr, 8, Hk, 64, D, ATTN_BF16};
    const attn_rows r{kBase, (int64_t)Hq * D, D};
    g_decode.clear();
    CHECK(attn_decode(&c, &r, &r, nullptr, n, Hq, (int32_t *)kBase, 2048, (int32_t *)kBase, 1.f, kBase, bytes, nullptr, nullptr) == MOE_OK);
    const qattn::DecodeArgs &a = g_decode.at(0);
    const size_t tiles = (size_t)Hk * qattn::group_tiles(Hq, Hk);
    CHECK((uint8_t *)a.arrived == kBase && (uintptr_t)a.part % 256 == 0);
    CHECK(n * tiles * 4 <= attn_decode_counter_bytes(n, Hq, Hk));
    const size_t sums = (uint8_t *)a.part - kBase;
    return {n * tiles * 4, sums, sums + qattn::decode_pieces(n, Hq, Hk) * tiles * 16 * (D + 2) * 4};
}

// Calls of any number of sequences, heads and sizes on one workspace: nobody's sums stand where anybody's counters are.
static void test_calls_that_share_a_workspace() {
    struct Shape { int Hq, Hk, D; };
    const std::vector<Shape> shapes = {{32, 8, 128}, {8, 8, 16}, {71, 1, 64}, {1, 1, 16}, {5, 5, 112}, {64, 2, 80}, {1024, 1024, 16}};
    for (int most : {1, 2, 9, 64, 65, 300, 1000}) {
        std::vector<int> ns = {1, 2, 3, 8, 31, 32, 33, 63, 64, 65, 299, 1000};
        for (size_t spare : {0, 1, 255, 256, 4096, 1 << 20}) {
            for (const Shape &s : shapes) {                      // sequences up to `most`, one shape
                const size_t bytes = attn_decode_workspace_bytes(most, s.Hq, s.Hk, s.D) + spare;
                size_t counters = 0, sums = bytes;
                for (int n : ns) {
                    if (n > most) continue;
                    const Used u = decode(n, s.Hq, s.Hk, s.D, bytes);
                    CHECK(u.end <= bytes);
                    counters = std::max(counters, u.counters);
                    sums = std::min(sums, u.sums);
                }
                CHECK(counters <= sums);
            }
            size_t bytes = 0, counters = 0;                      // and all shapes on one that is enough for each
            for (const Shape &s : shapes) bytes = std::max(bytes, attn_decode_workspace_bytes(most, s.Hq, s.Hk, s.D) + spare);
            size_t sums = bytes;
            for (const Shape &s : shapes)
                for (int n : ns) {
                    if (n > most) continue;
                    const Used u = decode(n, s.Hq, s.Hk, s.D, bytes);
                    CHECK(u.end <= bytes);
                    counters = std::max(counters, u.counters);
                    sums = std::min(sums, u.sums);
                }
            CHECK(counters <= sums);
        }
    }
}

// A workspace of the stated size, or a little more, is enough.
static void test_workspaces_are_long_enough() {
    for (int n = 1; n <= 4000; ++n)
        for (size_t spare : {0, 1, 256, 257}) {
            const size_t bytes = attn_decode_workspace_bytes(n, 8, 8, 16) + spare;
            const Used u = decode(n, 8, 8, 16, bytes);
            CHECK(u.counters <= u.sums && u.end <= bytes);
        }
}

// The workgroups of a call, as it launches them: all of them, in order, no launch of 2^32 threads.
static void test_launches_of_many_workgroups() {
    struct Call { int n, Hq, Hk; bool several; };
    for (const Call &c : {Call{1, 32, 8, false}, Call{64, 32, 8, false}, Call{65535, 64, 64, false}, Call{65535, 256, 256, true}, Call{16400, 1024, 1024, true},
                          Call{65535, 1024, 1024, true}, Call{65535, 1024, 1, false}}) {
        decode(c.n, c.Hq, c.Hk, 16, attn_decode_workspace_bytes(c.n, c.Hq, c.Hk, 16));
        const long all = qattn::decode_workgroups(g_decode.at(0));
        CHECK(all >= (long)c.n * c.Hk * qattn::group_tiles(c.Hq, c.Hk));
        long next = 0;
        int launches = 0;
        qattn::in_launches(all, [&](int at, unsigned n) {
            CHECK(at == next && n > 0 && (unsigned long long)n * 256 < 1ull << 32);
            next += n;
            ++launches;
        });
        CHECK(next == all && (launches > 1) == c.several);
    }
    for (long all : {0l, 1l, (1l << 23) - 1, 1l << 23, (1l << 23) + 1, 5l << 23}) {
        long next = 0;
        qattn::in_launches(all, [&](int at, unsigned n) { CHECK(at == next); next += n; });
        CHECK(next == all);
    }
}

// Calls of nothing: tensors without elements have no address.
static void test_calls_of_nothing() {
    const attn_cache c{kBase, kBase, nullptr, nullptr, 8, 4, 64, 64, ATTN_BF16};
    const attn_rows none{nullptr, 0, 0};
    for (const attn_place &p : {attn_place{nullptr, nullptr, nullptr, 0, 0}, attn_place{nullptr, nullptr, (int32_t *)kBase, 3, 4}, attn_place{nullptr, nullptr, nullptr, 0, 4}}) {
        CHECK(attn_append(&c, &none, &none, &none, &none, &none, 8, 0, &p, nullptr, nullptr, nullptr) == MOE_OK);
        CHECK(attn_append(&c, nullptr, &none, &none, nullptr, nullptr, 0, 0, &p, nullptr, nullptr, nullptr) == MOE_OK);
        CHECK(attn_read(&c, &p, 0, &none, &none, nullptr, nullptr) == MOE_OK);
        CHECK(attn_append(&c, &none, &none, &none, &none, &none, 8, 1, &p, nullptr, nullptr, nullptr) == MOE_E_ARG);
    }
    CHECK(attn_prompt(&none, &none, &none, &none, nullptr, nullptr, nullptr, 0, 0, 0, 8, 4, 64, 1.f, 1, nullptr, 0, nullptr) == MOE_OK);
    CHECK(attn_prompt(&none, &none, &none, &none, nullptr, (int32_t *)kBase, (int32_t *)kBase, 3, 0, 0, 8, 4, 64, 1.f, 1, nullptr, 0, nullptr) == MOE_OK);
    CHECK(attn_decode(&c, &none, &none, nullptr, 0, 8, nullptr, 0, nullptr, 1.f, nullptr, 0, nullptr, nullptr) == MOE_OK);
}

int main() {
    test_calls_of_nothing();
    test_launches_of_many_workgroups();
    test_workspaces_are_long_enough();
    test_calls_that_share_a_workspace();
    std::printf(g_fail ? "%d checks failed\n" : "all attention host checks passed\n", g_fail);
    return g_fail ? 1 : 0;
}
