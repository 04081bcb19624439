// Checks of the dense calls' host side (qdense_api.hip) on the CPU: the kernels' launchers are recording stubs, nothing is computed.
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "qdense_internal.h"

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

static std::vector<qdense::NormArgs> g_norm;
static std::vector<qdense::LinearArgs> g_linear;
static size_t g_bytes;

namespace qdense {
hipError_t launch_norm(const NormArgs &a, hipStream_t) {
    g_norm.push_back(a);
    return hipSuccess;
}
hipError_t launch_pack4(const uint8_t *, const uint8_t *, int, int, uint8_t *, uint8_t *, hipStream_t) { return hipSuccess; }
size_t linear_workspace(int, int, int, int) { return 4096; }
hipError_t launch_linear(LinearArgs a, size_t bytes, hipStream_t) {
    g_linear.push_back(a);
    g_bytes = bytes;
    return hipSuccess;
}
}  // namespace qdense

// Addresses that nothing looks at.
static uint8_t *at(int n) { return (uint8_t *)((uintptr_t)(n + 1) << 40); }

static void test_norm() {
    const int T = 5, H = 3, D = 64;
    const dense_rows x{at(0), nullptr, 256, 72, DENSE_BF16}, wide{at(1), nullptr, 192, 64, DENSE_F32}, out{at(2), nullptr, 192, 64, DENSE_BF16};
    const dense_rows total{at(3), nullptr, 192, 64, DENSE_F32}, eight{at(4), at(5), 192, 64, DENSE_FP8};
    CHECK(dense_norm(&x, &wide, &total, &eight, at(6), DENSE_F32, 1.f, 1e-5f, T, H, D, nullptr) == MOE_OK);
    const qdense::NormArgs &a = g_norm.back();
    CHECK(a.rows == T * H && a.heads == H && a.dim == D && a.add_type == DENSE_F32 && a.out_type == DENSE_FP8 && a.weight_type == DENSE_F32 && a.shift == 1.f && a.eps == 1e-5f);
    CHECK(a.x.p == (char *)at(0) && a.x.ts == 256 && a.x.hs == 72 && a.add.p == (char *)at(1) && a.total.p == (char *)at(3) && a.out.p == (char *)at(4) && a.out.scale == at(5));
    // rows over themselves
    dense_rows over = wide;
    CHECK(dense_norm(&x, &wide, &over, &out, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_OK);
    over.token_stride = 256;
    size_t before = g_norm.size();
    CHECK(dense_norm(&x, &wide, &over, &out, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_E_ARG);
    CHECK(dense_norm(&x, &wide, &over, &out, nullptr, 0, 0.f, 1e-5f, 1, H, D, nullptr) == MOE_OK && g_norm.size() == ++before);      // of one token the stride is nothing
    const dense_rows same = x;
    CHECK(dense_norm(&x, nullptr, nullptr, &same, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_OK && g_norm.size() == ++before);
    dense_rows other = x, bad = eight, sums = wide;
    other.head_stride = 80;
    CHECK(dense_norm(&x, nullptr, nullptr, &other, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_E_ARG);
    bad.data = x.data;
    CHECK(dense_norm(&x, nullptr, nullptr, &bad, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_E_ARG);
    bad.data = wide.data;
    CHECK(dense_norm(&x, &wide, nullptr, &bad, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_E_ARG);
    for (void *p : {x.data, out.data}) {
        sums.data = p;
        CHECK(dense_norm(&x, &wide, &sums, &out, nullptr, 0, 0.f, 1e-5f, T, H, D, nullptr) == MOE_E_ARG);
    }
    CHECK(g_norm.size() == before);
    // the most rows
    const dense_rows far{at(0), nullptr, 1l << 40, 0, DENSE_BF16}, to{at(2), nullptr, 1l << 40, 0, DENSE_BF16};
    CHECK(dense_norm(&far, nullptr, nullptr, &to, nullptr, 0, 0.f, 1e-5f, 1 << 30, 1, 32768, nullptr) == MOE_OK && g_norm.back().rows == 1 << 30 && g_norm.back().x.ts == 1l << 40);
}

static void test_linear() {
    const dense_matrix4 w{at(0), at(1), 1 << 24, 1 << 20};
    const dense_rows x{at(2), nullptr, 0, 0, DENSE_BF16}, out{(char *)at(3) + 2, nullptr, (1 << 24) + 1, 0, DENSE_BF16};
    CHECK(dense_linear(&x, &w, &out, 1 << 24, nullptr, 1 << 20, nullptr) == MOE_OK && g_bytes == 0);                   // no workspace, whatever is said of its size
    CHECK(dense_linear(&x, &w, &out, 7, at(4), 100, nullptr) == MOE_OK && g_bytes == 100);
    const qdense::LinearArgs &a = g_linear.back();
    CHECK(a.R == 1 << 24 && a.K == 1 << 20 && a.n_tokens == 7 && a.ranges == 1 && a.part == (float *)at(4) && a.x.p == (char *)at(2) && a.out.ts == (1 << 24) + 1);
    const size_t before = g_linear.size();
    dense_rows over = out;
    over.data = x.data;
    CHECK(dense_linear(&x, &w, &over, 1, nullptr, 0, nullptr) == MOE_E_ARG);
    CHECK(dense_linear(&x, &w, &out, 1, x.data, 1 << 20, nullptr) == MOE_E_ARG);
    CHECK(dense_linear(&x, &w, &out, 0, nullptr, 0, nullptr) == MOE_OK && g_linear.size() == before);
}

int main() {
    test_norm();
    test_linear();
    if (g_fail) return 1;
    std::printf("all dense host checks passed\n");
    return 0;
}
