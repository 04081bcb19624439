// Which outputs dense_norm refuses because their rows overlap, on the CPU: every layout of a few tokens and heads against all pairs of rows.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "qdense_internal.h"

static int g_fail = 0;
#define CHECK(c, ...) do { if (!(c)) { std::printf("FAILED line %d: %s (", __LINE__, #c); std::printf(__VA_ARGS__); std::printf(")\n"); ++g_fail; } } while (0)

namespace qmoe {
int32_t set_error(int32_t code, const char *, ...) { return code; }
}  // namespace qmoe
namespace qdense {
hipError_t launch_norm(const NormArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_pack4(const uint8_t *, const uint8_t *, int, int, uint8_t *, uint8_t *, hipStream_t) { return hipSuccess; }
size_t linear_workspace(int, int, int, int) { return 0; }
hipError_t launch_linear(LinearArgs, size_t, hipStream_t) { return hipSuccess; }
}  // namespace qdense

static uint8_t *at(int n) { return (uint8_t *)((uintptr_t)(n + 1) << 40); }

static bool apart(int T, int H, long ts, long hs, long dim) {
    for (int a = 0; a < T * H; ++a)
        for (int b = 0; b < a; ++b) {
            const long d = (a / H - b / H) * ts + (a % H - b % H) * hs;
            if (d < dim && -d < dim) return false;
        }
    return true;
}

static int32_t norm(int T, int H, long ts, long hs, int dim, int which) {
    const dense_rows in{at(0), nullptr, 1 << 20, 1 << 10, DENSE_BF16}, add{at(1), nullptr, 1 << 20, 1 << 10, DENSE_BF16}, plain{at(2), nullptr, 1 << 20, 1 << 10, DENSE_BF16};
    const dense_rows odd{at(3), nullptr, ts, hs, DENSE_BF16};
    return dense_norm(&in, &add, which ? &odd : nullptr, which ? &plain : &odd, nullptr, 0, 0.f, 1e-5f, T, H, dim, nullptr);
}

int main() {
    int fine = 0, refused = 0;
    for (int T = 1; T <= 5; ++T)
        for (int H = 1; H <= 5; ++H)
            for (long ts = 0; ts <= 24 * 8; ts += 8)
                for (long hs = 0; hs <= 24 * 8; hs += 8)
                    for (int dim : {8, 24, 40}) {
                        const bool ok = apart(T, H, ts, hs, dim);
                        for (int which = 0; which < 2; ++which)
                            CHECK(norm(T, H, ts, hs, dim, which) == (ok ? MOE_OK : MOE_E_ARG), "%d tokens, %d heads, strides %ld %ld, dim %d, %s", T, H, ts, hs, dim, which ? "total" : "out");
                        ++(ok ? fine : refused);
                    }
    CHECK(fine > 5000 && refused > 5000, "%d %d", fine, refused);
    // the most tokens and heads, and strides whose products pass 64 bits
    CHECK(norm(1 << 20, 1024, 8, 8, 8, 0) == MOE_E_ARG, "one place");
    CHECK(norm(1 << 20, 1024, 8 * 1024, 8, 8, 0) == MOE_OK, "tokens first");
    CHECK(norm(1 << 20, 1024, 8, 8l << 20, 8, 0) == MOE_OK, "heads first");
    CHECK(norm(1 << 20, 1024, 1l << 60, 1l << 60, 8, 0) == MOE_E_ARG, "far, one place");
    CHECK(norm(1 << 20, 1024, 1l << 60, (1l << 60) + 8, 8, 0) == MOE_OK, "far, apart");
    CHECK(norm(1 << 20, 1024, (1l << 62) + 8, 1l << 62, 16, 1) == MOE_E_ARG, "far, half a row apart");
    if (g_fail) return 1;
    std::printf("all rows that overlap are refused\n");
    return 0;
}
