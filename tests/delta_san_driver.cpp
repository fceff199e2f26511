// Host code of the operators of a gated delta rule layer under AddressSanitizer + UndefinedBehaviorSanitizer: validation, extents of strided tensors,
// workspace sizes, with sizes from the edges of what is accepted.  No call here may reach a launch: each one that is otherwise in order is given
// outputs that overlap.
#define SYSCONV_NO_HIP_HEADER
#include "sysconv.h"

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

static int failures = 0;

static void expect(int got, int want, const char* what)
{
    if (got != want) {
        std::fprintf(stderr, "%s: %s, expected %s\n", what, sys_status_string(got), sys_status_string(want));
        ++failures;
    }
}

static void wrong(const char* what)
{
    std::fprintf(stderr, "%s\n", what);
    ++failures;
}

static char* address(int i) { return (char*)((uintptr_t)(i + 1) << 36); }

int main()
{
    const long long far = 1LL << 40;
    for (int n : {0, 1, 16, 17, 64, 65, 4097, 1 << 20, 1 << 30, (1 << 30) + 1, INT32_MAX})
        for (int b : {0, 1, 5, 65536, INT32_MAX})
            for (int heads : {1, 2, 48, 1 << 17, INT32_MAX})
                for (int dim : {1, 64, 65, 128, 129, 512, 513, 1024, 1025, INT32_MAX})
                    for (int dtype = 0; dtype < 3; ++dtype) {
                        const long long row = (long long)heads * dim;
                        if (row > 1LL << 32) continue;         // (far beyond what is taken)
                        const long long rows = n * row > far ? far : n * row;
                        const bool norm_fits = n <= (1 << 30) && dim <= SYS_MAX_HEAD_DIM && row <= (1 << 24) && n * row <= far;
                        sys_head_norm_t norm = {dtype, SYS_F32, SYS_NORM_L2, 0, 1, b, n, heads, heads, dim, 0, 1e-6f, rows, row, rows, row, rows, row, rows, row};
                        {
                            const size_t w = sys_head_norm_backward_workspace(&norm);
                            if (!norm_fits && n <= (1 << 30) && (long long)n * row <= far && w) wrong("workspace of a refused norm");
                            const int st = sys_head_norm(&norm, address(1), address(2), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, address(1), address(5), nullptr);
                            if (norm_fits && b && n) expect(st, SYS_ERR_ALIAS, "norm");
                            else if (b && n && st == SYS_OK) wrong("a norm beyond the limits");
                            const int back = sys_head_norm_backward(&norm, address(1), address(2), address(3), address(4), address(5), nullptr, nullptr, nullptr, nullptr,
                                                                    nullptr, address(1), address(6), address(7), nullptr, address(8), nullptr);
                            if (norm_fits && b && n) expect(back, SYS_ERR_ALIAS, "gradients of the norm");
                            else if (b && n && back == SYS_OK) wrong("gradients of a norm beyond the limits");
                        }
                        for (int key_dim : {1, 64, 128, 129}) {
                            const long long keys = (long long)heads * key_dim;
                            const bool fits = n <= (1 << 30) && dim <= SYS_MAX_VALUE_DIM && key_dim <= SYS_MAX_KEY_DIM && row <= (1 << 24) && keys <= (1 << 24) &&
                                              (n <= 1 || (row <= SYS_MAX_DELTA_ROW && keys <= SYS_MAX_DELTA_ROW)) && (long long)n * row <= far;
                            if (keys > far) continue;
                            sys_gated_delta_t delta = {dtype, 1, 1, b, n, heads, heads, key_dim, dim, b, 1.0f, 0, 0, keys, 0, keys, rows, row, 0, heads, 0, heads, rows, row};
                            const size_t w = sys_gated_delta_rule_workspace(&delta) + sys_gated_delta_rule_backward_workspace(&delta);
                            if (!fits && (long long)n * row <= far && n <= (1 << 30) && w) wrong("workspace of a refused delta rule");
                            if (!b || !n) continue;
                            int st = sys_gated_delta_rule(&delta, address(1), address(2), address(3), address(4), (float*)address(5), address(6), nullptr, nullptr, nullptr,
                                                          address(3), nullptr, address(9), nullptr);
                            if (fits) expect(st, SYS_ERR_ALIAS, "delta rule");
                            else if (st == SYS_OK) wrong("a delta rule beyond the limits");
                            st = sys_gated_delta_rule_backward(&delta, address(1), address(2), address(3), address(4), address(5), (float*)address(6), address(7), nullptr,
                                                               nullptr, nullptr, nullptr, address(8), address(9), address(4), address(10), (float*)address(11), address(12),
                                                               nullptr, nullptr, address(13), nullptr);
                            if (fits) expect(st, SYS_ERR_ALIAS, "gradients of the delta rule");
                            else if (st == SYS_OK) wrong("gradients of a delta rule beyond the limits");
                            delta.q_batch = delta.k_batch = keys, delta.v_batch = delta.y_batch = row, delta.delta_batch = delta.beta_batch = heads;
                            st = sys_gated_delta_rule_update(&delta, address(1), address(2), address(3), address(4), (float*)address(5), address(6), nullptr,
                                                             (float*)address(7), nullptr, address(3), (float*)address(7), nullptr);
                            if (dim <= SYS_MAX_VALUE_DIM && key_dim <= SYS_MAX_KEY_DIM && row <= (1 << 24) && keys <= (1 << 24) && n <= (1 << 30))
                                expect(st, SYS_ERR_ALIAS, "token of the delta rule");
                            else if (st == SYS_OK) wrong("a token beyond the limits");
                        }
                    }
    expect(sys_head_norm(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr), SYS_ERR_NULL, "no description");
    std::printf(failures ? "%d failures\n" : "clean\n", failures);
    return failures != 0;
}
