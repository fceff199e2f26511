// Host code of the operators on channels-last sequences under AddressSanitizer + UndefinedBehaviorSanitizer: validation, extents of
// strided tensors, workspace sizes, with sizes from the edges of what is accepted.  No call here may reach a launch: each one that is
// otherwise in order is given outputs that overlap.
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

static char* address(int i) { return (char*)((uintptr_t)(i + 1) << 36); }

int main()
{
    const int lengths[] = {0, 1, 63, 64, 65, 4097, 1 << 20, 1 << 30, (1 << 30) + 1, INT32_MAX};
    const int channels[] = {1, 7, 8, 63, 64, 4096, 1 << 24, (1 << 24) + 1, INT32_MAX};
    const int batches[] = {0, 1, 5, 65536, INT32_MAX};
    for (int n : lengths)
        for (int c : channels)
            for (int b : batches)
                for (int dtype = 0; dtype < 3; ++dtype) {
                    const long long row = c, batch = (long long)n * c > (1LL << 40) ? (1LL << 40) : (long long)n * c;
                    const bool fits = n <= (1 << 30) && c <= (1 << 24);
                    sys_causal_conv1d_t conv = {dtype, SYS_F32, SYS_ACT_SILU, 4, b, n, c, b, batch, row, batch, row};
                    const size_t cw = sys_causal_conv1d_backward_workspace(&conv);
                    if (!fits && cw) ++failures, std::fprintf(stderr, "workspace of a refused call\n");
                    // y over x
                    const int st = sys_causal_conv1d(&conv, address(1), address(2), nullptr, nullptr, nullptr, address(1), nullptr, nullptr);
                    if (b && n && fits && (long long)n * c <= (1LL << 40)) expect(st, SYS_ERR_ALIAS, "convolution");
                    else if (b && n && st == SYS_OK) ++failures;
                    for (int states : {1, 16, 64}) {
                        const long long srow = states, sbatch = (long long)n * states;
                        sys_selective_scan_t scan = {dtype, 1, b, n, c, states, 1, b, batch, row, batch, row, batch, row, sbatch, srow, sbatch, srow, batch, row};
                        const size_t w = sys_selective_scan_backward_workspace(&scan) + sys_selective_scan_workspace(&scan);
                        if (!fits && w) ++failures;
                        if (!b || !n) continue;
                        const int got = sys_selective_scan(&scan, address(1), address(2), (float*)address(3), address(4), address(5), nullptr, nullptr, nullptr,
                                                           nullptr, nullptr, address(1), nullptr, address(9), nullptr);
                        if (fits && (long long)n * c <= (1LL << 40)) expect(got, SYS_ERR_ALIAS, "scan");
                    }
                    for (long long rows : {1LL, 5LL, (long long)n + 1, 1LL << 40, (1LL << 40) + 1}) {
                        sys_group_norm_t norm = {dtype, SYS_F32, SYS_ACT_RELU, 1, b, c, 1e-5f, 0, rows, 1LL << 40, row, 1LL << 40, row};
                        sys_group_norm_workspace(&norm);
                        sys_group_norm_backward_workspace(&norm);
                    }
                }
    expect(sys_causal_conv1d(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr), SYS_ERR_NULL, "no description");
    std::printf(failures ? "%d failures\n" : "clean\n", failures);
    return failures != 0;
}
