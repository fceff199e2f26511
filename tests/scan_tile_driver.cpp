// The sizes of the buffers through which the selective scan's kernels address their rows (csrc/scan_tile.h), on the host: what no row holds is
// out of every buffer's reach, and every row that exists is in it.
#include <cstdio>

#include "scan_tile.h"

using namespace sysconv;

static int failures = 0;

static void expect(bool ok, const char* what, long long value)
{
    if (!ok) std::printf("%s: %lld\n", what, value), ++failures;
}

int main()
{
    for (int shift = 0; shift < 63; ++shift)
        for (long long near = -20; near <= 20; ++near) {
            const long long bytes = (1LL << shift) + near;
            const unsigned size = buffer_size(bytes);
            expect(size <= kNowhere, "a buffer that reaches kNowhere", bytes);
            expect(bytes > 0 || size == 0, "a buffer of rows that do not exist", bytes);
            expect(bytes < 0 || bytes > (long long)kNowhere || size == (unsigned)bytes, "a buffer of another size than its rows", bytes);
            expect(buffer_size(-bytes) == (bytes >= 0 ? 0 : (unsigned)-bytes), "a buffer of rows that do not exist", -bytes);
        }
    std::puts(failures ? "failed" : "clean");
    return failures != 0;
}
