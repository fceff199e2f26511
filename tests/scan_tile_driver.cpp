// The sizes of the buffers through which the selective scan's kernels address their rows (csrc/scan_tile.h), on the host: what no row holds is
// out of every buffer's reach, and every row that exists is in it.
#include <cstdio>
#include <initializer_list>

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
    // no row, no bytes: empty sequences and chunks behind a sequence's end, also where rows are used again or overlap
    for (long long row : {0LL, 1LL, 63LL, 64LL, (long long)SYS_MAX_SCAN_ROW})
        for (int columns : {1, 64, 1 << 24})
            for (int t0 : {0, 16, 1 << 29})
                for (size_t element : {(size_t)2, (size_t)4}) {
                    for (int end : {0, t0 / 2, t0}) expect(buffer_size(bytes_left(t0, end, row, columns, element)) == 0, "bytes of no row", row);
                    expect(bytes_left(t0, t0 + 1, row, columns, element) == (long long)(columns * element), "bytes of one row", row);
                    expect(bytes_left(t0, t0 + 40, row, columns, element) == (long long)((39 * row + columns) * element), "bytes of forty rows", row);
                }
    std::puts(failures ? "failed" : "clean");
    return failures != 0;
}
