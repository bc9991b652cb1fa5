// The index steps of csrc/layers_internal.hpp at the ends of 32 bits, and the launch grids, on the host.
#include <cstdio>

#include "layers_internal.hpp"

using namespace olive;

int main() {
    const int64_t top = 0x7fffffff;
    const int ends[] = {0, 1, 15, 16, 17, 127, 128, 1000, (int)top - 128, (int)top - 64, (int)top - 1, (int)top};
    const int steps[] = {1, 16, 32, 64, 128};
    for (int end : ends)
        for (int n : steps) {
            for (int64_t at = end; at >= 0 && at > (int64_t)end - 300; --at) {
                const int64_t want = at + n < end ? at + n : end;
                if (upto((int)at, n, end) != want) {
                    std::printf("upto(%lld, %d, %d)\n", (long long)at, n, end);
                    return 1;
                }
            }
            // past the end (a tile that a row does not see)
            if (end < top - 1000 && upto(end + 5, n, end) != end) return 2;
            // a loop in such steps visits what one in 64 bits does
            int64_t count = 0, first = end > 1000 ? (int64_t)end - 1000 : 0;
            for (int at = (int)first; at < end; at = upto(at, n, end)) ++count;
            if (count != (end - first + n - 1) / n) return 3;
        }
    const int64_t sizes[] = {1, 255, kGridRow - 1, kGridRow, kGridRow + 1, 2 * kGridRow, 7 * kGridRow + 5, kMostBlocks};
    for (int64_t n : sizes) {
        const dim3 g = grid_of(n);
        const int64_t all = (int64_t)g.x * g.y * g.z;
        if (all < n || all - n >= kGridRow || all > top || (int64_t)g.x * 256 >= (int64_t)1 << 32 || g.y > 65535 ||
            g.z != 1 || (n <= kGridRow && all != n)) {
            std::printf("grid_of(%lld) = %u x %u\n", (long long)n, g.x, g.y);
            return 4;
        }
    }
    std::printf("ok\n");
    return 0;
}
