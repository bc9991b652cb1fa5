// The division by a constant of csrc/layers_internal.hpp against the machine's own, on the host.
#include <cstdio>

#include "layers_internal.hpp"

int main() {
    const auto check = [](int64_t d, int64_t n) {
        const olive::Div v = olive::Div::of(d);
        const int q = v.quot((int)n);
        if (q != n / d || v.rem((int)n, q) != n % d) {
            std::printf("%lld / %lld: %d\n", (long long)n, (long long)d, q);
            return false;
        }
        return true;
    };
    const int64_t top = 0x7fffffff;
    uint64_t x = 88172645463325252ull;
    const auto next = [&] { x ^= x << 13; x ^= x >> 7; x ^= x << 17; return x; };
    for (int i = 0; i < 300000; ++i) {
        // divisors of every size, and the numerators beside their multiples
        const int64_t d = i < 70000 ? i + 1 : 1 + (int64_t)(next() % (uint64_t)(top >> (next() % 31)) );
        const int64_t m = top / d * d, k = (int64_t)(next() % (uint64_t)(top / d + 1)) * d;
        for (int64_t n : {(int64_t)0, d - 1, d, d + 1, m - 1, m, top, k, k - 1, (int64_t)(next() % (uint64_t)top)})
            if (n >= 0 && n <= top && !check(d, n)) return 1;
    }
    std::printf("ok\n");
    return 0;
}
