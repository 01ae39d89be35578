// Strided tensors against the sets of their bytes, for test_spans.py: prints how many pairs were told wrongly, and how many share.
#include "spans.h"

#include <cstdio>
#include <random>
#include <set>
#include <vector>

int main() {
    using cbtbe::Span;
    std::mt19937 rng(5);
    auto below = [&](int n) { return static_cast<long>(rng() % static_cast<unsigned>(n)); };
    long wrong = 0, sharing = 0;
    for (int t = 0; t < 100000; ++t) {
        Span s[2];
        std::set<long> bytes[2];
        const long steps[4] = {below(12), below(40), below(90), below(200)};
        for (int x = 0; x < 2; ++x) {
            const long begin = 1000 + below(150), width = below(7), levels = below(4);
            s[x] = Span(reinterpret_cast<void*>(begin), width);
            std::vector<long> at{begin};
            for (long k = 0; k < levels; ++k) {
                const long n = below(6) ? 1 + below(5) : below(2), step = below(3) ? steps[below(4)] : below(120);
                s[x].by(n, step);
                std::vector<long> to;
                for (const long p : at)
                    for (long i = 0; i < n; ++i) to.push_back(p + i * step);
                at = to;
            }
            for (const long p : at)
                for (long i = 0; i < width; ++i) bytes[x].insert(p + i);
        }
        bool want = false;
        for (const long b : bytes[0]) want = want || bytes[1].count(b);
        wrong += cbtbe::share(s[0], s[1]) != want;
        sharing += want;
    }
    // Slices of large buffers, side by side and one byte into one another; strides of 2^42 bytes and 2^31 rows.
    auto heads = [](long begin, long n) { return Span(reinterpret_cast<void*>(begin), 256).by(long{1} << 20, 6144).by(n, 256); };
    wrong += cbtbe::share(heads(1 << 20, 8), heads((1 << 20) + 2048, 8)) || !cbtbe::share(heads(1 << 20, 8), heads((1 << 20) + 2047, 8));
    auto far = [](long begin) { return Span(reinterpret_cast<void*>(begin), 64).by(long{1} << 31, long{1} << 42); };
    wrong += cbtbe::share(far(4096), far(4160)) || !cbtbe::share(far(4096), far(4159));
    std::printf("%ld %ld\n", wrong, sharing);
}
