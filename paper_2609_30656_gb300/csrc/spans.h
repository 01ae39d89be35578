// spans.h -- whether two strided tensors share memory (host).
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>

namespace cbtbe {

using wide = __int128;  // strides and counts are any that fit 64 bits

// Rows of `width` bytes at begin + i * step, i < n, for up to three such strides (in bytes, not negative).
struct Span {
    static constexpr int kLevels = 3;
    uintptr_t begin = 0;
    wide end = 0;    // behind the last byte
    wide width = 0;  // 0: nothing
    int levels = 0;
    int64_t n[kLevels], step[kLevels];

    Span() = default;
    Span(const void* p, int64_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(begin), width(p && bytes > 0 ? bytes : 0) {
        end += width;
    }
    Span& by(int64_t count, int64_t stride_bytes) {
        if (count <= 0) {
            width = 0;
        } else if (count > 1 && stride_bytes > 0 && width > 0) {
            n[levels] = count;
            step[levels++] = stride_bytes;
            end += static_cast<wide>(count - 1) * stride_bytes;
        }
        return *this;
    }
    bool reaches(const Span& o) const { return end > static_cast<wide>(o.begin) && o.end > static_cast<wide>(begin); }
};

namespace spans {

// The largest stride first, each once, rows that follow one another without a gap as one.
inline void tidy(Span& a) {
    for (int k = 1; k < a.levels; ++k)
        for (int i = k; i > 0 && a.step[i] > a.step[i - 1]; --i) {
            std::swap(a.step[i], a.step[i - 1]);
            std::swap(a.n[i], a.n[i - 1]);
        }
    for (int k = a.levels - 1; k > 0; --k)
        if (a.step[k] == a.step[k - 1]) {  // one stride in two dimensions
            a.n[k - 1] += a.n[k] - 1;
            for (int i = k; i + 1 < a.levels; ++i) {
                a.n[i] = a.n[i + 1];
                a.step[i] = a.step[i + 1];
            }
            --a.levels;
        }
    while (a.levels && a.step[a.levels - 1] <= a.width) {
        --a.levels;
        a.width += static_cast<wide>(a.n[a.levels] - 1) * a.step[a.levels];
    }
}
inline wide floor_div(wide a, wide b) { return a / b - (a % b != 0 && a < 0); }
// Both with strides among two: d of the larger and e of the smaller apart, rows meet where -b.width < D + d s0 + e s1 < a.width.
inline bool meet(const Span& a, const Span& b, const wide (&s)[2], int64_t& looks) {
    auto count = [&](const Span& x, int which) {
        for (int k = 0; k < x.levels; ++k)
            if (x.step[k] == s[which]) return static_cast<wide>(x.n[k]);
        return wide{1};
    };
    const wide D = static_cast<wide>(b.begin) - static_cast<wide>(a.begin);
    const wide na = count(a, 0), nb = count(b, 0), ma = s[1] ? count(a, 1) : 1, mb = s[1] ? count(b, 1) : 1;
    auto between = [](wide low, wide high, wide step, wide least, wide most, wide& from, wide& to) {  // low < k * step < high
        from = std::max(least, floor_div(low, step) + 1);
        to = std::min(most, floor_div(high - 1, step));
    };
    wide d0, d1;
    between(-b.width - D - (mb - 1) * s[1], a.width - D + (ma - 1) * s[1], s[0], 1 - na, nb - 1, d0, d1);
    for (wide d = d0; d <= d1; ++d) {
        const wide x = D + d * s[0];
        if (!s[1]) return true;
        wide e0, e1;
        between(-b.width - x, a.width - x, s[1], 1 - ma, mb - 1, e0, e1);
        if (e0 <= e1 || --looks < 0) return true;
    }
    return false;
}
inline bool share(const Span& a, const Span& b, int64_t& looks) {
    if (!a.reaches(b)) return false;
    wide s[2] = {0, 0};
    int different = 0;
    for (const Span* x : {&a, &b})
        for (int k = 0; k < x->levels; ++k) {
            if (std::find(s, s + std::min(different, 2), static_cast<wide>(x->step[k])) != s + std::min(different, 2)) continue;
            if (different < 2) s[different] = x->step[k];
            ++different;
        }
    if (different == 0) return true;
    if (s[0] < s[1]) std::swap(s[0], s[1]);
    if (different <= 2) return meet(a, b, s, looks);
    // Three strides or more: the rows of one, along its largest, by themselves.
    const bool of_a = a.levels && (!b.levels || a.n[0] <= b.n[0]);
    Span part = of_a ? a : b;
    const int64_t n = part.n[0], step = part.step[0];
    part.end -= static_cast<wide>(n - 1) * step;
    for (int k = 1; k < part.levels; ++k) {
        part.n[k - 1] = part.n[k];
        part.step[k - 1] = part.step[k];
    }
    --part.levels;
    for (int64_t i = 0; i < n; ++i, part.begin += static_cast<uintptr_t>(step), part.end += step)
        if (--looks < 0 || share(of_a ? part : a, of_a ? b : part, looks)) return true;
    return false;
}

}  // namespace spans

// Whether two tensors have a byte in common. Where they lie between one another in strides of three kinds and more it is looked
// for up to 2^16 times, and taken for granted then.
inline bool share(const Span& x, const Span& y) {
    if (x.width <= 0 || y.width <= 0 || !x.reaches(y)) return false;
    Span a = x, b = y;
    spans::tidy(a);
    spans::tidy(b);
    int64_t looks = 1 << 16;
    return spans::share(a, b, looks);
}
// Whether what is written shares memory with something else that is written, or read.
inline bool overlap(std::initializer_list<Span> written, std::initializer_list<Span> read) {
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (auto o = w + 1; o != written.end(); ++o)
            if (share(*w, *o)) return true;
        for (const Span& r : read)
            if (share(*w, r)) return true;
    }
    return false;
}

}  // namespace cbtbe
