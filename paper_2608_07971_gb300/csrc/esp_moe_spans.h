// Whether matrices in memory have a byte in common (host): results that must not lie over what a call still reads.
#pragma once

#include <cstdint>
#include <initializer_list>

namespace esp_moe_impl {

// `rows` rows of `width` bytes, `step` apart (at least `width`, where there are several); nothing where p is null.
struct Span {
    const void *p;
    int64_t rows, step, width;
};

// Columns of one matrix side by side have no byte in common. Of matrices with different steps whose rows are interleaved
// it may say that they meet where they do not.
inline bool meet(Span a, Span b)
{
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0)
        return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const auto length = [](const Span &s) { return (unsigned __int128)(s.rows - 1) * s.step + s.width; };   // past 64 bits: of a wrong step
    if (pa + length(a) <= pb || pb + length(b) <= pa)
        return false;
    if (a.rows == 1)
        a.step = b.step;
    if (b.rows == 1)
        b.step = a.step;
    if (a.step != b.step || (a.rows == 1 && b.rows == 1))
        return true;
    // where b's rows begin behind the beginning of one of a's
    const uintptr_t step = (uintptr_t)a.step, at = pb >= pa ? (pb - pa) % step : (step - (pa - pb) % step) % step;
    return at < (uintptr_t)a.width || at + b.width > step;
}

// Whether one of the written matrices meets another one, or one of those that are read.
inline bool written_over(std::initializer_list<Span> written, std::initializer_list<Span> read)
{
    for (const Span *w = written.begin(); w != written.end(); ++w) {
        for (const Span *o = w + 1; o != written.end(); ++o)
            if (meet(*w, *o))
                return true;
        for (const Span &r : read)
            if (meet(*w, r))
                return true;
    }
    return false;
}

}  // namespace esp_moe_impl
