// Matrices in memory that meet (csrc/esp_moe_spans.h), against their bytes: never missed, and never said of columns of one
// matrix, of single rows, or of ranges apart.

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "esp_moe_spans.h"

using namespace esp_moe_impl;

int main()
{
    std::mt19937 rng(1);
    const auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    unsigned char *const at = reinterpret_cast<unsigned char *>((uintptr_t)1 << 32);   // not looked at
    long met = 0, apart = 0;
    for (int i = 0; i < 400000; ++i) {
        std::vector<int> bytes(600, 0);
        Span s[2];
        bool common = false;
        for (int k = 0; k < 2; ++k) {
            const int width = pick(0, 8), step = k == 1 && pick(0, 2) ? (int)s[0].step : width + pick(0, 12);
            const int from = pick(0, 60);
            s[k] = Span{at + from, pick(0, 5), step, step < width ? step : width};
            for (int r = 0; r < s[k].rows; ++r)
                for (int c = 0; c < s[k].width; ++c) {
                    int &b = bytes[from + r * step + c];
                    common = common || (k == 1 && b);
                    b |= k == 0;
                }
        }
        const bool said = meet(s[0], s[1]);
        // exact where the steps are the same, or a row is alone
        const bool exact = s[0].step == s[1].step || s[0].rows == 1 || s[1].rows == 1;
        if (said != meet(s[1], s[0]) || (common && !said) || (exact && said != common)) {
            printf("said %d, common %d: %ld x %ld by %ld at %ld, %ld x %ld by %ld at %ld\n", said, common, (long)s[0].rows,
                   (long)s[0].width, (long)s[0].step, (long)((unsigned char *)s[0].p - at), (long)s[1].rows, (long)s[1].width,
                   (long)s[1].step, (long)((unsigned char *)s[1].p - at));
            return 1;
        }
        ++(said ? met : apart);
    }
    const Span far{at, (int64_t)1 << 31, (int64_t)1 << 40, 4}, in{at + ((int64_t)1 << 50) + 2, 1, 1, 1};
    if (!meet(far, in) || !meet(in, far) || meet(far, Span{at + ((int64_t)1 << 50) + 4, 1, 1, 1})) {
        printf("long steps\n");
        return 1;
    }
    const Span a{at, 4, 10, 4}, b{at + 5, 4, 10, 5}, c{at + 39, 1, 1, 1}, none{nullptr, 4, 10, 4};
    if (met < 10000 || apart < 10000 || written_over({a, b}, {none}) || !written_over({a, b}, {c}) || !written_over({c, b}, {}) ||
        written_over({a}, {b}) || !written_over({a}, {a}) || written_over({}, {a, a})) {
        printf("lists\n");
        return 1;
    }
    printf("ok\n");
}
