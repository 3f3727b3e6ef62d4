// The steps of a scored block (csrc/paged_plan.hpp, cut) on the host: every token that
// some row may see lies in one step of one split, for any content of the spans, and no
// step lies outside the table.
#include <cstdio>
#include <initializer_list>
#include <random>
#include <set>

#include "paged_plan.hpp"

using namespace quarot::paged;

static int failures = 0;

#define CHECK(cond, ...)                      \
    do {                                      \
        if (!(cond) && ++failures < 20) {     \
            std::printf("FAIL %s: ", #cond);  \
            std::printf(__VA_ARGS__);         \
            std::printf("\n");                \
        }                                     \
    } while (0)

int main()
{
    std::mt19937 rng(1);
    for (int i = 0; i < 20000; ++i) {
        const int cap = 16 * (1 + (int)(rng() % 200));
        auto any = [&]() {
            const uint32_t r = rng();
            return r % 13 == 0 ? (int)rng() : (int)(rng() % (cap + 100)) - 50;
        };
        const int low = any(), hi = any(), sinks = rng() % 3 ? (int)(rng() % 300) : (int)(rng() >> 2);
        const int splits = 1 + (int)(rng() % 9), least = 1 + (int)(rng() % 8);
        Span w = span(0, 1, 5, 1, cap, 1, 0, 16, 0, 0, 1, 1);
        cut(w, low, hi, cap, sinks, splits, least);
        CHECK(w.hi >= 0 && w.hi <= cap && w.low >= 0 && w.low <= w.hi, "%d .. %d of %d", w.low, w.hi, cap);
        CHECK(w.used >= 1 && w.used <= splits && w.per >= 1, "%d splits of %d", w.used, w.per);
        CHECK((int64_t)w.used * w.per >= w.steps, "%d steps", w.steps);
        std::multiset<int> at;
        for (int s = 0; s < w.used; ++s)
            for (int k = s * w.per; k < w.steps && k < (s + 1) * w.per; ++k)
                at.insert(step_token(w, k) / STEP);
        CHECK((int)at.size() == w.steps, "%d of %d", (int)at.size(), w.steps);
        for (int t = 0; t < cap; ++t) {
            const bool seen = t < w.hi && (t >= low || t < sinks);
            CHECK(!seen || at.count(t / STEP) == 1, "token %d of %d .. %d, sinks %d", t, low, hi, sinks);
        }
        for (int b : at)
            CHECK(b >= 0 && b * STEP < cap + STEP, "step %d", b);
    }
    if (!failures)
        std::printf("ok\n");
    return failures != 0;
}
