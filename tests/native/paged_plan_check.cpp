// The arithmetic of the paged attention's work (csrc/paged_plan.hpp) on the
// host: the division by a page size, the blocks of ragged batches, the steps of
// a block and their split, and the bounds of all of them for contents of cu_new
// and seq_lens that break the rules.
#include <cstdio>
#include <initializer_list>
#include <random>
#include <vector>

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

static void division(std::mt19937 &rng)
{
    for (int page = 16; page <= 4096; page += 16) {
        const Divisor d = divisor(page);
        auto quo = [&](uint32_t t) { return (uint32_t)(((uint64_t)t * d.mul) >> 32) >> d.sh; };
        for (int i = 0; i < 2000; ++i) {
            const uint32_t t = rng() >> 1;
            CHECK(quo(t) == t / page, "%u / %d", t, page);
        }
        for (uint32_t k : {0u, 1u, 2u, 1000u, 0x7FFFFFFFu / page})
            for (int o : {-1, 0, 1}) {
                const int64_t t = (int64_t)k * page + o;
                if (t >= 0 && t <= 0x7FFFFFFF)
                    CHECK(quo((uint32_t)t) == (uint32_t)t / page, "%lld / %d", (long long)t, page);
            }
    }
    for (int page : {1 << 20, (1 << 20) + 16, 1 << 30, (1 << 29) + 48, 999999984}) {
        const Divisor d = divisor(page);
        for (int64_t t : {int64_t(0), int64_t(page) - 1, int64_t(page), int64_t(page) + 1,
                          int64_t(0x7FFFFFFF), 2 * int64_t(page) - 1, 2 * int64_t(page)})
            if (t <= 0x7FFFFFFF)
                CHECK((uint32_t)(((uint64_t)t * d.mul) >> 32) >> d.sh == (uint32_t)(t / page),
                      "%lld / %d", (long long)t, page);
    }
}

// every row of a batch in exactly one block, every token that a row sees in
// exactly one step of that block
static void batches(std::mt19937 &rng)
{
    for (int round = 0; round < 3000; ++round) {
        const int B = 1 + rng() % 6, rep = 1 + rng() % 9;
        const int mr = std::vector<int>{32, 64, 128, 256}[rng() % 4];
        const int window = rng() % 3 ? 0 : 1 + rng() % 300, sinks = rng() % 90;
        const int splits = 1 + rng() % 9, least = 1 + rng() % 6;
        std::vector<int> cu(B + 1, 0), len(B);
        for (int b = 0; b < B; ++b) {
            const int n = rng() % 4 ? rng() % 5 : rng() % 400;
            cu[b + 1] = cu[b] + n;
            len[b] = n + (int)(rng() % 700) - (rng() % 8 ? 0 : 20);
        }
        const int T = cu[B] + rng() % 3, cap = rng() % 5 ? 2048 : 320;
        std::vector<int> seen((size_t)T * rep, 0);
        const int64_t total = slots(Part{ALL, mr, 1, 1}, T, B, rep);
        for (int64_t slot = 0; slot < total; ++slot)
            for (int b = 0; b < B; ++b) {
                const int64_t f = first_slot((int64_t)cu[b] * rep, b, mr);
                if (f > slot || slot >= first_slot((int64_t)cu[b + 1] * rep, b + 1, mr))
                    continue;
                const Span w = span(cu[b], cu[b + 1], len[b], T, cap, rep, slot - f, mr, window, sinks,
                                    splits, least);
                CHECK(w.used >= 1 && w.used <= splits, "used %d of %d", w.used, splits);
                if (!w.rows)
                    continue;
                CHECK((w.used == 1 || 2 * w.per >= least) && w.per * w.used >= w.steps && w.per * (w.used - 1) <= w.steps,
                      "steps");
                std::vector<char> walked((size_t)(std::max(w.hi, 0) + 2 * STEP), 0);
                for (int i = 0; i < w.steps; ++i) {
                    const int t0 = step_token(w, i);
                    CHECK(t0 >= 0 && t0 < w.hi, "step %d at %d of %d", i, t0, w.hi);
                    for (int t = t0; t < t0 + STEP; ++t)
                        ++walked[t];
                }
                for (int r = w.row0; r < w.row0 + mr && r < w.rows; ++r) {
                    ++seen[(size_t)(cu[b]) * rep + r];
                    const int p = w.pos0 + r / rep;
                    CHECK(w.pos0 == std::max(len[b], 0) - (cu[b + 1] - cu[b]), "pos");
                    for (int t = 0; t < cap; ++t) {
                        const bool see = t <= p && (window == 0 || t > p - window || t < sinks);
                        if (see)
                            CHECK(t < w.hi && (t >= w.low || t < sinks) && walked[t] == 1,
                                  "row %d token %d walked %d", r, t, t < w.hi ? walked[t] : -1);
                    }
                }
            }
        for (int r = 0; r < cu[B] * rep; ++r)
            CHECK(seen[r] == 1, "row %d seen %d times", r, seen[r]);
    }
}

// contents that break the rules: still inside the batch and the table
static void bad_contents(std::mt19937 &rng)
{
    const int odd[] = {-2147483647 - 1, -1, 0, 1, 7, 100, 1 << 30, 0x7FFFFFFF};
    for (int c0 : odd)
        for (int c1 : odd)
            for (int len : odd)
                for (int64_t block : {int64_t(-5), int64_t(0), int64_t(1), int64_t(1) << 20})
                    for (int window : {0, 1, 1 << 30})
                        for (int cap : {16, 1 << 30})
                            for (int T : {8, 1 << 30}) {
                                const Span w = span(c0, c1, len, T, cap, 1, block, 64, window,
                                                    window, 3, 4);
                                if (!w.rows)
                                    continue;
                                CHECK(c0 >= 0 && (int64_t)c0 + w.rows <= T && w.row0 >= 0 &&
                                          w.row0 < w.rows, "rows");
                                CHECK(w.hi >= 0 && w.hi <= cap && w.low >= 0 && w.low <= w.hi, "tokens");
                                CHECK(w.steps >= 0 && (w.steps == 0 ||
                                      step_token(w, w.steps - 1) < w.hi), "steps");
                            }
    (void)rng;
}

static void plans()
{
    bool taken[4] = {}, cut = false, two = false;
    for (int64_t T : {1, 2, 16, 64, 333, 2048, 16384, 1 << 20})
        for (int64_t B : {1, 2, 16, 64, 300, 5000})
            for (int64_t hkv : {1, 2, 8, 64})
                for (int64_t rep : {1, 4, 5, 8, 64})
                    for (int64_t D : {64, 128, 256})
                        for (int64_t len : {1, 64, 300, 4096, 32768, 1 << 30})
                            for (int64_t window : {0, 1, 1000, 1 << 30}) {
                                const Plan p = plan(T, B, hkv, rep, D, len, window,
                                                    1 << 30);
                                CHECK(p.n == 1 || p.n == 2, "launches");
                                // every sequence in one launch
                                CHECK(p.n == 1 ? p.part[0].which == ALL
                                               : p.part[0].which == MANY && p.part[1].which == FEW,
                                      "which");
                                for (int i = 0; i < p.n; ++i) {
                                    const Part &t = p.part[i];
                                    CHECK(t.least >= 1 && (int64_t)t.least * t.splits < 1 << 20, "least");
                                    CHECK(t.splits >= 1 && t.splits <= 128, "splits %d", t.splits);
                                    CHECK(t.rows == 16 || t.rows == 64 || t.rows == 128 || t.rows == 256, "rows");
                                    CHECK(t.which != FEW || t.rows == FEW_ROWS, "few");
                                    // partial rows of every block fit
                                    CHECK(t.splits == 1 || part_row(t.which, B - 1, T - 1, rep) <
                                                               part_rows(t, T, B, rep), "partial rows");
                                    taken[t.rows == 16 ? 0 : t.rows == 64 ? 1 : t.rows == 128 ? 2 : 3] = true;
                                    cut = cut || t.splits > 1;
                                }
                                two = two || p.n == 2;
                            }
    CHECK(taken[0] && taken[1] && taken[2] && taken[3] && cut && two, "a kernel is never taken");
}

int main()
{
    std::mt19937 rng(1);
    division(rng);
    batches(rng);
    bad_contents(rng);
    plans();
    if (!failures)
        std::printf("ok\n");
    return failures != 0;
}
