// The arithmetic of the paged attention's work: positions to pages, the blocks
// of a ragged batch, the steps of a block and their split, and the host's choice
// of kernel.  Plain C++ with no HIP, so that it builds and is checked on any
// host; what kernels run of it is marked QUAROT_HD.
#pragma once

#include <algorithm>
#include <cstdint>

#if defined(__HIP__)
#define QUAROT_HD __host__ __device__ inline
#else
#define QUAROT_HD inline
#endif

namespace quarot {
namespace paged {

constexpr int STEP = 64;          // tokens of a step
constexpr int FEW_ROWS = 16;      // query rows of a block of the kernel for single tokens
constexpr int MAX_THREADS = 512;  // of an attention block

// t / page = (t * mul >> 32) >> sh for 0 <= t < 2^31: with L = ceil(log2(page))
// and mul = floor(2^(31 + L) / page) + 1 (below 2^32, page >= 2),
// t mul / 2^(31 + L) exceeds t / page by less than 1 / page, which changes no
// quotient.
struct Divisor {
    uint32_t mul;
    int sh;
};

inline Divisor divisor(int page)
{
    int L = 1;
    while ((int64_t(1) << L) < page)
        ++L;
    return Divisor{(uint32_t)(((uint64_t)1 << (31 + L)) / (uint64_t)page + 1), L - 1};
}

// Blocks of MR query rows (new tokens times query heads of a cache head) of a
// ragged batch: sequence b takes the slots from first_slot(cu[b] rep, b, MR) to
// that of b + 1, at least as many as its rows fill (the floor of a sum is no
// less than the sum of floors, and b adds one for each sequence), so a block
// finds its sequence from two entries of cu and no sum over those before it.
QUAROT_HD int64_t first_slot(int64_t rows_before, int64_t b, int mr)
{
    return rows_before / mr + b;
}

// What a block works on.
struct Span {
    int row0, rows;  // first row, rows of the sequence; rows 0: nothing to do
    int pos0;        // position of the sequence's first new token
    int hi, low;     // tokens low .. hi - 1 and the sinks are seen by some row
    int lo, first;   // steps 0 .. lo - 1 are sinks, step i >= lo is token block i - lo + first
    int steps;       // in all
    int per, used;   // steps of a split, splits that have any (1 at least)
};

// The steps of a block whose rows see tokens low .. hi - 1 and the sinks before hi, and
// their splits.
QUAROT_HD void share(Span &w, int splits, int least)
{
    w.used = (w.steps + least - 1) / least;
    w.used = w.used < 1 ? 1 : w.used > splits ? splits : w.used;
    w.per = (w.steps + w.used - 1) / w.used;
    w.per = w.per > 1 ? w.per : 1;
    w.used = (w.steps + w.per - 1) / w.per;
    w.used = w.used > 1 ? w.used : 1;
}

QUAROT_HD void cut(Span &w, int low, int hi, int cap, int sinks, int splits, int least)
{
    w.hi = hi > cap ? cap : hi < 0 ? 0 : hi;
    w.low = low < 0 ? 0 : low > w.hi ? w.hi : low;
    w.first = w.low / STEP;
    w.lo = ((sinks < w.hi ? sinks : w.hi) + STEP - 1) / STEP;
    w.lo = w.lo < w.first ? w.lo : w.first;
    w.steps = (w.hi + STEP - 1) / STEP + w.lo - w.first;
    share(w, splits, least);
}

// Sequence of rows cu0 .. cu1 - 1 of a batch of T, len cached tokens; block
// `slot - first_slot` of it; a table of cap positions; window 0: none; at most
// `splits` equal splits, for each `least` steps one.  Any content of cu0, cu1 and len gives a span inside the
// batch and the table.  cap and T are at most 2^30, window and sinks too.
QUAROT_HD Span span(int cu0, int cu1, int len, int T, int cap, int rep, int64_t block, int mr,
                    int window, int sinks, int splits, int least)
{
    Span w = {};
    const int64_t row0 = block * mr, rows = ((int64_t)cu1 - cu0) * rep;
    w.used = 1;
    if (cu0 < 0 || cu1 > T || block < 0 || row0 >= rows)
        return w;
    const int n = cu1 - cu0;
    len = len < 0 ? 0 : len;
    w.row0 = (int)row0;
    w.rows = (int)rows;
    w.pos0 = len - n;
    const int last = (int)(row0 + mr < rows ? row0 + mr : rows) - 1;
    const int p0 = w.pos0 + w.row0 / rep, p1 = w.pos0 + last / rep;
    w.hi = p1 + 1 > cap ? cap : p1 + 1 < 0 ? 0 : p1 + 1;
    w.steps = (w.hi + STEP - 1) / STEP;
    if (window > 0) {
        w.low = p0 - window + 1 < 0 ? 0 : p0 - window + 1 > w.hi ? w.hi : p0 - window + 1;
        w.first = w.low / STEP;
        w.lo = ((sinks < w.hi ? sinks : w.hi) + STEP - 1) / STEP;
        w.lo = w.lo < w.first ? w.lo : w.first;
        w.steps += w.lo - w.first;
    }
    share(w, splits, least);
    return w;
}

// First token of step i.
QUAROT_HD int step_token(const Span &w, int i)
{
    return (i < w.lo ? i : i - w.lo + w.first) * STEP;
}

// Which sequences a launch works on, by their query rows.  FEW takes a block row
// for each sequence, the others one for each slot.
enum Which { ALL, MANY /* more than FEW_ROWS */, FEW /* at most FEW_ROWS */ };

struct Part {
    Which which;
    int rows;    // query rows of a block
    int splits;  // blocks that share a block row's tokens, at most
    int least;   // steps of a split, at least
};

struct Plan {
    int n;  // launches
    Part part[2];
};

// Block rows of a launch.
inline int64_t slots(const Part &p, int64_t T, int64_t B, int64_t rep)
{
    return p.which == FEW ? B : T * rep / p.rows + B;
}

// Rows that a launch keeps partial results of: those of a sequence from
// part_row(...) on.
inline int64_t part_rows(const Part &p, int64_t T, int64_t B, int64_t rep)
{
    return p.splits == 1 ? 0 : p.which == FEW ? B * FEW_ROWS : T * rep;
}

QUAROT_HD int64_t part_row(Which which, int64_t b, int64_t tok0, int64_t rep)
{
    return which == FEW ? b * FEW_ROWS : tok0 * rep;
}

// Few rows: splits of such a length that 512 of them, two a CU, hold the steps of a
// batch of full sequences.  Shorter ones pay for their starts and their joining (64
// sequences of 1024 tokens and 8 heads: 27 us in splits of 8 steps, 21 whole; 256
// of 1 .. 2048 tokens: 97 and 75), longer ones leave CUs idle behind the longest
// (64 of 1 .. 8192: 73 us in splits of 32 steps, 89 of 64), and few steps do best
// in pieces of 4 (one of 4096: 10.5 us, 13 of 8, 21 of 24; but one of 32768: 22 of
// 4, 19 of 8).  8192 blocks at most, which bounds the workspace as well.
// Beside long sequences there are fewer than B of them (a mixed batch of 16: 291 us
// for 512, 285 for 2048).
inline Part few_part(Which which, int64_t steps, int64_t B, int64_t hkv)
{
    const int fill = which == FEW ? 2048 : 512;
    const int64_t rows = std::min<int64_t>(B * hkv, 1 << 20);
    const int least = (int)std::min<int64_t>(32, std::max<int64_t>(4, steps * rows / fill));
    const int64_t splits = std::min<int64_t>({(steps + least - 1) / least, 128, 8192 / (B * hkv)});
    return Part{which, FEW_ROWS, (int)std::max<int64_t>(1, splits), least};
}

// Tiles: 256 blocks, one a CU as LDS holds them (two of the 64-row tile): a second
// turn of blocks costs more than the joining of fewer splits saves (512 new tokens
// over 16384, 64 heads on 8: 319 us in 256 blocks, 329 in 512; 4 x 64 over 8192: 70
// and 101; 64-row tiles that 16 sequences of one row fill: 142 us in 512 blocks, 223
// in 256).
inline Part tile_part(Which which, int64_t steps, int64_t rows, int64_t T, int64_t B, int64_t hkv,
                      int64_t rep, int64_t D)
{
    Part p{which, D == 256 ? 128 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256, 1, 4};
    const int64_t blocks = hkv * std::max<int64_t>((T * rep + p.rows - 1) / p.rows, which == MANY ? 1 : B);
    const int64_t fill = (p.rows == 64 ? 512 : 256) / blocks;
    // (slots that no sequence fills cost a start each)
    const int64_t most = 2048 / (hkv * slots(p, T, B, rep));
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(steps + 3) / 4, fill, most, 128}));
    return p;
}

// T new tokens of B sequences, hkv cache heads with rep query heads each, at
// most max_len cached tokens.  Only a rule of speed: any content of cu and len
// is right under any plan.
inline Plan plan(int64_t T, int64_t B, int64_t hkv, int64_t rep, int64_t D,
                 int64_t max_len, int64_t window, int64_t sinks)
{
    // query rows of a sequence: on average, and of the longest at most (where
    // the others have a token each)
    const int64_t rows = (T * rep + B - 1) / B, most = std::max<int64_t>(T - B + 1, 1) * rep;
    const int64_t seen = window > 0 ? std::min(max_len, window + sinks + T / B) : max_len;
    const int64_t steps = (seen + STEP - 1) / STEP;
    if (rep > FEW_ROWS || (B == 1 && rows > FEW_ROWS))
        return Plan{1, {tile_part(ALL, steps, rows, T, B, hkv, rep, D)}};
    // Sequences of few rows: guessed tokens of 64 sequences, 16 rows each, take 66 us
    // so and 92 with a launch for longer ones beside; but a batch of single tokens
    // may hold a chunk of all the rest, which the tiles read four times as fast, so
    // only up to 1024 rows of it.  (300 sequences with 4 rows a token: 900 tokens of one
    // over 16384 and a token each of the others 550 us by two launches, 600 so; 3 tokens
    // each over 2048 lose by it, 163 and 145.)
    if (rows <= FEW_ROWS && most <= 64 * FEW_ROWS)
        return Plan{1, {few_part(ALL, steps, B, hkv)}};
    // Chunks, with single tokens among them maybe: 64 sequences, half of them one
    // token, 244 us so and 285 in tiles alone, where nothing but chunks loses 4 us.  The
    // tiles are for a chunk of up to all the rest, which a quarter of that stands for:
    // 64 sequences with 8 rows a token over 4096, 193 tokens of one and one each of the
    // others 155 us so and 210 in tiles for the average.  Short chunks alike have the same
    // sizes here and pay for it: 4 tokens each 357 us so, 274 by the average, 164 in
    // blocks of FEW_ROWS rows, which the 193 over 16384 would lose by (244 and 318).
    return Plan{2, {tile_part(MANY, steps, std::max(rows, most / 4), T, B, hkv, rep, D),
                    few_part(FEW, steps, B, hkv)}};
}

}  // namespace paged
}  // namespace quarot
