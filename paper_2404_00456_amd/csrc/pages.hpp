// The pages of the 4-bit KV cache: what their kernels and their entry points share.
#pragma once

#include "paged.hpp"

namespace quarot {

constexpr int PAGES_MAX_BATCH = 16384;  // sequences of a table (an int each in LDS)

// A table of sequences, their lengths, and for each page the number of entries that hold
// it (0: it is free).
struct PagesArgs {
    int32_t *table;  // [B, P]
    int32_t *lens;   // [B]
    int32_t *refs;   // [n]
    int B, P, n;
};

struct ForkArgs : PagesArgs {
    const int32_t *parent;  // [B]
};

struct ReserveArgs : PagesArgs {
    const int32_t *n_new;     // [B]
    int32_t *cu, *src, *dst;  // [B + 1], [B], [B]
    int32_t *missing;         // [1]
    int32_t *ws;              // [4 n]
    int page;
    paged::Divisor div;       // by page
};

struct CompactArgs : PagesArgs {
    int32_t *src, *dst;  // [n / 2]
    int32_t *live;       // [1]
    int32_t *ws;         // [n]
};

struct CopyArgs {
    PagedPool kp, vp;
    const int32_t *src, *dst;  // [count]
    int count, n;
    int64_t code_bytes, const_bytes;  // of a page's codes, and of its scales or zeros
};

hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t s);
hipError_t launch_pages_reserve(const ReserveArgs &a, hipStream_t s);
hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s);
hipError_t launch_pages_copy(const CopyArgs &a, hipStream_t s);

}  // namespace quarot
