// Drives the host code of the scored attention, the pages and the sampling with no device:
// argument validation (null, negative, oversized and misaligned arguments, extreme sizes),
// the no-device path of valid calls and the workspace query.  Built with the address and
// undefined-behaviour sanitizers by tests/test_serving_host.py against counting stand-ins
// of the kernel launchers.
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <limits>

#include "../../paper_2404_00456_amd/csrc/pages.hpp"
#include "../../paper_2404_00456_amd/csrc/sample.hpp"
#include "quarot.h"

extern int quarot_stub_launches;  // tests/native/launch_stubs.cpp

namespace quarot {

static hipError_t count()
{
    ++quarot_stub_launches;
    return hipErrorInvalidValue;
}

hipError_t launch_paged_attention(const PagedAttnArgs &, int, hipStream_t) { return count(); }
hipError_t launch_scored_attention(const ScoredAttnArgs &, int, hipStream_t) { return count(); }
hipError_t launch_pages_fork(const ForkArgs &, hipStream_t) { return count(); }
hipError_t launch_pages_reserve(const ReserveArgs &, hipStream_t) { return count(); }
hipError_t launch_pages_compact(const CompactArgs &, hipStream_t) { return count(); }
hipError_t launch_pages_copy(const CopyArgs &, hipStream_t) { return count(); }
hipError_t launch_sample(const SampleArgs &, bool, int64_t, hipStream_t) { return count(); }

}  // namespace quarot

static int failures = 0;

#define EXPECT(call, want)                                                                   \
    do {                                                                                     \
        const long long got_ = (long long)(call);                                            \
        if (got_ != (long long)(want)) {                                                     \
            std::printf("FAIL line %d: %s -> %lld, want %lld\n", __LINE__, #call, got_,      \
                        (long long)(want));                                                  \
            ++failures;                                                                      \
        }                                                                                    \
    } while (0)

int main()
{
    void *P = reinterpret_cast<void *>(uintptr_t(1) << 20);
    quarot_f16 *H = static_cast<quarot_f16 *>(P);
    quarot_f16 *O = reinterpret_cast<quarot_f16 *>((uintptr_t(1) << 20) + 4096);
    int32_t *I = static_cast<int32_t *>(P);
    float *F = static_cast<float *>(P);
    const int64_t BIG = INT64_MAX, LOW = INT64_MIN;
    uint8_t *C = static_cast<uint8_t *>(P);

    const quarot_paged_kv kv = {C, H, H, C, H, H, I, I, I, 2, 2, 128, 128, 9, 16, 4};
    auto scored = [&](quarot_scoring s, int64_t T = 8, int64_t heads = 8, int64_t most = 64,
                      int64_t window = 0, int64_t sinks = 0, int64_t stride = 1024) {
        return quarot_kv_paged_attention_scored(H, stride, O, 1024, &kv, &s, T, heads, most, window, sinks, 0.1f,
                                                P, size_t(1) << 40, nullptr);
    };
    for (float cap : {0.0f, 1.0f, 0x1p-64f, 0x1p64f})
        EXPECT(scored({cap, F, I, I}), QUAROT_ERR_NO_DEVICE);
    EXPECT(scored({0, nullptr, nullptr, nullptr}), QUAROT_ERR_NO_DEVICE);
    EXPECT(scored({1e30f, nullptr, nullptr, nullptr}), QUAROT_ERR_UNSUPPORTED_SIZE);
    EXPECT(scored({-0x1p-140f, nullptr, nullptr, nullptr}), QUAROT_ERR_INVALID_ARG);
    EXPECT(scored({std::numeric_limits<float>::quiet_NaN(), nullptr, nullptr, nullptr}), QUAROT_ERR_INVALID_ARG);
    for (int64_t x : {BIG, LOW}) {
        const bool big = x > 0;
        EXPECT(scored({1, F, I, I}, x), big ? QUAROT_ERR_UNSUPPORTED_SIZE : QUAROT_ERR_INVALID_ARG);
        EXPECT(scored({1, F, I, I}, 8, x), QUAROT_ERR_INVALID_ARG);
        EXPECT(scored({1, F, I, I}, 8, 8, x), big ? QUAROT_ERR_NO_DEVICE : QUAROT_ERR_INVALID_ARG);
        EXPECT(scored({1, F, I, I}, 8, 8, 64, x), big ? QUAROT_ERR_NO_DEVICE : QUAROT_ERR_INVALID_ARG);
        EXPECT(scored({1, F, I, I}, 8, 8, 64, 0, x), big ? QUAROT_ERR_NO_DEVICE : QUAROT_ERR_INVALID_ARG);
        EXPECT(scored({1, F, I, I}, 8, 8, 64, 0, 0, x), big ? QUAROT_ERR_UNSUPPORTED_SIZE : QUAROT_ERR_INVALID_ARG);
    }

    auto fork = [&](int64_t B, int64_t most, int64_t n) {
        return quarot_kv_pages_fork(I, I, I, I, B, most, n, nullptr);
    };
    auto reserve = [&](int64_t B, int64_t most, int64_t n, int64_t page) {
        return quarot_kv_pages_reserve(I, I, I, I, I, I, I, I, B, most, n, page, P, size_t(1) << 40, nullptr);
    };
    auto compact = [&](int64_t B, int64_t most, int64_t n) {
        return quarot_kv_pages_compact(I, I, I, I, I, B, most, n, P, size_t(1) << 40, nullptr);
    };
    EXPECT(fork(16384, 1 << 26, 1 << 30), QUAROT_ERR_NO_DEVICE);
    EXPECT(reserve(16384, 1 << 26, 1 << 30, 16), QUAROT_ERR_NO_DEVICE);
    EXPECT(reserve(1, 1, 1, 1 << 30), QUAROT_ERR_NO_DEVICE);
    EXPECT(compact(16384, 1 << 26, 1 << 30), QUAROT_ERR_NO_DEVICE);
    for (int64_t x : {BIG, LOW, (int64_t)0}) {
        const quarot_status st = x > 0 ? QUAROT_ERR_UNSUPPORTED_SIZE : QUAROT_ERR_INVALID_ARG;
        EXPECT(fork(x, 4, 9), st);
        EXPECT(fork(2, x, 9), st);
        EXPECT(fork(2, 4, x), st);
        EXPECT(reserve(x, 4, 9, 16), st);
        EXPECT(reserve(2, x, 9, 16), st);
        EXPECT(reserve(2, 4, x, 16), st);
        EXPECT(reserve(2, 4, 9, x), st);
        EXPECT(compact(x, 4, 9), st);
        EXPECT(quarot_kv_pages_workspace_size(x), 0);
        EXPECT(quarot_kv_pages_copy(&kv, I, I, x, nullptr), x ? st : QUAROT_OK);
        quarot_paged_kv bad = kv;
        bad.page_size = x;
        EXPECT(quarot_kv_pages_copy(&bad, I, I, 3, nullptr), st);
        bad = kv;
        bad.n_pages = x;
        EXPECT(quarot_kv_pages_copy(&bad, I, I, 3, nullptr), st);
        bad = kv;
        bad.n_kv_heads = x;
        EXPECT(quarot_kv_pages_copy(&bad, I, I, 3, nullptr), st);
    }
    EXPECT(quarot_kv_pages_copy(&kv, I, I, int64_t(1) << 30, nullptr), QUAROT_ERR_NO_DEVICE);
    EXPECT(quarot_kv_pages_workspace_size(int64_t(1) << 30), size_t(1) << 34);

    auto sample = [&](int64_t rows, int64_t vocab, int64_t stride) {
        return quarot_sample(P, stride, 0, F, F, I, F, F, I, rows, vocab, nullptr);
    };
    EXPECT(sample(5, 1 << 20, 1 << 20), QUAROT_ERR_NO_DEVICE);
    EXPECT(sample(1, 1, LOW), QUAROT_ERR_NO_DEVICE);
    EXPECT(sample(0, 7, 7), QUAROT_OK);
    EXPECT(sample(BIG, 7, 7), QUAROT_ERR_UNSUPPORTED_SIZE);
    EXPECT(sample(LOW, 7, 7), QUAROT_ERR_INVALID_ARG);
    EXPECT(sample(2, BIG, BIG), QUAROT_ERR_UNSUPPORTED_SIZE);
    EXPECT(sample(2, LOW, 7), QUAROT_ERR_INVALID_ARG);
    EXPECT(sample(2, 7, BIG), QUAROT_ERR_UNSUPPORTED_SIZE);
    EXPECT(sample(2, 7, LOW), QUAROT_ERR_INVALID_ARG);
    EXPECT(quarot_stub_launches, 0);
    if (!failures)
        std::printf("ok\n");
    return failures != 0;
}
