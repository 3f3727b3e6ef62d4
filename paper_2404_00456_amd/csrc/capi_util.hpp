// What the C ABI's source files share: argument rules, the device check and
// the error that quarot_last_hip_error() reports.  Host code only.
#pragma once

#include "../../include/quarot.h"

#include <cmath>

#include "common.hpp"

namespace quarot {

inline bool aligned16(const void *p)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
}

// RN32(1/sqrt(n)), through double (exact square root, one division).
inline float rotation_scale(int64_t n)
{
    return (float)(1.0 / std::sqrt((double)n));
}

inline bool clip_ok(float c)
{
    return c > 0.0f && c <= 1.0f;
}

// Records the error for quarot_last_hip_error() on this thread.
quarot_status hip_fail(hipError_t e);

// The calling thread's device must be a gfx950; `call` names the entry point
// (for the failure injection).
quarot_status check_device(const char *call);

}  // namespace quarot
