// Argument checks shared by the C-ABI sources (host only).
#pragma once

#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>

#include <hip/hip_runtime.h>

#include "forge.h"

namespace {

constexpr int64_t kMaxElems = (int64_t(1) << 31) - 1;

struct Range {
    uintptr_t lo, hi;   // [lo, hi)
};

inline bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

inline Range range_of(const void *p, int64_t bytes)
{
    uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Range{lo, lo + static_cast<uintptr_t>(bytes)};
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool finite(float x) { return std::isfinite(x); }

inline forge_status check_hyper(float lr, float b1, float b2, float eps, float wd, int64_t step)
{
    if (step < 1) return FORGE_ERR_INVALID_HYPERPARAM;
    if (!finite(lr) || !finite(b1) || !finite(b2) || !finite(eps) || !finite(wd))
        return FORGE_ERR_INVALID_HYPERPARAM;
    if (!(b1 >= 0.0f && b1 < 1.0f) || !(b2 >= 0.0f && b2 < 1.0f)) return FORGE_ERR_INVALID_HYPERPARAM;
    if (!(eps > 0.0f) || !(lr >= 0.0f)) return FORGE_ERR_INVALID_HYPERPARAM;
    return FORGE_OK;
}

// The current device must be a gfx950; the answer is cached per device ordinal.
inline forge_status check_device()
{
    static std::mutex mu;
    static int known[64] = {0};   // 0 unknown, 1 ok, 2 not ok
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) {
        (void)hipGetLastError();
        return FORGE_ERR_NO_DEVICE;
    }
    if (dev >= 64) return FORGE_ERR_NO_DEVICE;
    std::lock_guard<std::mutex> lock(mu);
    if (known[dev] == 0) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) {
            (void)hipGetLastError();
            return FORGE_ERR_NO_DEVICE;
        }
        known[dev] = (std::strncmp(prop.gcnArchName, "gfx950", 6) == 0) ? 1 : 2;
    }
    return known[dev] == 1 ? FORGE_OK : FORGE_ERR_NO_DEVICE;
}

inline forge_status from_hip(hipError_t e)
{
    if (e == hipSuccess) return FORGE_OK;
    if (e == hipErrorNoDevice || e == hipErrorInvalidDevice) return FORGE_ERR_NO_DEVICE;
    return FORGE_ERR_LAUNCH;
}

}  // namespace
