// Host-side argument checks and status conversion shared by the C-ABI translation units.
#pragma once

#include <atomic>

#include "smile_internal.hpp"

namespace smile {

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// required pointer: non-NULL and 16-byte aligned
inline bool bad(const void *p) { return p == nullptr || !aligned16(p); }
// optional pointer: NULL or 16-byte aligned
inline bool bad_opt(const void *p) { return p != nullptr && !aligned16(p); }

inline smile_status from_hip(hipError_t e)
{
    if (e == hipSuccess) return SMILE_OK;
    (void)hipGetLastError();   // do not leave a sticky launch error behind for the caller's next call
    return SMILE_HIP_ERROR;
}

// The compute units of the current device, asked for once per device
inline Tuning device_tuning()
{
    constexpr int kDevices = 64;
    static std::atomic<int> known_cus[kDevices];
    Tuning t;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices) {
        (void)hipGetLastError();
        return t;
    }
    int cus = known_cus[dev].load(std::memory_order_relaxed);
    if (cus == 0) {
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
            (void)hipGetLastError();
            return t;
        }
        known_cus[dev].store(cus, std::memory_order_relaxed);
    }
    t.cus = cus;
    return t;
}

}  // namespace smile
