// What the entry points of the operators share: errors, the device of a call, launches.
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>
#include <string>

#include "../../include/klay.h"

namespace klay {

// Leaves the message for klay_last_error and returns the status.
__attribute__((visibility("hidden"))) klay_status report(klay_status status, const std::string& message);

// Makes `device` current for a call, and the earlier one again afterwards.
struct OnDevice {
    int before = -1;
    bool changed = false;
    hipError_t status;
    explicit OnDevice(int device) {
        status = hipGetDevice(&before);
        if (status == hipSuccess && before != device) {
            status = hipSetDevice(device);
            changed = status == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed) (void)hipSetDevice(before);
    }
};

constexpr int kComputeUnits = 256;
inline bool known_dtype(int32_t t) { return t == KLAY_F32 || t == KLAY_BF16 || t == KLAY_F16; }
inline int dtype_bytes(int32_t t) { return t == KLAY_F32 ? 4 : 2; }

// All of them multiples of `bytes`?
inline bool aligned_to(size_t bytes, std::initializer_list<const void*> all) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
    return bits % bytes == 0;
}

}  // namespace klay

// Launch errors come as the launch's own status; what an earlier call has left is none of ours.
#define KLAY_LAUNCH_SHARED(kernel, grid, block, shared, stream, ...)                                     \
    do {                                                                                                 \
        (void)hipGetLastError();                                                                         \
        hipLaunchKernelGGL(kernel, grid, block, shared, static_cast<hipStream_t>(stream), __VA_ARGS__);  \
        const hipError_t e__ = hipGetLastError();                                                        \
        if (e__ != hipSuccess)                                                                           \
            return klay::report(KLAY_EHIP, std::string("hipGetLastError(): ") + hipGetErrorString(e__)); \
    } while (0)
#define KLAY_LAUNCH(kernel, grid, block, stream, ...) KLAY_LAUNCH_SHARED(kernel, grid, block, 0, stream, __VA_ARGS__)
