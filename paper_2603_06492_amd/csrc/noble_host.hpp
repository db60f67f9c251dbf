// Host code that the entry points of libnoble share: pointer checks, the device check, the launch.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstring>

#include "noble.h"

namespace noble {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A required buffer: non-NULL and 16-byte aligned, unless it holds no bytes.
inline noble_status need(const void* p, bool nonempty) {
    if (!p) return nonempty ? NOBLE_ERR_NULL_ARG : NOBLE_OK;
    return aligned16(p) ? NOBLE_OK : NOBLE_ERR_MISALIGNED;
}
inline noble_status optional(const void* p) { return (!p || aligned16(p)) ? NOBLE_OK : NOBLE_ERR_MISALIGNED; }

#define NOBLE_TRY(expr)                              \
    do {                                             \
        noble_status s_ = (expr);                    \
        if (s_ != NOBLE_OK) return s_;               \
    } while (0)

// gfx950 check, cached per device ordinal (0 unknown, 1 ok, 2 unsupported).
inline std::atomic<int> g_arch_ok[256];

inline noble_status check_device(int* dev_out = nullptr) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return NOBLE_ERR_HIP;
    if (dev_out) *dev_out = dev;
    if (dev < 0 || dev >= 256) return NOBLE_ERR_UNSUPPORTED_DEVICE;
    int s = g_arch_ok[dev].load(std::memory_order_relaxed);
    if (s == 0) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return NOBLE_ERR_HIP;
        s = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? 1 : 2;
        g_arch_ok[dev].store(s, std::memory_order_relaxed);
    }
    return s == 1 ? NOBLE_OK : NOBLE_ERR_UNSUPPORTED_DEVICE;
}

// Launch of a kernel that takes one argument struct, with the status of this
// launch itself (the thread's last-error state would also carry, and clear,
// an earlier failure of the caller's).  lds: bytes for the kernel's own use beside those it declares.
template <typename Arg>
noble_status launch(void (*kernel)(Arg), dim3 grid, dim3 block, hipStream_t st, const Arg& arg, size_t lds = 0) {
    void* argv[] = {const_cast<Arg*>(&arg)};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, argv, lds, st) == hipSuccess
               ? NOBLE_OK
               : NOBLE_ERR_HIP;
}

inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace noble
