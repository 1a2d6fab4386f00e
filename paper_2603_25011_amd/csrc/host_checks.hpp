// Host-side checks and sizes that every entry point of the library shares.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "lsr_head.h"

namespace lsr {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline int check_device(int* n_cus) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); return LSR_ERR_ARCH; }
    static int ok_dev[64] = {0};     // holds the CU count once a device has been checked
    if (dev >= 0 && dev < 64 && ok_dev[dev]) { *n_cus = ok_dev[dev]; return LSR_OK; }
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) { (void)hipGetLastError(); return LSR_ERR_ARCH; }
    if (strncmp(prop.gcnArchName, "gfx950", 6) != 0) return LSR_ERR_ARCH;
    if (prop.multiProcessorCount < 1) return LSR_ERR_ARCH;
    *n_cus = prop.multiProcessorCount;
    if (dev >= 0 && dev < 64) ok_dev[dev] = prop.multiProcessorCount;
    return LSR_OK;
}

inline int launch_status() { return hipGetLastError() == hipSuccess ? LSR_OK : LSR_ERR_LAUNCH; }

}  // namespace lsr
