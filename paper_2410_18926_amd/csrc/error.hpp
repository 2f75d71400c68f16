// Error reporting and pointer classification shared by the library's translation units (defined in lorann.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/lorann.h"

namespace lorann {

// Stores the message for lorann_last_error() and returns `code`.
__attribute__((visibility("hidden"), format(printf, 2, 3))) int fail(int code, const char* fmt, ...);
// Device memory (or managed memory, which every GPU reaches); `gpu`: the GPU that it is on, -1 for managed memory.
__attribute__((visibility("hidden"))) bool is_device_ptr(const void* p, int* gpu = nullptr);

#define HIP_TRY(expr)                                                                                      \
    do {                                                                                                   \
        hipError_t e_ = (expr);                                                                            \
        if (e_ != hipSuccess)                                                                              \
            return fail(e_ == hipErrorOutOfMemory ? LORANN_E_NOMEM : LORANN_E_DEVICE, "%s failed: %s", #expr, \
                        hipGetErrorString(e_));                                                            \
    } while (0)

}  // namespace lorann
