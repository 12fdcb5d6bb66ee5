// Error reporting of the C entries, shared by the host sources.
#pragma once

#include <hip/hip_runtime.h>

namespace lif {

// Writes the message of lif_last_error_string (one per thread) and returns `code`.
int fail(int code, const char* fmt, const char* detail = "");

}  // namespace lif

#define LIF_HIP(call)                                                             \
    do {                                                                          \
        hipError_t e_ = (call);                                                   \
        if (e_ != hipSuccess) return lif::fail(LIF_HIP_ERROR, #call ": %s", hipGetErrorString(e_)); \
    } while (0)
