// Error reporting of the C entry points: the status goes back to the caller, the text to ttc_lqr_last_error.
#pragma once

#include <cuda_runtime.h>

#include "../../include/ttc_lqr.h"

namespace ttc {

// Sets the calling thread's error text and returns `status`.
int fail(int status, const char* fmt, ...);

} // namespace ttc

#define TTC_CUDA(call)                                                                   \
    do {                                                                                 \
        cudaError_t e_ = (call);                                                         \
        if (e_ != cudaSuccess)                                                           \
            return fail(TTC_STATUS_CUDA_ERROR, "%s: %s", #call, cudaGetErrorString(e_)); \
    } while (0)
