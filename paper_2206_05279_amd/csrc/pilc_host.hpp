// What the library's translation units share on the host: how a failure of the HIP runtime is reported.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/pilc.h"

namespace pilc {

// Keeps the text for pilc_last_hip_error and returns PILC_E_HIP.
int hip_fail(hipError_t e, const char *what);

uint32_t compute_units();

}  // namespace pilc

#define HIP_TRY(expr)                                   \
    do {                                                \
        hipError_t e_ = (expr);                         \
        if (e_ != hipSuccess) return pilc::hip_fail(e_, #expr); \
    } while (0)
