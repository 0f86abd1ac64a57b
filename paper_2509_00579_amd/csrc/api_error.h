// How the C entry points report a failure: the status, and the text that kvcomp_last_error() returns on this thread.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/kvcomp.h"

namespace kvc {

__attribute__((format(printf, 2, 3))) kvcomp_status fail(kvcomp_status st, const char *fmt, ...);

}  // namespace kvc

#define HIP_TRY(expr)                                                                                   \
    do {                                                                                                \
        hipError_t e_ = (expr);                                                                         \
        if (e_ != hipSuccess) return kvc::fail(KVCOMP_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)
