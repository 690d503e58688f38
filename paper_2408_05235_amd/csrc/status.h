// Errors of the C ABI: each returns the status and keeps the calling thread's
// message for tl_last_error (api.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "tl.h"

namespace tl {

tl_status fail(tl_status st, const char* fmt, ...);
tl_status ok();
tl_status from_hip(hipError_t e, const char* what);

}  // namespace tl
