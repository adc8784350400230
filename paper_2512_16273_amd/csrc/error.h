// Errors found on the host: the message that tslt_last_error() gives, and the code that the call returns.
#pragma once
#include <hip/hip_runtime.h>

namespace tslt {

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...);
int hip_fail(hipError_t e, const char* what);

}  // namespace tslt
