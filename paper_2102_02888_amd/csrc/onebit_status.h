// Failure reporting shared by the C ABI's source files: both functions describe
// the failure for onebit_last_error() (per thread) and return the status.
#pragma once

#include <hip/hip_runtime.h>

namespace onebit {

int fail(int status, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char *where);

}  // namespace onebit
