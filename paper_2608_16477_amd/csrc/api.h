// What the files of the C ABI share: the thread's error message and the checks of
// a pool.
#pragma once

#include <hip/hip_runtime.h>

#include "pallas.h"

namespace pallas {

// Sets the calling thread's message (pallas_last_error) and returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* where);
int check_pool(const pallas_kv_pool* p, const char* what);

}  // namespace pallas
