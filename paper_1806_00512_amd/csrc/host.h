// What the host files of the library share (defined in lstmss_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lstmss {

// Sets the calling thread's detail message and returns `code`.
int32_t api_fail(int32_t code, const char *text);

// Runs launch(arg), between two events of `kind` on `s` while the timing
// hooks are on.
hipError_t api_timed(int kind, hipStream_t s, hipError_t (*launch)(const void *), const void *arg);

} // namespace lstmss
