// What the files of C entry points share: the calling thread's error detail
// and the checks that come before any launch.
#pragma once
#include <hip/hip_runtime.h>

#define SAGE_API extern "C" __attribute__((visibility("default")))

namespace sage {

// Sets the calling thread's error detail; returns `status`.
int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears it; returns SAGE_OK.
int ok();
bool aligned16(const void* p);
// SAGE_OK when the current device is a gfx950 (cached per device ordinal).
int check_device();
// A launch's status as the entry point's return value.
int hip_status(hipError_t e, const char* what);

}  // namespace sage
