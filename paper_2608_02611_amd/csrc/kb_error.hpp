// kb_error.hpp -- the calling thread's error text (kb_api.hip): fail() stores
// the message and returns code, clear_error() empties it.
#pragma once

#include <hip/hip_runtime.h>

namespace kb {

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail_hip(hipError_t e, const char* what);
void clear_error();

}  // namespace kb
