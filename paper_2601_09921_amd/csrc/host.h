// What the library's host sources share: the calling thread's error message.
#pragma once
#include <hip/hip_runtime.h>

// Sets the message of decoder_last_error and returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((visibility("hidden"), format(printf, 2, 3)));

#define HIP_OK(call)                                                                     \
    do {                                                                                 \
        hipError_t e_ = (call);                                                          \
        if (e_ != hipSuccess)                                                            \
            return fail(PWD_EHIP, "%s failed: %s", #call, hipGetErrorString(e_));        \
    } while (0)
