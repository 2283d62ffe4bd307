// Errors of the C entry points: a status and the calling thread's message.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "../../include/recmg.h"

namespace recmg {

// Keeps the message for recmg_last_error and returns the code.
int32_t fail(int32_t code, const std::string &msg);

#define HIP_TRY(expr)                                                                              \
    do {                                                                                           \
        hipError_t e_ = (expr);                                                                    \
        if (e_ != hipSuccess) return recmg::fail(RECMG_E_HIP, std::string(#expr) + ": " + hipGetErrorString(e_)); \
    } while (0)

// For entries without a handle: an error that some other call of the thread left is not reported as this call's.
inline void forget_errors() { (void)hipGetLastError(); }

}  // namespace recmg
