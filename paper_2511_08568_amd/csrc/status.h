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

// The launches of one call of an entry without a handle, up to the first that fails.  Their own return values say so: the
// thread's last error may be another call's, which is neither reported as this call's nor taken from the caller.
struct Launches {
    hipStream_t stream;
    hipError_t error = hipSuccess;

    template <typename... P, typename... A>
    void operator()(void (*kernel)(P...), dim3 grid, unsigned block, const A &...args) {
        if (error == hipSuccess) error = enqueue(kernel, grid, block, static_cast<P>(args)...);
    }

    int32_t status() const {
        if (error == hipSuccess) return RECMG_OK;
        (void)hipGetLastError();  // reported here
        return fail(RECMG_E_HIP, std::string("kernel launch: ") + hipGetErrorString(error));
    }

private:
    template <typename... P> hipError_t enqueue(void (*kernel)(P...), dim3 grid, unsigned block, P... args) {
        void *at[] = {&args...};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(block), at, 0, stream);
    }
};

}  // namespace recmg
