// ea_check.hpp -- error texts and argument checks that the entry points beside
// the round share (ea_train_api.cpp, ea_layer_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>

#include "ea_train.h"

namespace {

// Errors share the round's text: ea_last_error() gives the calling thread's
// buffer (512 bytes, not const where it is defined), of which these calls write
// the first half at most.
constexpr size_t kErrorBytes = 256;

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(const_cast<char*>(ea_last_error()), kErrorBytes, fmt, ap);
    va_end(ap);
    return code;
}

int hip_status(hipError_t e, const char* what)
{
    if (e != hipSuccess) return fail(EA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    const_cast<char*>(ea_last_error())[0] = '\0';
    return EA_OK;
}

struct PtrCheck {
    int rc = EA_OK;
    void need(const void* ptr, bool required, uintptr_t align, const char* name)
    {
        if (rc) return;
        if (!ptr) {
            if (required) rc = fail(EA_ERR_ARG, "%s is NULL", name);
            return;
        }
        if ((uintptr_t)ptr % align) rc = fail(EA_ERR_ALIGN, "%s is not %u-byte aligned", name, (unsigned)align);
    }
};

bool known_type(int32_t type)
{
    return type == EA_F32 || type == EA_BF16 || type == EA_F16;
}

uintptr_t type_bytes(int32_t type)
{
    return type == EA_F32 ? 4 : 2;
}

}  // namespace
