// ea_host.hpp -- error state and argument checks shared by the files of the C
// ABI (defined in ea_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ea.h"

namespace ea {

// Records the calling thread's error text and returns `code`.
__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...);
// Clears it and returns EA_OK.
int ok();
// ok(), or EA_ERR_HIP with the runtime's description.
int hip_status(hipError_t e, const char* what);
// The argument checks of a schedule and of a step index.
int check_schedule(const ea_schedule_t* s);
int check_t(int64_t t);

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

}  // namespace ea
