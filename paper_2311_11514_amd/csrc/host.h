// What the host files of the library share: how a HIP call's failure becomes a status.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/hexgen.h"

#define HX_HIP(expr)                                                          \
    do {                                                                      \
        hipError_t e_ = (expr);                                               \
        if (e_ != hipSuccess) {                                               \
            (void)hipGetLastError();                                          \
            return e_ == hipErrorOutOfMemory ? HEXGEN_ERR_OOM : HEXGEN_ERR_DEVICE; \
        }                                                                     \
    } while (0)
#define HX_TRY(expr)                              \
    do {                                          \
        hexgen_status_t s_ = (expr);              \
        if (s_ != HEXGEN_OK) return s_;           \
    } while (0)
