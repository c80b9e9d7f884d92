// What the translation units of librcd share on the host: error reporting, workspace carving.
#pragma once
#include <hip/hip_runtime.h>
#include <cstddef>

#include "../../include/rcd.h"

// Notes the text of a failed HIP call for rcd_last_hip_error() of the calling thread; returns RCD_ERR_HIP.
__attribute__((visibility("hidden"))) int rcd_note_hip_error(const char *what, hipError_t e);

// The encoder's part of rcd_init(): what its kernels need once per device.
__attribute__((visibility("hidden"))) int rcd_set_up_encoder();

#define ENC_HIP_TRY(expr)                                            \
    do {                                                             \
        hipError_t e_ = (expr);                                      \
        if (e_ != hipSuccess) return rcd_note_hip_error(#expr, e_);  \
    } while (0)

#define ENC_TRY(expr)                  \
    do {                               \
        int rc_ = (expr);              \
        if (rc_ != RCD_OK) return rc_; \
    } while (0)
