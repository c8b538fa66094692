// What the library's sources share on the host: the text of a thread's last HIP error, and the two ways an error leaves a call.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdio>

#include "../../include/knnssd.h"

extern thread_local char g_hip_err[256];

#define HIP_TRY(expr)                                                                              \
    do {                                                                                           \
        hipError_t e_ = (expr);                                                                    \
        if (e_ != hipSuccess) {                                                                    \
            snprintf(g_hip_err, sizeof(g_hip_err), "%s at %s:%d", hipGetErrorString(e_), __FILE__, __LINE__); \
            return KNNSSD_EHIP;                                                                    \
        }                                                                                          \
    } while (0)

#define KS_TRY(expr)                    \
    do {                                \
        int32_t rc_ = (expr);           \
        if (rc_ != KNNSSD_OK) return rc_; \
    } while (0)
