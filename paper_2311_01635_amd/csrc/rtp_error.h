// How the C entry points report errors: a status, and its text for rtp_last_error().
#pragma once
#include "../../include/rtp.h"

namespace rtp {
rtp_status fail(rtp_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
}

#define HIP_TRY(expr)                                                                                       \
    do {                                                                                                    \
        hipError_t e_ = (expr);                                                                             \
        if (e_ != hipSuccess) return rtp::fail(RTP_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_));        \
    } while (0)

#define RTP_TRY(expr)                       \
    do {                                    \
        rtp_status s_ = (expr);             \
        if (s_ != RTP_OK) return s_;        \
    } while (0)
