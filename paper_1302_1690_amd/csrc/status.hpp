// Statuses and the calling thread's message, shared by the host sides (defined in mpcnn.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/mpcnn.h"

namespace mpcnn {

// Notes the message that mpcnn_last_error returns and hands the status back
mpcnn_status fail(mpcnn_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace mpcnn

#define HIP_TRY(expr)                                                                             \
    do {                                                                                          \
        hipError_t e_ = (expr);                                                                   \
        if (e_ != hipSuccess)                                                                     \
            return mpcnn::fail(MPCNN_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), \
                               __FILE__, __LINE__);                                               \
    } while (0)
