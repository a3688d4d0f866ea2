// The error message and status of a C-ABI call, shared by the host sources.
#pragma once

#include <hip/hip_runtime_api.h>

#include "digest.h"

namespace digest {

// Keeps the message for digest_last_error() on this thread; returns st.
digest_status fail(digest_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
digest_status hip_check(hipError_t e, const char *what);

}  // namespace digest
