// The status and error detail that every C entry returns through.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

#include "oaa.h"

namespace oaa {

// Alignment of caller-owned workspaces.
constexpr size_t kWorkspaceAlign = 256;

// Record the thread's error detail (oaa_last_error_detail) and return st.
oaa_status_t fail(oaa_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// OAA_OK, or OAA_ERR_HIP with `what` and the runtime's message.
oaa_status_t hip_status(hipError_t e, const char* what);

}  // namespace oaa
