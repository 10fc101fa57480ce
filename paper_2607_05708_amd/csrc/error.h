// The thread's last-error message behind mem_last_error, shared by the C
// entry points.
#pragma once

#include <hip/hip_runtime.h>

#include "memattn.h"

namespace memattn {

// Record the message of a failed call and return its status.
mem_status fail(mem_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// MEM_OK, or MEM_ERR_DEVICE with the HIP error's text.
mem_status device_status(hipError_t e, const char* what);

// Forget the last message (every call that can fail starts with this).
void clear_error();

}  // namespace memattn
