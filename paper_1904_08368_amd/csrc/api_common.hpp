// What the files of the C-ABI layer share: the status with its message for relay_last_error(), and the checks of pointers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/relay_fused.h"

namespace relay {

// leaves the message for the calling thread and returns st
relay_status fail(relay_status st, const char* fmt, ...);

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline relay_status device_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return RELAY_OK;
  return fail(RELAY_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace relay
