// What the C ABI's source files share: the message of a thread's last
// failure, the guard around every entry point's body, argument checks.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <new>

#include "../../include/libmssa.h"

namespace mssa {

// Record the message that mssa_last_error() returns on this thread and pass
// the status on (defined in abi.cpp; never allocates, so it cannot throw).
mssa_status fail(mssa_status s, const char* msg) noexcept;
mssa_status fail(mssa_status s, const char* what, const char* detail) noexcept;

// Body of an entry point: no C++ exception leaves the library.  A failed
// host allocation is MSSA_ERR_NO_MEMORY, anything else MSSA_ERR_INVALID_ARG.
template <class Body>
mssa_status guarded(const char* where, Body&& body) noexcept {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(MSSA_ERR_NO_MEMORY, where, "host allocation failed");
  } catch (...) {
    return fail(MSSA_ERR_INVALID_ARG, where, "unexpected internal error");
  }
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline mssa_status check_device(hipError_t e, const char* what) {
  if (e == hipSuccess) return MSSA_OK;
  return fail(MSSA_ERR_DEVICE, what, hipGetErrorString(e));
}

}  // namespace mssa
