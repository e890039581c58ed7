// What the host sources share: the calling thread's last error, HIP error checks, buffer alignment.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace ham {

// sets the calling thread's ham_last_error message; returns `code`
int fail(int code, const char* fmt, ...);

inline size_t al(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace ham

#define HIP_TRY(call)                                                                        \
  do {                                                                                       \
    hipError_t e_ = (call);                                                                  \
    if (e_ != hipSuccess) return ham::fail(HAM_EHIP, "%s: %s", #call, hipGetErrorString(e_)); \
  } while (0)
