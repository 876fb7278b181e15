// Host-side helpers shared by the C ABI's sources.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "../../include/xpipe.h"
#include "xp_kernels.h"

namespace xp {

// records the message of xpipe_last_error() for the calling thread and returns s
xpipe_status fail(xpipe_status s, const std::string& msg);

#define XP_HIP(call)                                                                     \
  do {                                                                                   \
    hipError_t e_ = (call);                                                              \
    if (e_ != hipSuccess)                                                                \
      return fail(XPIPE_EHIP, std::string(#call) + ": " + hipGetErrorString(e_));        \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// xpipe_grad_norm's launches, for checked arguments; part: its workspace, of `blocks`
// doubles (0: one launch and no workspace)
hipError_t grad_norm(const xpipe_tensor* tensors, int32_t n, int32_t dtype, double max_norm, double* sumsq, float* norm_coef,
                     double* part, int64_t blocks, hipStream_t s);

}  // namespace xp
