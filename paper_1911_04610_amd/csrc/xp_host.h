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

// the two launches of xpipe_grad_norm over one fp32 tensor (part: norm_blocks(n) doubles)
hipError_t grad_norm_flat(const float* g, int64_t n, double max_norm, double* part, float* norm_coef, hipStream_t s);

}  // namespace xp
