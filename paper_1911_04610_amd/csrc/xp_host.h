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

#define XP_TRY(call)                        \
  do {                                      \
    xpipe_status r_ = (call);               \
    if (r_ != XPIPE_OK) return r_;          \
  } while (0)

inline bool known_dtype(int32_t d) { return d == XPIPE_F32 || d == XPIPE_BF16; }
inline int esize(int32_t dtype) { return dtype == XPIPE_BF16 ? 2 : 4; }

inline bool at_multiple(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

inline xpipe_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return XPIPE_OK;
  if (!ws) return fail(XPIPE_EINVAL, "null workspace");
  if (bytes < need) return fail(XPIPE_EINVAL, "workspace too small");
  if (!at_multiple(ws, 256)) return fail(XPIPE_EINVAL, "workspace must be 256-byte aligned");
  return XPIPE_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// xpipe_grad_norm's launches, for checked arguments; part: its workspace, of `blocks`
// doubles (0: one launch and no workspace)
hipError_t grad_norm(const xpipe_tensor* tensors, int32_t n, int32_t dtype, double max_norm, double* sumsq, float* norm_coef,
                     double* part, int64_t blocks, hipStream_t s);

}  // namespace xp
