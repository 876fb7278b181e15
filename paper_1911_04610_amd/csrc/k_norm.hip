// The global norm of gradients over many tensors and the clipping coefficient.
//
// Bandwidth-bound: every element is read once (16-byte loads where a tensor
// allows), squared and summed in fp64 (the squares of fp32 values neither
// overflow nor lose bits there), in an order that only the sizes and alignments
// decide.  1e8 fp32 elements 67 us, 6.0 TB/s, and 5 us for the second launch, which
// adds the workgroups' sums.
#include "xp_device.h"
#include "xp_lds.h"
#include "xp_kernels.h"

#include <algorithm>

namespace xp {

namespace {

constexpr int NORM_BLOCK = 256;
// elements per workgroup: 64 KB of fp32
constexpr int NORM_PER = 16384;

template <typename T>
XP_DEV double square_sum(const u32x4_t& u) {
  double s = 0.0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 4) {
      const double v = (double)__uint_as_float(u[q]);
      s += v * v;
    } else {
      const double lo = (double)__uint_as_float(u[q] << 16), hi = (double)__uint_as_float(u[q] & 0xffff0000u);
      s += lo * lo + hi * hi;
    }
  }
  return s;
}

// sum over the workgroup, in all lanes of the first wave
XP_DEV double block_sum(double s, double* sh) {
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) t += sh[w];
  return t;
}

// the tensor that unit u of the launch lies in: the last whose first unit is not behind it
XP_DEV int tensor_of(const NormArgs& a, int u) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.first[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// this thread's part (tid of threads) of the sum of squares of PER elements of a tensor, the unit-th ones
template <typename T, int PER, int THREADS>
XP_DEV double unit_sum(const NormArgs& a, int tensor, int unit, int tid) {
  constexpr int C = 16 / (int)sizeof(T);
  const int64_t beg = (int64_t)unit * PER, end = min(a.n[tensor], beg + PER);
  const T* p = (const T*)a.p[tensor] + beg;
  const int cnt = (int)(end - beg);
  // elements before the first multiple of 16 bytes
  const int head = min(cnt, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
  const int vecs = (cnt - head) / C;
  const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + head);
  double s = 0.0;
#pragma unroll 8
  for (int i = tid; i < vecs; i += THREADS) s += square_sum<T>(q[i]);
  if (tid < head) {
    const double v = ldd(p + tid);
    s += v * v;
  }
  const int rest = head + vecs * C + tid;
  if (rest < cnt) {
    const double v = ldd(p + rest);
    s += v * v;
  }
  return s;
}

template <typename T>
__global__ __launch_bounds__(NORM_BLOCK) void k_grad_sumsq(NormArgs a) {
  __shared__ double sh[NORM_BLOCK / 64];
  const int t = tensor_of(a, blockIdx.x);
  const double s = block_sum(unit_sum<T, NORM_PER, NORM_BLOCK>(a, t, blockIdx.x - a.first[t], threadIdx.x), sh);
  if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

// {norm, min(1, max_norm / (norm + 1e-6))} from the sum of squares
XP_DEV void write_norm(double s, double max_norm, double* sumsq, float* out) {
  if (sumsq) *sumsq = s;
  if (!out) return;
  const double norm = sqrt(s), c = max_norm / (norm + 1e-6);
  out[0] = (float)norm;
  out[1] = (float)(c < 1.0 || c != c ? c : 1.0);  // NaN stays
}

__global__ __launch_bounds__(1024) void k_clip_coef(const double* __restrict__ part, int64_t n, double max_norm,
                                                     double* __restrict__ sumsq, float* __restrict__ out) {
  __shared__ double sh[16];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_sum(s, sh);
  if (threadIdx.x == 0) write_norm(s, max_norm, sumsq, out);
}

// All of it in one workgroup, for up to NORM_SMALL_UNITS units of NORM_SMALL_PER
// elements, two for each of its waves: a small model's call is two launches' latency otherwise.
template <typename T>
__global__ __launch_bounds__(1024) void k_grad_norm_small(NormArgs a, int units, double max_norm, double* __restrict__ sumsq,
                                                           float* __restrict__ out) {
  __shared__ double sh[16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  double s = 0.0;
  for (int u = wave; u < units; u += 16) {
    const int t = tensor_of(a, u);
    s += unit_sum<T, NORM_SMALL_PER, 64>(a, t, u - a.first[t], lane);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) write_norm(s, max_norm, sumsq, out);
}

}  // namespace

int64_t norm_blocks(int64_t n) { return (n + NORM_PER - 1) / NORM_PER; }

hipError_t launch_grad_norm_small(int dtype, const NormArgs& a, int units, double max_norm, double* sumsq, float* out,
                                  hipStream_t s) {
  const double bytes = (double)units * NORM_SMALL_PER * (dtype == DT_BF16 ? 2 : 4);
  if (dtype == DT_BF16)
    XP_LAUNCH("k_grad_norm_small<bf16>", bytes, k_grad_norm_small<bf16_t>, dim3(1), dim3(1024), 0, s, a, units, max_norm, sumsq, out);
  else
    XP_LAUNCH("k_grad_norm_small<f32>", bytes, k_grad_norm_small<float>, dim3(1), dim3(1024), 0, s, a, units, max_norm, sumsq, out);
  return hipGetLastError();
}

hipError_t launch_grad_sumsq(int dtype, const NormArgs& a, int blocks, hipStream_t s) {
  if (blocks <= 0) return hipSuccess;
  const double bytes = (double)blocks * NORM_PER * (dtype == DT_BF16 ? 2 : 4);
  if (dtype == DT_BF16) XP_LAUNCH("k_grad_sumsq<bf16>", bytes, k_grad_sumsq<bf16_t>, dim3(blocks), dim3(NORM_BLOCK), 0, s, a);
  else XP_LAUNCH("k_grad_sumsq<f32>", bytes, k_grad_sumsq<float>, dim3(blocks), dim3(NORM_BLOCK), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_clip_coef(const double* part, int64_t n, double max_norm, double* sumsq, float* out, hipStream_t s) {
  XP_LAUNCH("k_clip_coef", 8.0 * n, k_clip_coef, dim3(1), dim3(1024), 0, s, part, n, max_norm, sumsq, out);
  return hipGetLastError();
}

}  // namespace xp
