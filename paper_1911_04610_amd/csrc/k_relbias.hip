// The learned relative position bias: a table of one value per bucket and head,
// spread over distances (key position - query position) for attention to read,
// and its gradient.
//
// A distance a >= 0 lies in one of n buckets: below n / 2 each has its own, beyond
// they grow with the logarithm, bucket n / 2 + floor(log(2 a / n) / log(2 far / n) (n - n / 2)),
// the last one from there on.  In fp64; a distance on a border belongs to the bucket that
// starts there: the quotient is raised by 2^-44 of itself, a few times what its logarithms and
// products round by, so one that lies below a border by less than that counts as on it (over all max distances up to
// 2^20: no distance with 8, 16, 32 or 64 buckets a direction, 3 with 128).
#include "xp_device.h"
#include "xp_kernels.h"

namespace xp {

namespace {

struct Buckets {
  int n, half;      // of one direction; those of single distances
  double scale;     // (n - half) / log(far / half)
  int both, far;
};

XP_DEV int bucket_of(const Buckets& b, int away) {
  if (away < b.half) return away;
  const int k = (int)(log((double)away / b.half) * b.scale * (1.0 + 0x1p-44));
  return min(b.n - 1, b.half + k);
}
XP_DEV int bucket_at(const Buckets& b, int d) {  // d: key position - query position
  if (!b.both) return bucket_of(b, max(-d, 0));
  return d > 0 ? b.n + bucket_of(b, d) : bucket_of(b, -d);
}

// A thread takes one distance and up to 16 heads: the logarithm costs more than the heads'
// values do.  Bound by that, and by the launch: 65537 distances, 64 heads 6.9 us (16.8 MB, 2.4 TB/s); 257, 12 2.8 us.
constexpr int HEADS_PER = 16;

__global__ __launch_bounds__(256) void k_relbias_fwd(const float* __restrict__ table, Buckets b, int heads, float* __restrict__ bias) {
  const int x = blockIdx.x * 256 + threadIdx.x, width = 2 * b.far + 1;
  if (x >= width) return;
  const float* row = table + (int64_t)bucket_at(b, x - b.far) * heads;
  const int h0 = blockIdx.y * HEADS_PER, h1 = min(heads, h0 + HEADS_PER);
  for (int h = h0; h < h1; ++h) bias[(int64_t)h * width + x] = row[h];
}

// The first distance 0 .. far in bucket k or a later one; far + 1 if none.  From the border
// itself, at most a few steps from what bucket_of says.
XP_DEV int first_of(const Buckets& b, int k) {
  if (k <= b.half) return k;
  if (k >= b.n) return b.far + 1;
  int d = max(b.half, min(b.far, (int)ceil(b.half * exp((k - b.half) / b.scale))));
  while (d > b.half && bucket_of(b, d - 1) >= k) --d;
  while (d <= b.far && bucket_of(b, d) < k) ++d;
  return d;
}

// this thread's part of the sum of n consecutive values
template <int THREADS>
XP_DEV double run_sum(const float* p, int n) {
  double s = 0.0;
  int i = threadIdx.x * 4;
#pragma unroll 4
  for (; i + 4 <= n; i += THREADS * 4) {
    float v[4];
    __builtin_memcpy(v, p + i, 16);
    s += ((double)v[0] + v[1]) + ((double)v[2] + v[3]);
  }
  for (; i < n; ++i) s += p[i];  // (one thread has such a rest)
  return s;
}

// One workgroup per bucket and 2 heads: the bucket's distances are one run of each head's row.
// Finding its ends costs as much as a short run, so one wave does it for all of them.
// THREADS: 1024 where runs are long.
// Bound by the order of the launch and the ends: the bucket of all keys behind the query holds half of a row, and of 2048
// workgroups of 1024 threads, 512 at a time, the last of that bucket starts in the fourth round; each finds its ends anew by
// logarithms and an exponential in fp64.  65537 distances, 64 heads, 64 buckets: 21 us, with the forward 27.3 (1 head a workgroup
// 31.5, 4 heads 29.7); 257 distances, 12 heads 5 us, with the forward 9.5 (9.7, 9.6), of which the ends are half.
constexpr int RUNS = 2;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_relbias_bwd(const float* __restrict__ dbias, Buckets b, int heads, float* __restrict__ grad) {
  __shared__ double sh[RUNS][THREADS / 64];
  __shared__ int ends[2];
  const int k = blockIdx.x, side = b.both && k >= b.n, kk = side ? k - b.n : k, h0 = blockIdx.y * RUNS;
  if (threadIdx.x < 64) {
    const int d = first_of(b, kk + (threadIdx.x & 1));  // the bucket's distances: [ends[0], ends[1])
    if (threadIdx.x < 2) ends[threadIdx.x] = d;
  }
  __syncthreads();
  const int lo = side ? max(ends[0], 1) : ends[0], hi = ends[1];
  // (keys behind the query count as distance 0 where there is one direction)
  const int first = side ? lo : 1 - hi, last = side ? hi : !b.both && kk == 0 ? b.far + 1 : 1 - lo;
  double s[RUNS];
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const float* row = dbias + (int64_t)min(h0 + i, heads - 1) * (2 * b.far + 1) + b.far;
    s[i] = run_sum<THREADS>(row + first, last - first);
  }
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    s[i] = wave_sum(s[i]);
    if ((threadIdx.x & 63) == 0) sh[i][threadIdx.x >> 6] = s[i];
  }
  __syncthreads();
  const int h = h0 + threadIdx.x;
  if (threadIdx.x < RUNS && h < heads) {
    float* g = grad + (int64_t)k * heads + h;
    double t = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) t += sh[threadIdx.x][w];
    *g = (float)((double)*g + t);
  }
}

Buckets describe(const RelBiasArgs& a) {
  Buckets b{};
  b.both = a.both;
  b.n = a.both ? a.buckets / 2 : a.buckets;
  b.half = b.n / 2;
  b.far = a.far;
  b.scale = (b.n - b.half) / log((double)a.far / b.half);
  return b;
}

}  // namespace

hipError_t launch_relbias_fwd(const RelBiasArgs& a, hipStream_t s) {
  const int width = 2 * a.far + 1;
  XP_LAUNCH("k_relbias_fwd", 4.0 * width * a.heads, k_relbias_fwd, dim3((width + 255) / 256, (a.heads + HEADS_PER - 1) / HEADS_PER),
            dim3(256), 0, s, a.table, describe(a), a.heads, a.bias);
  return hipGetLastError();
}

hipError_t launch_relbias_bwd(const RelBiasArgs& a, hipStream_t s) {
  const double bytes = 4.0 * (2 * a.far + 1) * a.heads;
  const dim3 grid(a.buckets, (a.heads + RUNS - 1) / RUNS);
  if (a.far > 4096) XP_LAUNCH("k_relbias_bwd", bytes, k_relbias_bwd<1024>, grid, dim3(1024), 0, s, a.dbias, describe(a), a.heads, a.grad);
  else XP_LAUNCH("k_relbias_bwd", bytes, k_relbias_bwd<256>, grid, dim3(256), 0, s, a.dbias, describe(a), a.heads, a.grad);
  return hipGetLastError();
}

}  // namespace xp
