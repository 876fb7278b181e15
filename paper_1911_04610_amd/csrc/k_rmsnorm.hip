// Root-mean-square norm of a token network's rows with the skip connection's
// addition in front, and its gradients.
//
//   forward:  h = x + residual;  n = 1 / sqrt(mean(h^2) + eps);  y = h n w
//   backward: g = dy w;  dx = n (g - h n^2 mean(g h)) + residual;  grad_w += sum over rows of dy h n
//
// Bandwidth-bound: a row is read once and held in the registers of the G threads
// that share it (E elements each), the sums go over those threads, in fp64 (squares of
// fp32 values neither overflow nor lose bits there; in bf16 storage a thread's own elements are
// summed in fp32 where that holds them); the rest is fp32, each stored value is rounded once.
#include "xp_device.h"
#include "xp_lds.h"
#include "xp_kernels.h"

#include <algorithm>

namespace xp {

namespace {

template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);

// n elements (more than CHUNK: a whole chunk) from p on, which may start anywhere; zeros behind them
template <typename T>
XP_DEV u32x4_t ld_raw(const T* p, int n) {
  u32x4_t u = {0, 0, 0, 0};
  if (n >= CHUNK<T>) {
    __builtin_memcpy(&u, p, 16);
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < CHUNK<T>; ++i) {
      uint32_t e = 0;
      if (i < n) {
        if constexpr (sizeof(T) == 4) e = __float_as_uint(p[i]);
        else e = p[i];
      }
      if constexpr (sizeof(T) == 4) w[i] = e;
      else w[i / 2] |= e << (16 * (i & 1));
    }
    u = (u32x4_t){w[0], w[1], w[2], w[3]};
  }
  return u;
}
template <typename T>
XP_DEV void unpack(const u32x4_t& u, float* v) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(u[i]);
    else v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  }
}
template <typename T>
XP_DEV void ld_elems(const T* p, int n, float* v) { unpack<T>(ld_raw(p, n), v); }
template <typename T>
XP_DEV void st_elems(T* p, int n, const float* v) {
  if (n >= CHUNK<T>) {
    u32x4_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(v[i]);
      else u[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
    }
    __builtin_memcpy(p, &u, 16);
  } else {
#pragma unroll
    for (int i = 0; i < CHUNK<T>; ++i)
      if (i < n) std_(p + i, (double)v[i]);
  }
}

// Threads of a workgroup, and the rows that they hold at a time.
template <int G> constexpr int THREADS = G < 256 ? 256 : G;
template <int G> constexpr int ROWS = THREADS<G> / G;

// Sums of N values over a row's G threads, in all of them.  sh: two sets of N x 16
// doubles, used in turn (so that one barrier a row is enough).
template <int G, int N>
XP_DEV void row_sums(double (&v)[N], double (*sh)[16], int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int off = (G < 64 ? G : 64) / 2; off > 0; off >>= 1) v[i] += __shfl_xor(v[i], off, 64);
  if constexpr (G > 64) {
    double(*s)[16] = sh + turn * N;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i][threadIdx.x >> 6] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0;
      for (int w = 0; w < G / 64; ++w) v[i] += s[i][w];
    }
  }
}

// A thread's part of a row's sums.  In bf16 storage over E elements in fp32 (an fp64 sum takes
// longer than the row's bytes do: 16384x4096 backward 118 us with it, 87 without); a row whose sums leave the
// range where that is exact to fp32 is summed again in fp64.  The squares: with a sum between these none has
// overflowed, and what underflows is below 2^-60 of it.  The products: one that overflowed leaves the row's sum infinite or
// NaN, and 2^15 that lost 2^-149 each are below 2^-34 of a sum beyond 1e-30 (a row without a gradient is summed twice).
XP_DEV bool in_range(double squares) { return squares > 1e-20 && squares < 1e36; }
XP_DEV bool held(double products) { return fabs(products) > 1e-30 && fabs(products) < 1e300; }
template <typename T, int E>
XP_DEV void squares(const float (&h)[E], double& out) {
  if constexpr (sizeof(T) == 4) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i) s += (double)h[i] * h[i];
    out = s;
  } else {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[i & 3] += h[i] * h[i];
    out = (double)((s[0] + s[1]) + (s[2] + s[3]));
  }
}
template <typename T, int E>
XP_DEV void products(const float (&h)[E], const float (&dy)[E], const float (&w)[E], double& out) {
  if constexpr (sizeof(T) == 4) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i) s += (double)(dy[i] * w[i]) * h[i];
    out = s;
  } else {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[i & 3] += dy[i] * w[i] * h[i];
    out = (double)((s[0] + s[1]) + (s[2] + s[3]));
  }
}
template <int E>
XP_DEV void wide_sums(const float (&h)[E], const float (&dy)[E], const float (&w)[E], double (&s)[2]) {
  squares<float, E>(h, s[0]);
  products<float, E>(h, dy, w, s[1]);
}

// 16384x4096 bf16 with residual and sum: 97 us, 5.6 TB/s, of what a copy reaches (5.2 torch's, 6.2 the library's
// probe); 8192x4096 fp32 92 us, 5.8 TB/s; one row: 3 us, a launch.
// No __restrict__: sum and y may be x's or residual's buffer (every element is read
// by the thread that writes it, before).
template <typename T, int G, int E>
__global__ __launch_bounds__(THREADS<G>) void k_rms_fwd(RmsArgs a) {
  constexpr int C = CHUNK<T>, V = E / C;
  __shared__ double sh[2][16];
  const int lt = threadIdx.x % G;
  float w[E];
#pragma unroll
  for (int j = 0; j < V; ++j) ld_elems(a.w + (lt + j * G) * C, min(4, a.dim - (lt + j * G) * C), w + j * C);
  if constexpr (C == 8)
#pragma unroll
    for (int j = 0; j < V; ++j) ld_elems(a.w + (lt + j * G) * C + 4, min(4, a.dim - (lt + j * G) * C - 4), w + j * C + 4);
  int turn = 0;
  // (workgroup-uniform where the sums need a barrier: ROWS is 1 there)
  for (int64_t row = (int64_t)blockIdx.x * ROWS<G> + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.x * ROWS<G>) {
    float h[E];
    double ss[1] = {0.0};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = (lt + j * G) * C;
      ld_elems((const T*)a.x + row * a.ldx + at, a.dim - at, h + j * C);
    }
    if (a.res) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int at = (lt + j * G) * C;
        float r[C];
        ld_elems((const T*)a.res + row * a.ldr + at, a.dim - at, r);
#pragma unroll
        for (int i = 0; i < C; ++i) h[j * C + i] += r[i];
      }
    }
    squares<T, E>(h, ss[0]);
    row_sums<G, 1>(ss, sh, turn);
    turn ^= 1;
    if (sizeof(T) == 2 && !in_range(ss[0])) {  // (the row's threads agree)
      squares<float, E>(h, ss[0]);
      row_sums<G, 1>(ss, sh, turn);
      turn ^= 1;
    }
    const float n = (float)(1.0 / sqrt(ss[0] / a.dim + a.eps));
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = (lt + j * G) * C;
      if (a.out) st_elems((T*)a.out + row * a.ldo + at, a.dim - at, h + j * C);
      float y[C];
#pragma unroll
      for (int i = 0; i < C; ++i) y[i] = h[j * C + i] * n * w[j * C + i];
      st_elems((T*)a.y + row * a.ldy + at, a.dim - at, y);
    }
  }
}

// One workgroup's rows: their dx, and its part of grad_w: the sum of its rows' terms in
// fp32 (MOST_TERMS of them a thread at most: more rows are another launch), over the ROWS rows at a time in LDS.  The parts
// are added in fp64 by k_rms_join; a single workgroup adds its own.  The next row's
// h and dy are on their way while this one's sums are joined.
// Bound by the bytes of large calls (16384x4096 bf16: 84 us with the join, 4.8 TB/s for h, dy and dx; 262144x4096
// 1230 us, 5.2 TB/s) and by the two launches of small ones: 1001x999 fp32 6.5 us and 5.  The skip's gradient is
// read behind the next row's h and dy, not ahead, and its wait is a wait for them: 8192x2048 with it 36 us (134 MB, 3.7 TB/s).
template <typename T, int G, int E>
__global__ __launch_bounds__(THREADS<G>) void k_rms_bwd(RmsArgs a) {
  constexpr int C = CHUNK<T>, V = E / C;
  __shared__ double sh[4][16];
  __shared__ float gsum[ROWS<G> > 1 ? G * E * ROWS<G> : 1];
  const int lt = threadIdx.x % G;
  float acc[E], w[E];
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int p = 0; p < C; p += 4) ld_elems(a.w + (lt + j * G) * C + p, min(4, a.dim - (lt + j * G) * C - p), w + j * C + p);
  u32x4_t hr[V], dr[V];
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = (lt + j * G) * C;
      hr[j] = ld_raw((const T*)a.x + row * a.ldx + at, a.dim - at);
      dr[j] = ld_raw((const T*)a.dy + row * a.lddy + at, a.dim - at);
    }
  };
  int turn = 0;
  const int64_t step = (int64_t)gridDim.x * ROWS<G>;
  int64_t row = (int64_t)blockIdx.x * ROWS<G> + threadIdx.x / G;
  if (row < a.rows) fetch(row);
  for (; row < a.rows; row += step) {
    float h[E], dy[E];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      unpack<T>(hr[j], h + j * C);
      unpack<T>(dr[j], dy + j * C);
    }
    if (row + step < a.rows) fetch(row + step);
    double s[2];
    squares<T, E>(h, s[0]);
    products<T, E>(h, dy, w, s[1]);
    row_sums<G, 2>(s, sh, turn);
    turn ^= 1;
    if (sizeof(T) == 2 && !(in_range(s[0]) && held(s[1]))) {  // (the row's threads agree)
      wide_sums<E>(h, dy, w, s);
      row_sums<G, 2>(s, sh, turn);
      turn ^= 1;
    }
    const double nd = 1.0 / sqrt(s[0] / a.dim + a.eps);
    const float n = (float)nd, c = (float)(nd * nd * s[1] / a.dim);
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += dy[i] * (h[i] * n);
    if (a.y) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int at = (lt + j * G) * C;
        float r[C], dx[C];
        if (a.res) ld_elems((const T*)a.res + row * a.ldr + at, a.dim - at, r);
#pragma unroll
        for (int i = 0; i < C; ++i) {
          dx[i] = n * (dy[j * C + i] * w[j * C + i] - h[j * C + i] * c);
          if (a.res) dx[i] += r[i];
        }
        st_elems((T*)a.y + row * a.ldy + at, a.dim - at, dx);
      }
    }
  }
  if (!a.grad) return;
  if constexpr (ROWS<G> > 1) {
    const int grp = threadIdx.x / G;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < C; ++i) gsum[grp * (G * E) + (lt + j * G) * C + i] = acc[j * C + i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += THREADS<G>) {
      float t = 0.f;
      for (int r = 0; r < ROWS<G>; ++r) t += gsum[r * (G * E) + c];
      if (gridDim.x == 1) a.grad[c] += t;
      else a.part[(int64_t)blockIdx.x * a.dim + c] = t;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int c = (lt + j * G) * C + i;
        if (c < a.dim) {
          if (gridDim.x == 1) a.grad[c] += acc[j * C + i];
          else a.part[(int64_t)blockIdx.x * a.dim + c] = acc[j * C + i];
        }
      }
  }
}

// grad[c] += sum of n parts, 16 columns and 16 runs of parts a workgroup
__global__ __launch_bounds__(256) void k_rms_join(const float* __restrict__ part, int64_t n, int dim, float* __restrict__ grad) {
  __shared__ double sh[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;
  double s = 0.0;
  if (col < dim) {
#pragma unroll 8
    for (int64_t i = r; i < n; i += 16) s += (double)part[i * dim + col];
  }
  sh[r][c] = s;
  __syncthreads();
  if (r == 0 && col < dim) {
    s = 0.0;
    for (int i = 0; i < 16; ++i) s += sh[i][c];
    grad[col] = (float)((double)grad[col] + s);
  }
}

// calls f(threads a row, elements a thread) for rows of dim elements: a wave a row where it holds
// it (8192x2048 backward 30.5 us; 256 threads of 8 elements each 34.8)
template <typename F>
void by_size(int dim, F&& f) {
  using std::integral_constant;
  if (dim <= 64) f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else if (dim <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  else if (dim <= 256) f(integral_constant<int, 32>{}, integral_constant<int, 8>{});
  else if (dim <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else if (dim <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
  else if (dim <= 2048) f(integral_constant<int, 64>{}, integral_constant<int, 32>{});
  else if (dim <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 16>{});
  else if (dim <= 8192) f(integral_constant<int, 256>{}, integral_constant<int, 32>{});
  else if (dim <= 16384) f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 32>{});
}

// Two workgroups a CU (8192x2048 with the skip's gradient 47.2 us, 4096x8192 91.9, 16384x4096 119; three: 50.0,
// 99.3, 110; four: 53.9, 107, 132).
template <int G>
int bwd_blocks(int64_t rows) { return (int)std::min<int64_t>((rows + ROWS<G> - 1) / ROWS<G>, G >= 1024 ? 256 : 512); }
// Rows of a launch, and the parts of grad_w that all launches leave.
constexpr int MOST_TERMS = 256;
template <int G>
constexpr int64_t LAUNCH_ROWS = (int64_t)(G >= 1024 ? 256 : 512) * ROWS<G> * MOST_TERMS;
template <int G>
int64_t bwd_parts(int64_t rows) {
  const int last = bwd_blocks<G>(rows % LAUNCH_ROWS<G>);  // (a single workgroup adds its own)
  return rows / LAUNCH_ROWS<G> * bwd_blocks<G>(LAUNCH_ROWS<G>) + (last > 1 ? last : 0);
}

template <typename T>
hipError_t fwd(const RmsArgs& a, hipStream_t s) {
  by_size(a.dim, [&](auto G, auto E) {
    constexpr int g = decltype(G)::value, e = decltype(E)::value;
    constexpr int64_t most = g <= 64 && e == 8 ? 2048 : ((int64_t)1 << 31) / THREADS<g>;  // (a launch has less than 2^32 threads)
    const int blocks = (int)std::min<int64_t>((a.rows + ROWS<g> - 1) / ROWS<g>, most);
    const double bytes = (double)sizeof(T) * a.rows * a.dim * (2 + (a.res != nullptr) + (a.out != nullptr));
    XP_LAUNCH(sizeof(T) == 2 ? "k_rms_fwd<bf16>" : "k_rms_fwd<f32>", bytes, (k_rms_fwd<T, g, e>), dim3(blocks),
              dim3(THREADS<g>), 0, s, a);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(RmsArgs a, void* workspace, hipStream_t s) {
  const auto from = [](const void* p, int64_t row, int64_t ld) { return p ? (char*)p + row * ld * (int64_t)sizeof(T) : nullptr; };
  by_size(a.dim, [&](auto G, auto E) {
    constexpr int g = decltype(G)::value, e = decltype(E)::value;
    int64_t parts = 0;
    for (int64_t row = 0; row < a.rows; row += LAUNCH_ROWS<g>) {
      RmsArgs b = a;
      b.rows = std::min(a.rows - row, LAUNCH_ROWS<g>);
      b.dy = from(a.dy, row, a.lddy);
      b.x = from(a.x, row, a.ldx);
      b.res = from(a.res, row, a.ldr);
      b.y = from(a.y, row, a.ldy);
      b.part = a.grad ? (float*)workspace + parts * a.dim : nullptr;
      const int blocks = bwd_blocks<g>(b.rows);
      const double bytes = (double)sizeof(T) * b.rows * a.dim * (2 + (a.y != nullptr) + (a.res != nullptr));
      XP_LAUNCH(sizeof(T) == 2 ? "k_rms_bwd<bf16>" : "k_rms_bwd<f32>", bytes, (k_rms_bwd<T, g, e>), dim3(blocks),
                dim3(THREADS<g>), 0, s, b);
      if (blocks > 1) parts += blocks;
    }
    if (a.grad && parts > 0)
      XP_LAUNCH("k_rms_join", 4.0 * parts * a.dim, k_rms_join, dim3((a.dim + 15) / 16), dim3(256), 0, s, (const float*)workspace, parts, a.dim, a.grad);
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_fwd(int dtype, const RmsArgs& a, hipStream_t s) {
  return dtype == DT_BF16 ? fwd<bf16_t>(a, s) : fwd<float>(a, s);
}

size_t rms_bwd_bytes(int64_t rows, int dim) {
  size_t n = 0;
  by_size(dim, [&](auto G, auto) { n = (size_t)bwd_parts<decltype(G)::value>(rows) * dim * sizeof(float); });
  return n;
}

hipError_t launch_rms_bwd(int dtype, const RmsArgs& a, void* workspace, hipStream_t s) {
  return dtype == DT_BF16 ? bwd<bf16_t>(a, workspace, s) : bwd<float>(a, workspace, s);
}

}  // namespace xp
