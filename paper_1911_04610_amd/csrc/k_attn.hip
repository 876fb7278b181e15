// Attention of a token network and its gradients.  For a query i of head h and the
// keys j that its masks leave:
//
//   x_ij = scale q_i . k_j;  s_ij = cap tanh(x_ij / cap) (or x_ij) + bias[h][clamp(j - pos_i)]
//   m_i = max_j s_ij;  l_i = sum_j exp(s_ij - m_i);  P_ij = exp(s_ij - m_i) / l_i;  o_i = sum_j P_ij v_j
//   dP_ij = do_i . v_j;  dS_ij = P_ij (dP_ij - do_i . o_i);  dX_ij = dS_ij (1 - tanh^2) scale
//   dv_j = sum_i P_ij do_i;  dq_i = sum_j dX_ij k_j;  dk_j = sum_i dX_ij q_i;  dbias = sums of dS along diagonals
//
// One pass over the keys with the running maximum and sum; scores never leave the
// registers.  The products are arranged so that a lane holds one query (forward, dq) or
// one key (dk, dv) and 16 of the other: the matrix unit's result of "rows in LDS times
// columns in registers" then is, without a move, the register operand of the product
// with those rows (their order within a block of 16 is permuted in both operands), and
// whatever belongs to a query (maximum, sum, limits) is one value a lane.
//
// In bf16 storage P and dX are rounded to bf16 for the second products, as every operand of
// a bf16 product is; scores, sums and statistics are fp32 throughout.
#include "xp_device.h"
#include "xp_lds.h"
#include "xp_kernels.h"

#include <algorithm>
#include <climits>

namespace xp {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float NEG_INF = -__builtin_inff();
constexpr int ROWS = 128;  // query rows (dk, dv: keys) of a workgroup: 4 waves of 32
constexpr int QT = 32;     // queries of a step of k_attn_dkv

template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);
// keys of a step of the forward, and of k_attn_dq
template <typename T> constexpr int BN = sizeof(T) == 2 ? 64 : 32;
template <typename T, int DP> constexpr int BN_DQ = sizeof(T) == 2 && DP == 64 ? 64 : 32;
// waves of a SIMD that a kernel's registers leave room for: 512 of them a lane, one wave
// where both operands' columns and the results need more than 256
template <typename T, int DP> constexpr int WAVES = sizeof(T) == 4 && DP == 128 ? 1 : 2;

// ---------------------------------------------------------------- tiles in LDS
// Rows of DP elements, chunk c of row r at position c ^ swz(r).  Read along rows, 16
// bytes of 16 rows at a time, and down columns (bf16: the transposing read, 4 rows of 16
// columns for every 16 lanes; fp32: 32 columns of two rows four apart): the swizzle gives
// 16 rows different places, and four neighbouring rows different groups of four chunks.
template <typename T, int DP>
XP_DEV int swz(int r) {
  if constexpr (sizeof(T) == 4) return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
  else if constexpr (DP == 128) return (r & 3) << 2 | ((r >> 2) & 3);
  else return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

template <typename T, int DP> constexpr int ROW = DP * (int)sizeof(T);  // bytes
// Tiles are named by their byte address in LDS, a multiple of ROW: where a lane's reads differ in
// the chunk, they then differ by an exclusive or of a constant, and where they differ in the
// row, by an offset in the instruction.
template <typename V>
XP_DEV __attribute__((address_space(3))) V* lds(uint32_t at) {
  return (__attribute__((address_space(3))) V*)at;
}
template <typename V>
XP_DEV uint32_t lds_address(V* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)p;
}

// The same value, of which the compiler knows nothing: what is computed from it is computed
// where it stands.  (Every lane's place in every tile would otherwise be computed ahead of the
// loops and kept in registers that the operands need.)
XP_DEV int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// n of a chunk's elements (more: all) from p on, which may start anywhere; zeros behind them
template <typename T>
XP_DEV u32x4_t ld_chunk(const T* p, int n) {
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
XP_DEV void widen(const u32x4_t& u, float (&v)[CHUNK<T>]) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(u[i]);
    else v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  }
}

// N rows of DP elements on their way from memory to LDS: loaded a step ahead into
// registers, stored when the step before is done.  Rows are 16-byte aligned, of `dim`
// elements in whole chunks; a chunk that is not to be read has an offset past the buffer's
// end, which loads zeros.
template <typename T, int DP, int N>
struct Stager {
  static constexpr int CPR = DP / CHUNK<T>, STEP = 256 / CPR, PER = N / STEP;
  static_assert(N % STEP == 0 && PER >= 1, "whole passes");
  u32x4_t r[PER];
  int off;  // of the lane's chunk in the first rows, in bytes; negative behind dim
  int step;
  XP_DEV Stager(int64_t stride, int dim) {
    const int c = threadIdx.x % CPR, at = threadIdx.x / CPR;
    off = c * CHUNK<T> < dim ? (int)((at * stride + c * CHUNK<T>) * (int64_t)sizeof(T)) : -1;
    step = (int)(STEP * stride * (int64_t)sizeof(T));
  }
  // rows from p on; zeros from the limit-th on, and where doc is negative
  XP_DEV void load(const T* p, int limit, const int32_t* doc) {
    const int off = fresh(this->off);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, 0x7ffffff0, 0x00020000);
    if (limit >= N && !doc) {
#pragma unroll
      for (int i = 0; i < PER; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, off < 0 ? off : off + i * step, 0, 0);
    } else {
      const int at = fresh(threadIdx.x) / CPR;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = at + i * STEP;
        bool use = off >= 0 && row < limit;
        if (doc && use) use = doc[row] >= 0;
        r[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, use ? off + i * step : -1, 0, 0);
      }
    }
  }
  XP_DEV void store(uint32_t tile) const {
    const int tid = fresh(threadIdx.x), c = tid & (CPR - 1), at = (tid & 255) / CPR;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int row = at + i * STEP;
      *lds<u32x4_t>(tile + row * ROW<T, DP> + ((c ^ swz<T, DP>(row)) << 4)) = r[i];
    }
  }
};

// a row's part for the lane as a column operand: chunks 2 s + lane / 32
template <typename T, int DP>
XP_DEV void ld_column(const T* row, bool valid, int dim, u32x4_t (&f)[DP / CHUNK<T> / 2]) {
  const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int s = 0; s < DP / CHUNK<T> / 2; ++s) {
    const int at = (2 * s + h) * CHUNK<T>;
    u32x4_t u = {0, 0, 0, 0};
    if (valid && at < dim) u = *reinterpret_cast<const u32x4_t*>(row + at);
    f[s] = u;
  }
}

// [batch][token][head][dim] with any strides to contiguous rows of ldim elements, zeros behind dim
template <typename T>
__global__ __launch_bounds__(256) void k_attn_pack(AttnMat from, T* __restrict__ to, int64_t rows, int tokens, int heads, int dim, int ldim) {
  const int per = ldim / CHUNK<T>;
  const int64_t n = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int c = (int)(i % per) * CHUNK<T>, h = (int)(row % heads), t = (int)(row / heads % tokens);
    const int64_t b = row / heads / tokens;
    const T* p = (const T*)from.p + b * from.b + t * from.t + h * from.h + c;
    *reinterpret_cast<u32x4_t*>(to + i * CHUNK<T>) = ld_chunk(p, dim - c);
  }
}

// ---------------------------------------------------------------- products
template <typename T>
XP_DEV f32x16_t mma(const u32x4_t& a, const u32x4_t& b, f32x16_t c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
}
// Row of a block that register r of a result holds: 8 (r / 4) + 4 (lane / 32) + r % 4.
XP_DEV int row_of(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x >> 5) & 1) + (r & 3); }

// A lane's first address in a tile at 0, for reads along rows and down columns.
template <typename T, int DP>
XP_DEV uint32_t row_place() {
  const int r = threadIdx.x & 31, h = (threadIdx.x >> 5) & 1;
  return r * ROW<T, DP> + ((h ^ swz<T, DP>(r)) << 4);
}
template <typename T, int DP>
XP_DEV uint32_t column_place() {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int row = 4 * h + ((lane & 15) >> 2), chunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    return row * ROW<T, DP> + ((chunk ^ swz<T, DP>(row)) << 4) + 8 * (lane & 1);
  } else {
    const int col = lane & 31;
    return 4 * h * ROW<T, DP> + (((col >> 2) ^ swz<T, DP>(4 * h)) << 4) + 4 * (col & 3);
  }
}

// 32 rows of a tile, `more` bytes from it on, times the lanes' N columns; at: row_place + tile
template <typename T, int DP, int N>
XP_DEV void rows_times(uint32_t at, int more, const u32x4_t (&col)[N][DP / CHUNK<T> / 2], f32x16_t (&out)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) out[c][i] = 0.f;
#pragma unroll
  for (int s = 0; s < DP / CHUNK<T> / 2; ++s) {
    const u32x4_t a = *lds<u32x4_t>((at ^ (s * 32)) + more);
#pragma unroll
    for (int c = 0; c < N; ++c) out[c] = mma<T>(a, col[c][s], out[c]);
  }
}
template <typename T, int DP>
XP_DEV f32x16_t rows_times(uint32_t at, int more, const u32x4_t (&col)[DP / CHUNK<T> / 2]) {
  f32x16_t out[1];
  rows_times<T, DP, 1>(at, more, reinterpret_cast<const u32x4_t(&)[1][DP / CHUNK<T> / 2]>(col), out);
  return out[0];
}

// acc[c][d][lane's column] += sum over 32 rows of tile[row][d] w[c][row]; at: column_place + tile
template <typename T, int DP, int N>
XP_DEV void add_transposed(f32x16_t (&acc)[N][DP / 32], uint32_t at, int more, const float (&w)[N][16]) {
  if constexpr (sizeof(T) == 2) {
    typedef short v4i16 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < 2; ++b) {  // 16 rows: 4 lane / 32 + 0 .. 3 of them, and 8 further on
      u32x4_t f[N];
#pragma unroll
      for (int c = 0; c < N; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) f[c][i] = f32x2_to_bf16x2(w[c][8 * b + 2 * i], w[c][8 * b + 2 * i + 1]);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        v4i16 part[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          part[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds<v4i16>((at ^ (d * 64 + k * 32)) + (more + (16 * b + 8 * k) * ROW<T, DP>)));
        const u32x4_t x = __builtin_bit_cast(u32x4_t, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int c = 0; c < N; ++c) acc[c][d] = mma<T>(x, f[c], acc[c][d]);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const float x = *lds<float>((at ^ (d * 128 + ((r >> 2) & 1) * 64 + (r & 3) * 16)) + (more + (8 * (r >> 2) + (r & 3)) * ROW<T, DP>));
#pragma unroll
        for (int c = 0; c < N; ++c) acc[c][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w[c][r], acc[c][d], 0, 0, 0);
      }
  }
}
template <typename T, int DP>
XP_DEV void add_transposed(f32x16_t (&acc)[DP / 32], uint32_t at, int more, const float (&w)[16]) {
  add_transposed<T, DP, 1>(reinterpret_cast<f32x16_t(&)[1][DP / 32]>(acc), at, more, reinterpret_cast<const float(&)[1][16]>(w));
}

// The lane's column of a result [DP][32], times f, to a row of dim elements in memory.
template <typename T, int DP>
XP_DEV void st_column(T* row, int dim, const f32x16_t (&acc)[DP / 32], float f) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at = d * 32 + row_of(4 * g);
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = acc[d][4 * g + i] * f;
      if (at + 4 <= dim) {
        if constexpr (sizeof(T) == 4) {
          __builtin_memcpy(row + at, v, 16);
        } else {
          const uint32_t u[2] = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
          __builtin_memcpy(row + at, u, 8);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at + i < dim) std_(row + at + i, (double)v[i]);
      }
    }
}

// Nothing moves over this line: without it the compiler starts the next product's reads so
// early that the registers do not hold them.
XP_DEV void phase() { __builtin_amdgcn_sched_barrier(0); }

// ---------------------------------------------------------------- halves and waves
// the larger, and the sum, of a value in lanes l and l ^ 32
XP_DEV float both_max(float v) {
  const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
}
XP_DEV float both_sum(float v) {
  const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(u[0]) + __uint_as_float(u[1]);
}
XP_DEV float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// ---------------------------------------------------------------- masks
// The keys that a query sees of its own sequence are the first kend of them (causal: up
// to its own position, which is that of the last queries of the sequence; a prefix that
// is longer; never beyond the sequence's keys), those of other documents left out.
struct Seq {
  int ql, kl, off, prefix;  // off: key position of query 0
  bool causal;
  XP_DEV Seq(const AttnArgs& a, int b) {
    ql = a.q_len ? min(max(a.q_len[b], 0), a.nq) : a.nq;
    kl = a.k_len ? min(max(a.k_len[b], 0), a.nk) : a.nk;
    off = kl - ql;
    prefix = a.prefix ? a.prefix[b] : 0;
    causal = a.causal != 0;
  }
  // not falling with i, for i < ql
  XP_DEV int kend(int i) const { return causal ? min(kl, max(max(i + off + 1, prefix), 0)) : kl; }
};

// Tiles of a walk over keys or queries, those left out that hold no document of [lo, hi].
struct Walk {
  const int4* tab;
  int end, lo, hi, chunk;
  uint64_t mask;
  XP_DEV Walk(const int4* t, int e, int l, int h) : tab(t), end(e), lo(l), hi(h), chunk(-1), mask(0) {}
  // the first tile from t on, or end
  XP_DEV int next(int t) {
    if (!tab) return min(t, end);
    while (t < end) {
      if ((t >> 6) != chunk) {
        chunk = t >> 6;
        const int at = chunk * 64 + (threadIdx.x & 63);
        const int4 e = at < end ? tab[at] : make_int4(INT_MAX, -1, 1, 0);
        mask = __ballot(e.x <= hi && e.y >= lo);
      }
      const uint64_t m = mask >> (t & 63);
      if (m) return __builtin_amdgcn_readfirstlane(t + __builtin_ctzll(m));
      t = (chunk + 1) * 64;
    }
    return end;
  }
};

// {smallest, largest document, whether the tile holds several or padding, whether padding} of each tile
__global__ __launch_bounds__(64) void k_attn_docs(const int32_t* __restrict__ doc, const int32_t* __restrict__ len, int n, int tile,
                                                   int4* __restrict__ tab) {
  const int b = blockIdx.y, limit = len ? min(max(len[b], 0), n) : n;
  const int at = blockIdx.x * tile + threadIdx.x;
  const bool in = (int)threadIdx.x < tile && at < limit;
  const int d = in ? doc[(int64_t)b * n + at] : -1;
  int lo = d >= 0 ? d : INT_MAX, hi = d;
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, 64));
    hi = max(hi, __shfl_xor(hi, o, 64));
  }
  const bool pad = __any((int)threadIdx.x < tile && d < 0);
  if (threadIdx.x == 0) tab[(int64_t)b * gridDim.x + blockIdx.x] = make_int4(lo, hi < 0 ? -1 : hi, lo != hi || pad, pad);
}

// smallest and largest document over a workgroup's rows, and over the wave's; negative ones do not count
struct DocRange { int lo, hi, wlo, whi; };
template <int N>
XP_DEV DocRange doc_range(const int (&doc)[N], int (*sh)[2]) {
  DocRange d;
  d.wlo = INT_MAX;
  d.whi = -1;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    d.wlo = min(d.wlo, doc[c] >= 0 ? doc[c] : INT_MAX);
    d.whi = max(d.whi, doc[c]);
  }
  for (int o = 32; o > 0; o >>= 1) {
    d.wlo = min(d.wlo, __shfl_xor(d.wlo, o, 64));
    d.whi = max(d.whi, __shfl_xor(d.whi, o, 64));
  }
  d.wlo = __builtin_amdgcn_readfirstlane(d.wlo);
  d.whi = __builtin_amdgcn_readfirstlane(d.whi);
  if ((threadIdx.x & 63) == 0) {
    sh[threadIdx.x >> 6][0] = d.wlo;
    sh[threadIdx.x >> 6][1] = d.whi;
  }
  __syncthreads();
  d.lo = min(min(sh[0][0], sh[1][0]), min(sh[2][0], sh[3][0]));
  d.hi = max(max(sh[0][1], sh[1][1]), max(sh[2][1], sh[3][1]));
  return d;
}

// The keys of a lane's block of 32 (from k0 on) that its query does not see, a bit for each
// register.  (Bits and selects: an element of a vector assigned under "a || b" is
// lost in places with this compiler.)
XP_DEV uint32_t hidden(int k0, int kend, const int* docs, int doc) {
  uint32_t m = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) m |= (uint32_t)(k0 + row_of(r) >= kend) << r;
  if (docs)
#pragma unroll
    for (int r = 0; r < 16; ++r) m |= (uint32_t)(docs[row_of(r)] != doc) << r;
  return m;
}

// ---------------------------------------------------------------- scores
// cap tanh(x / cap) for u = x / cap: |error| of the tanh below 2^-23 (1 - e is exact to half a
// step of 1); slope: its derivative, 4 e / (1 + e)^2
XP_DEV float capped(float u, float cap, float& slope) {
  const float e = exp2_(-2.f * LOG2E * fabsf(u)), r = __builtin_amdgcn_rcpf(1.f + e);
  slope = 4.f * e * r * r;
  return cap * copysignf((1.f - e) * r, u);
}

// The bias of a head for a lane, by distance; the two ends stand for all further ones.
struct Bias {
  const float* at;  // distance 0
  int range;
  float left, right;
  XP_DEV Bias(const AttnArgs& a, int head) {
    range = a.range;
    at = a.bias ? a.bias + (int64_t)head * (2 * range + 1) + range : nullptr;
    left = at ? at[-range] : 0.f;
    right = at ? at[range] : 0.f;
  }
  XP_DEV float get(int d) const { return at[min(max(d, -range), range)]; }
};

// Scores of a 32 x 32 block in place from its products (GEN; otherwise they stay products).
// KEYS: the rows are keys and the lane a query, dist = first key - the query's position;
// otherwise the lane is a key and dist = key - the first query's position.  dmin, dmax: the
// distances that the block holds.  slope: of the cap, 1 without one.
template <bool KEYS, bool SLOPE>
XP_DEV void scores(f32x16_t& s, const AttnArgs& a, const Bias& bias, int dist, int dmin, int dmax, float (&slope)[16]) {
  if (a.cap > 0.f) {
    const float f = a.scale / a.cap;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float c;
      s[r] = capped(s[r] * f, a.cap, c);
      if constexpr (SLOPE) slope[r] = c;
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] *= a.scale;
      if constexpr (SLOPE) slope[r] = 1.f;
    }
  }
  if (bias.at) {
    if (dmin >= bias.range || dmax <= -bias.range) {
      const float c = dmin >= bias.range ? bias.right : bias.left;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] += c;
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] += bias.get(KEYS ? dist + row_of(r) : dist - row_of(r));
    }
  }
}

// ---------------------------------------------------------------- forward
// One workgroup per 4 waves of 32 QB query rows of a head (with pk > 1: of the pk heads that
// share keys, row r being query r / pk of head r % pk), and part of the keys.
//
// The largest score enters the exponentials only when it has grown by more than 8 (base 2)
// since it last did: P is then at most 2^8, the sums stay in fp32's range, and the results
// are rarely multiplied.
template <typename T, int DP, bool GEN, int QB>
__global__ __launch_bounds__(256, QB == 2 && DP == 128 ? 1 : (WAVES<T, DP>)) void k_attn_fwd(AttnArgs a) {
  constexpr int KEYS = BN<T>, NB = KEYS / 32, WAVE = 32 * QB, GROUP = 4 * WAVE;
  constexpr int TILE = KEYS * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE];  // keys, values, twice
  __shared__ int sdoc[2][KEYS];
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.nq * a.pk, blocks = (rows + GROUP - 1) / GROUP, units = a.heads / a.pk;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int split = id % a.splits;
  id /= a.splits;
  const int blk = blocks - 1 - id % blocks;  // (causal: the longest first)
  id /= blocks;
  const int unit = id % units, b = id / units;
  const int kvh = unit * a.pk / (a.heads / a.kv_heads);
  const Seq seq(a, b);

  // limits of the workgroup's and the wave's rows (of those that count)
  const int last = min((min(rows, (blk + 1) * GROUP) - 1) / a.pk, seq.ql - 1), first = blk * GROUP / a.pk;
  const int kmax = first <= last ? seq.kend(last) : 0;
  const int row0 = blk * GROUP + wave * WAVE;
  const int wfirst = row0 / a.pk, wlast = min((row0 + WAVE - 1) / a.pk, min(a.nq, seq.ql) - 1);
  const int wmax = wfirst <= wlast ? seq.kend(wlast) : 0, wmin = wfirst <= wlast ? seq.kend(wfirst) : 0;

  int doc[QB], kend[QB], pos[QB], head[QB];
  u32x4_t q[QB][DP / CHUNK<T> / 2];
#pragma unroll
  for (int c = 0; c < QB; ++c) {
    const int row = row0 + c * 32 + (lane & 31), i = row / a.pk;
    const bool live = row < rows && i < seq.ql;
    head[c] = unit * a.pk + row % a.pk;
    doc[c] = a.q_doc ? (live ? a.q_doc[(int64_t)b * a.nq + i] : -1) : 0;
    kend[c] = live && doc[c] >= 0 ? seq.kend(i) : 0;
    pos[c] = i + seq.off;
    ld_column<T, DP>((const T*)a.q.p + b * a.q.b + (int64_t)i * a.q.t + head[c] * a.q.h, live, a.ldim, q[c]);
  }
  DocRange docs = {0, 0, 0, 0};
  if (a.q_doc) docs = doc_range<QB>(doc, sh);
  const T* kp = (const T*)a.k.p + b * a.k.b + kvh * a.k.h;
  const T* vp = (const T*)a.v.p + b * a.v.b + kvh * a.v.h;
  const int32_t* kdoc = a.k_doc ? a.k_doc + (int64_t)b * a.nk : nullptr;

  const int tiles = (kmax + KEYS - 1) / KEYS, per = (tiles + a.splits - 1) / a.splits;
  const int tab_tiles = (a.nk + KEYS - 1) / KEYS;
  Walk walk(a.k_tab ? a.k_tab + (int64_t)b * tab_tiles : nullptr, min(tiles, (split + 1) * per), docs.lo, docs.hi);

  // m: the largest of the products (GEN: of the scores) so far, base: the one in the
  // exponentials; l: this lane's part of the sum
  const float c1 = GEN ? LOG2E : a.scale * LOG2E;
  float m[QB], base[QB], l[QB];
  f32x16_t acc[QB][DP / 32];
#pragma unroll
  for (int c = 0; c < QB; ++c) {
    m[c] = base[c] = NEG_INF;
    l[c] = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[c][d][r] = 0.f;
  }

  Stager<T, DP, KEYS> ks(a.k.t, a.ldim), vs(a.v.t, a.ldim);
  int dreg = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = t * KEYS;
    const int32_t* pad = kdoc && walk.tab[t].w ? kdoc + j0 : nullptr;
    ks.load(kp + (int64_t)j0 * a.k.t, seq.kl - j0, pad);
    vs.load(vp + (int64_t)j0 * a.v.t, seq.kl - j0, pad);
    if (kdoc && threadIdx.x < KEYS) dreg = j0 + (int)threadIdx.x < seq.kl ? kdoc[j0 + threadIdx.x] : -1;
  };
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  auto store = [&](int buf) __attribute__((always_inline)) {
    ks.store(tile0 + buf * 2 * TILE);
    vs.store(tile0 + buf * 2 * TILE + TILE);
    if (kdoc && threadIdx.x < KEYS) sdoc[buf][threadIdx.x] = dreg;
  };
  int t = walk.next(min(tiles, split * per)), buf = 0;
  if (t < walk.end) {
    load(t);
    store(0);
  }
  while (t < walk.end) {
    const int tn = walk.next(t + 1);
    if (tn < walk.end) load(tn);
    __syncthreads();
    bool mixed = false, skip = t * KEYS >= wmax;
    if (kdoc) {
      const int4 e = walk.tab[t];
      skip = skip || e.x > docs.whi || e.y < docs.wlo;
      mixed = e.z || docs.wlo != docs.whi;
    }
    if (!skip) {
      const uint32_t rat = rplace + buf * 2 * TILE, cat = cplace + buf * 2 * TILE;
      const bool masked = mixed || (t + 1) * KEYS > wmin;
      f32x16_t s[NB][QB];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int n = 0; n < NB; ++n) rows_times<T, DP, QB>(rat, n * 32 * ROW<T, DP>, q, s[n]);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int k0 = t * KEYS + n * 32;
        if constexpr (GEN) {
          float none[16];
#pragma unroll
          for (int c = 0; c < QB; ++c) {
            const Bias bias(a, min(head[c], a.heads - 1));
            scores<true, false>(s[n][c], a, bias, k0 - pos[c], k0 - wlast - seq.off, k0 + 31 - wfirst - seq.off, none);
          }
        }
        if (masked) {
#pragma unroll
          for (int c = 0; c < QB; ++c) {
            const uint32_t hide = hidden(k0, kend[c], kdoc ? sdoc[buf] + n * 32 : nullptr, doc[c]);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][c][r] = hide >> r & 1 ? NEG_INF : s[n][c][r];
          }
        }
      }
      __builtin_amdgcn_s_setprio(0);
      bool grown = false;
#pragma unroll
      for (int c = 0; c < QB; ++c) {
        float top = s[0][c][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][c][r]);
        m[c] = fmaxf(m[c], both_max(top));
        grown = grown || (m[c] - base[c]) * c1 > 8.f;  // (from -inf on: infinite; while there is no key: NaN)
      }
      if (__any(grown)) {
#pragma unroll
        for (int c = 0; c < QB; ++c) {
          const float keep = m[c] == NEG_INF ? 1.f : exp2_((base[c] - m[c]) * c1);
          base[c] = m[c];
          l[c] *= keep;
#pragma unroll
          for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[c][d][r] *= keep;
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float p[QB][16];
#pragma unroll
        for (int c = 0; c < QB; ++c) {
          const float off = base[c] == NEG_INF ? 0.f : base[c], bc = off * c1;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            p[c][r] = GEN ? exp2_((s[n][c][r] - off) * c1) : exp2_(s[n][c][r] * c1 - bc);
            l[c] += p[c][r];
          }
        }
        add_transposed<T, DP, QB>(acc, cat, TILE + n * 32 * ROW<T, DP>, p);
      }
    }
    buf ^= 1;
    if (tn < walk.end) store(buf);
    t = tn;
  }

#pragma unroll
  for (int c = 0; c < QB; ++c) {
    const int row = row0 + c * 32 + (lane & 31), i = row / a.pk;
    // (a NaN among the scores leaves l NaN, and the row NaN)
    const float sum = both_sum(l[c]);
    const bool none = kend[c] == 0 || sum == 0.f;
    const float ms = none ? NEG_INF : GEN ? m[c] : m[c] * a.scale, ls = none ? 0.f : sum * exp2_((base[c] - m[c]) * c1);
    if (row >= rows) continue;
    if (a.splits > 1) {
      // (o's part belongs to `base`; a sum of zero leaves it unwritten)
      const int64_t r = ((int64_t)split * a.batch + b) * a.heads * a.nq + (int64_t)head[c] * a.nq + i;
      if (lane < 32) {
        a.part_ml[2 * r] = ms;
        a.part_ml[2 * r + 1] = ls;
      }
      st_column<float, DP>(a.part_o + r * DP, none ? 0 : DP, acc[c], exp2_((base[c] - m[c]) * c1));
      continue;
    }
    if (a.stats && lane < 32) {
      float* st = a.stats + 2 * (((int64_t)b * a.heads + head[c]) * a.nq + i);
      st[0] = ms;
      st[1] = ls;
    }
    if (none)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][d][r] = 0.f;
    st_column<T, DP>((T*)a.o.p + b * a.o.b + (int64_t)i * a.o.t + head[c] * a.o.h, a.dim, acc[c], none ? 0.f : 1.f / sum);
  }
}

// The parts of the keys joined: one wave per query row.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq, r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int i = (int)(r % a.nq), head = (int)(r / a.nq % a.heads), b = (int)(r / a.nq / a.heads);
  float m = NEG_INF;
  for (int p = 0; p < a.splits; ++p) m = fmaxf(m, a.part_ml[2 * (p * rows + r)]);
  const float base = m == NEG_INF ? 0.f : m;
  float l = 0.f, o[DP / 64];
#pragma unroll
  for (int d = 0; d < DP / 64; ++d) o[d] = 0.f;
  for (int p = 0; p < a.splits; ++p) {
    const float lp = a.part_ml[2 * (p * rows + r) + 1];
    if (lp == 0.f) continue;  // (its part of o was not written)
    const float w = exp2_((a.part_ml[2 * (p * rows + r)] - base) * LOG2E);
    l += lp * w;
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) o[d] += w * (lp == lp ? a.part_o[(p * rows + r) * DP + d * 64 + lane] : lp);
  }
  if (a.stats && lane == 0) {
    a.stats[2 * r] = m;
    a.stats[2 * r + 1] = l;
  }
  T* out = (T*)a.o.p + b * a.o.b + (int64_t)i * a.o.t + head * a.o.h;
#pragma unroll
  for (int d = 0; d < DP / 64; ++d) {
    const int at = d * 64 + lane;
    if (at < a.dim) std_(out + at, (double)(l == 0.f ? 0.f : o[d] / l));
  }
}

// ---------------------------------------------------------------- statistics of a row
// P = exp2(score' - row.a) with score' in units of log 2, where row.a has the sum's logarithm
// in it; GEN (a bias can be as large as fp32 goes): exp2((score - row.a) log2(e) - row.b) with
// the sum's logarithm apart.  A row without keys gives 0.
struct RowStat { float a, b; };
template <bool GEN>
XP_DEV RowStat row_stat(float m, float l) {
  if (l == 0.f) return {__builtin_inff(), 0.f};
  const float log2l = __builtin_amdgcn_logf(l);
  if constexpr (GEN) return {m, log2l};
  else return {m * LOG2E + log2l, 0.f};
}
template <bool GEN>
XP_DEV float weight(float s, float a, float b, float c1) {
  return GEN ? exp2_((s - a) * LOG2E - b) : exp2_(s * c1 - a);
}
// What k_attn_dkv needs of 32 query rows: row.a, row.b, sum of P dP, kend, document, 32 each, and
// room up to ROW_INFO floats.
constexpr int ROW_INFO = 256;

// Blocks of 32 keys (from key kw on) by 32 queries that hold a distance within the bias's
// range: the first one's index, of at most near_blocks().
XP_DEV int first_near(const AttnArgs& a, const Seq& seq, int kw) { return max(0, ((kw - 31 - seq.off - a.range) >> 5) + 1); }

// ---------------------------------------------------------------- gradient of the queries
// As the forward, a lane a query: scores and dP from the keys' and values' rows, then
// dq += dX K.  do . o comes from the stored o here (rounded, as dq itself will be); the same
// sum as P dP in fp32, which the loop makes by the way, is what k_attn_dkv reads: bias
// gradients are fp32, and a rounded o would show in their sums.
template <typename T, int DP, bool GEN>
__global__ __launch_bounds__(256, (WAVES<T, DP>)) void k_attn_dq(AttnArgs a) {
  constexpr int KEYS = BN_DQ<T, DP>, NB = KEYS / 32;
  constexpr int TILE = KEYS * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE];  // keys, values, twice
  __shared__ int sdoc[2][KEYS];
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (a.nq + ROWS - 1) / ROWS;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int blk = blocks - 1 - id % blocks;
  id /= blocks;
  const int head = id % a.heads, b = id / a.heads;
  const int kvh = head / (a.heads / a.kv_heads);
  const Seq seq(a, b);

  const int i = blk * ROWS + wave * 32 + (lane & 31);
  const bool in = i < a.nq, live = in && i < seq.ql;
  const int doc = a.q_doc ? (live ? a.q_doc[(int64_t)b * a.nq + i] : -1) : 0;
  const int kend = live && doc >= 0 ? seq.kend(i) : 0, pos = i + seq.off;
  const int last = min((blk + 1) * ROWS, min(a.nq, seq.ql)) - 1, first = blk * ROWS;
  const int kmax = first <= last ? seq.kend(last) : 0;
  const int wfirst = first + wave * 32, wlast = min(wfirst + 31, last);
  const int wmax = wfirst <= wlast ? seq.kend(wlast) : 0, wmin = wfirst <= wlast ? seq.kend(wfirst) : 0;
  DocRange docs = {0, 0, 0, 0};
  if (a.q_doc) docs = doc_range<1>({doc}, sh);

  u32x4_t q[DP / CHUNK<T> / 2], g[DP / CHUNK<T> / 2];
  const bool use = live && doc >= 0;
  ld_column<T, DP>((const T*)a.q.p + b * a.q.b + (int64_t)i * a.q.t + head * a.q.h, use, a.ldim, q);
  ld_column<T, DP>((const T*)a.dout.p + b * a.dout.b + (int64_t)i * a.dout.t + head * a.dout.h, use, a.ldim, g);
  const int64_t srow = ((int64_t)b * a.heads + head) * a.nq + i;
  float delta = 0.f;
  RowStat st = {__builtin_inff(), 0.f};
  if (kend > 0) {
    const int64_t at = b * a.o.b + (int64_t)i * a.o.t + head * a.o.h;
#pragma unroll
    for (int s = 0; s < DP / CHUNK<T> / 2; ++s) {
      const int c = (2 * s + (lane >> 5)) * CHUNK<T>;
      if (c < a.dim) {
        float x[CHUNK<T>], y[CHUNK<T>];
        widen<T>(g[s], x);
        widen<T>(ld_chunk((const T*)a.o.p + at + c, a.dim - c), y);
#pragma unroll
        for (int e = 0; e < CHUNK<T>; ++e) delta += x[e] * y[e];
      }
    }
    st = row_stat<GEN>(a.stats[2 * srow], a.stats[2 * srow + 1]);
  }
  delta = both_sum(delta);
  float exact = 0.f;

  const T* kp = (const T*)a.k.p + b * a.k.b + kvh * a.k.h;
  const T* vp = (const T*)a.v.p + b * a.v.b + kvh * a.v.h;
  const int32_t* kdoc = a.k_doc ? a.k_doc + (int64_t)b * a.nk : nullptr;
  const Bias bias(a, head);

  const int tiles = (kmax + KEYS - 1) / KEYS, tab_tiles = (a.nk + KEYS - 1) / KEYS;
  Walk walk(a.k_tab ? a.k_tab + (int64_t)b * tab_tiles : nullptr, tiles, docs.lo, docs.hi);
  const float c1 = a.scale * LOG2E;
  f32x16_t acc[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;

  Stager<T, DP, KEYS> ks(a.k.t, a.ldim), vs(a.v.t, a.ldim);
  int dreg = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = t * KEYS;
    const int32_t* pad = kdoc && walk.tab[t].w ? kdoc + j0 : nullptr;
    ks.load(kp + (int64_t)j0 * a.k.t, seq.kl - j0, pad);
    vs.load(vp + (int64_t)j0 * a.v.t, seq.kl - j0, pad);
    if (kdoc && threadIdx.x < KEYS) dreg = j0 + (int)threadIdx.x < seq.kl ? kdoc[j0 + threadIdx.x] : -1;
  };
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  auto store = [&](int buf) __attribute__((always_inline)) {
    ks.store(tile0 + buf * 2 * TILE);
    vs.store(tile0 + buf * 2 * TILE + TILE);
    if (kdoc && threadIdx.x < KEYS) sdoc[buf][threadIdx.x] = dreg;
  };
  int t = walk.next(0), buf = 0;
  if (t < walk.end) {
    load(t);
    store(0);
  }
  while (t < walk.end) {
    const int tn = walk.next(t + 1);
    if (tn < walk.end) load(tn);
    __syncthreads();
    bool mixed = false, skip = t * KEYS >= wmax;
    if (kdoc) {
      const int4 e = walk.tab[t];
      skip = skip || e.x > docs.whi || e.y < docs.wlo;
      mixed = e.z || docs.wlo != docs.whi;
    }
    if (!skip) {
      const uint32_t rat = rplace + buf * 2 * TILE, cat = cplace + buf * 2 * TILE;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int k0 = t * KEYS + n * 32;
        f32x16_t s = rows_times<T, DP>(rat, n * 32 * ROW<T, DP>, q);
        phase();
        const f32x16_t dp = rows_times<T, DP>(rat, TILE + n * 32 * ROW<T, DP>, g);
        phase();
        float slope[16], ds[16];
        if constexpr (GEN)
          scores<true, true>(s, a, bias, k0 - pos, k0 - wlast - seq.off, k0 + 31 - wfirst - seq.off, slope);
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = weight<GEN>(s[r], st.a, st.b, c1);
        if (mixed || k0 + 32 > wmin) {
          const uint32_t hide = hidden(k0, kend, kdoc ? sdoc[buf] + n * 32 : nullptr, doc);
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] = hide >> r & 1 ? 0.f : ds[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          exact += ds[r] * dp[r];
          ds[r] *= dp[r] - delta;
        }
        if constexpr (GEN) {
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] *= slope[r];
        }
        phase();
        add_transposed<T, DP>(acc, cat, n * 32 * ROW<T, DP>, ds);
        phase();
      }
    }
    buf ^= 1;
    if (tn < walk.end) store(buf);
    t = tn;
  }
  exact = both_sum(exact);
  if (lane < 32) {
    float* row = a.rows + (((int64_t)b * a.heads + head) * (blocks * 4) + blk * 4 + wave) * ROW_INFO + lane;
    row[0] = st.a;
    row[32] = st.b;
    row[64] = exact;
    row[96] = __int_as_float(kend);
    row[128] = __int_as_float(doc);
  }
  if (in) st_column<T, DP>((T*)a.dq.p + b * a.dq.b + (int64_t)i * a.dq.t + head * a.dq.h, a.dim, acc, a.scale);
}

// grad_bias[head][x] += the sum over sequences and key blocks of the blocks' diagonals at
// that distance: a workgroup takes 64 distances of a head, its 16 waves every 16th (sequence, 32 keys).
__global__ __launch_bounds__(1024) void k_attn_dbias(AttnArgs a) {
  __shared__ double sh[16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.y;
  const int x = blockIdx.x * 64 + lane, d = x - a.range, width = 2 * a.range + 1;
  const int blocks = (a.nk + ROWS - 1) / ROWS * 4;
  const bool outer = x == 0 || x >= width - 1;
  double s = 0.0;
  for (int b = 0; b < a.batch; ++b) {
    const Seq seq(a, b);
    const int64_t at0 = ((int64_t)b * a.heads + head) * blocks;
    const int used = min(blocks, (seq.kl + 31) / 32);
#pragma unroll 4
    for (int w = wave; w < used; w += 16) {
      const int64_t at = at0 + w;
      float v0 = 0.f, v1 = 0.f;
      if (outer) {
        if (x < width) v0 = a.tail[2 * at + (x == 0 ? 0 : 1)];
      } else {
        // of block t the distances from w 32 - 32 t - 31 - off on: places u in the two blocks that hold d
        const int near0 = first_near(a, seq, w * 32), from = d - w * 32 + 31 + seq.off, u = from & 31, t = (u - from) >> 5;
        const float* part = a.diag + at * a.near * 64;
        if (t >= near0 && t - near0 < a.near) v0 = part[(t - near0) * 64 + u];
        if (u < 31 && t + 1 >= near0 && t + 1 - near0 < a.near) v1 = part[(t + 1 - near0) * 64 + u + 32];
      }
      s += (double)v0 + v1;
    }
  }
  sh[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && x < width) {
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += sh[w][lane];
    float* g = a.grad_bias + (int64_t)head * width + x;
    *g = (float)((double)*g + s);
  }
}

// ---------------------------------------------------------------- gradients of keys and values
// A lane is a key, steps of 32 queries in LDS (those of all heads that share the keys, one
// head after another): dv += P^T do, dk += dX^T q.  WHAT: 3 both, 1 dv, 2 dk (fp32 rows of
// 128: both sums and both operands would not fit a lane's registers).  With grad_bias also
// the sums of dS along the diagonals of each block of 32 x 32 near the diagonal, and over
// the blocks beyond the bias's range on either side.
template <typename T, int DP, bool GEN, int WHAT>
__global__ __launch_bounds__(256, GEN && DP == 128 ? 1 : (WAVES<T, DP>)) void k_attn_dkv(AttnArgs a) {
  constexpr int TILE = QT * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE];  // q, dout, twice
  __shared__ float srow[2][5 * QT];
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (a.nk + ROWS - 1) / ROWS, group = a.heads / a.kv_heads;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int blk = id % blocks;  // (causal: the first keys have the most queries)
  id /= blocks;
  const int kvh = id % a.kv_heads, b = id / a.kv_heads;
  const Seq seq(a, b);
  const int k0 = blk * ROWS, kw = k0 + wave * 32, j = kw + (lane & 31);
  const bool in = j < a.nk;
  const int doc = a.k_doc ? (j < seq.kl ? a.k_doc[(int64_t)b * a.nk + j] : -1) : 0;
  DocRange docs = {0, 0, 0, 0};
  bool pad = false;
  if (a.k_doc) {
    docs = doc_range<1>({doc}, sh);
    pad = __any(doc < 0);
  }
  u32x4_t kc[DP / CHUNK<T> / 2], vc[DP / CHUNK<T> / 2];
  const bool use = j < seq.kl && doc >= 0;
  ld_column<T, DP>((const T*)a.k.p + b * a.k.b + (int64_t)j * a.k.t + kvh * a.k.h, use, a.ldim, kc);
  if constexpr (WHAT & 2)
    ld_column<T, DP>((const T*)a.v.p + b * a.v.b + (int64_t)j * a.v.t + kvh * a.v.h, use, a.ldim, vc);
  const int32_t* qdoc = a.q_doc ? a.q_doc + (int64_t)b * a.nq : nullptr;

  // queries that see a key of the workgroup: those with kend > k0, from the first such on
  int tiles = (seq.ql + QT - 1) / QT, t0 = 0;
  if (k0 >= seq.kl) tiles = 0;
  else if (seq.causal && seq.prefix <= k0) t0 = min(tiles, max(0, k0 - seq.off) / QT);
  const int tab_tiles = (a.nq + QT - 1) / QT;
  Walk walk(a.q_tab ? a.q_tab + (int64_t)b * tab_tiles : nullptr, tiles, docs.lo, docs.hi);

  f32x16_t dk[WHAT & 2 ? DP / 32 : 1], dv[WHAT & 1 ? DP / 32 : 1];
#pragma unroll
  for (auto& d : dk)
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = 0.f;
#pragma unroll
  for (auto& d : dv)
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = 0.f;
  const float c1 = a.scale * LOG2E;

  const bool diag = GEN && (WHAT & 2) && a.grad_bias;
  float left = 0.f, right = 0.f;
  const int near0 = first_near(a, seq, kw);
  const int64_t wblock = blk * 4 + wave, wblocks = blocks * 4;
  if (diag)  // blocks that no step reaches
    for (int h = kvh * group; h < (kvh + 1) * group; ++h) {
      const int64_t w = ((int64_t)b * a.heads + h) * wblocks + wblock;
      for (int n = 0; n < a.near; ++n) a.diag[(w * a.near + n) * 64 + lane] = 0.f;
      if (lane < 2) a.tail[2 * w + lane] = 0.f;
    }

  Stager<T, DP, QT> qs(a.q.t, a.ldim), gs(a.dout.t, a.ldim);
  const int row_tiles = (a.nq + ROWS - 1) / ROWS * 4;
  float rreg = 0.f;
  auto load = [&](int t, int head) __attribute__((always_inline)) {
    const int i0 = t * QT;
    const int32_t* pads = qdoc && walk.tab[t].w ? qdoc + i0 : nullptr;
    qs.load((const T*)a.q.p + b * a.q.b + head * a.q.h + i0 * a.q.t, seq.ql - i0, pads);
    gs.load((const T*)a.dout.p + b * a.dout.b + head * a.dout.h + i0 * a.dout.t, seq.ql - i0, pads);
    if (threadIdx.x < 5 * QT) rreg = a.rows[(((int64_t)b * a.heads + head) * row_tiles + t) * ROW_INFO + threadIdx.x];
  };
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  auto store = [&](int buf) __attribute__((always_inline)) {
    qs.store(tile0 + buf * 2 * TILE);
    gs.store(tile0 + buf * 2 * TILE + TILE);
    if (threadIdx.x < 5 * QT) srow[buf][threadIdx.x] = rreg;
  };
  int g = 0, t = walk.next(t0), buf = 0;
  const int t_first = t;
  const bool any = t < walk.end;
  if (any) {
    load(t, kvh * group);
    store(0);
  }
  while (any && g < group) {
    int tn = walk.next(t + 1), gn = g;
    if (tn >= walk.end) {
      tn = t_first;
      ++gn;
    }
    if (gn < group) load(tn, kvh * group + gn);
    __syncthreads();
    const int i0 = t * QT, i1 = min(i0 + QT, seq.ql) - 1;
    bool mixed = false, skip = seq.kend(i1) <= kw;
    if (qdoc) {
      const int4 e = walk.tab[t];
      skip = skip || e.x > docs.whi || e.y < docs.wlo;
      mixed = e.z || pad || docs.wlo != docs.whi;
    }
    if (!skip) {
      const uint32_t rat = rplace + buf * 2 * TILE, cat = cplace + buf * 2 * TILE;
      const int head = kvh * group + g;
      f32x16_t s = rows_times<T, DP>(rat, 0, kc);
      phase();
      float p[16], slope[16];
      if constexpr (GEN) {
        const Bias bias(a, head);
        const int dist = j - i0 - seq.off;
        scores<false, true>(s, a, bias, dist, kw - i1 - seq.off, kw + 31 - i0 - seq.off, slope);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = weight<GEN>(s[r], srow[buf][row_of(r)], GEN ? srow[buf][32 + row_of(r)] : 0.f, c1);
      const bool masked = mixed || i0 + QT > seq.ql || seq.kend(i0) < kw + 32;
      if (masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = j >= __float_as_int(srow[buf][96 + row_of(r)]) ? 0.f : p[r];
        if (qdoc)
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] = __float_as_int(srow[buf][128 + row_of(r)]) != doc ? 0.f : p[r];
      }
      if constexpr (WHAT & 1) {
        phase();
        add_transposed<T, DP>(dv, cat, TILE, p);
        phase();
      }
      if constexpr (WHAT & 2) {
        const f32x16_t dp = rows_times<T, DP>(rat, TILE, vc);
        phase();
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] *= dp[r] - srow[buf][64 + row_of(r)];
        if (diag) {
          const int dlow = kw - i0 - 31 - seq.off;  // the block's smallest distance
          if (dlow + 62 <= -a.range || dlow >= a.range) {
            float w = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) w += p[r];
            if (dlow >= a.range) right += w;
            else left += w;
          } else {
            // Register r holds query k = row_of(r) and key lane % 32: distance dlow + u, u =
            // lane % 32 - k + 31.  Pushed to lane u the first half's values lie in 32 lanes, and
            // the second half's, four queries on, go to the other 32 (u to lane u + 36 of 64).
            float lo = 0.f, hi = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int k = 8 * (r >> 2) + (r & 3), to = ((lane & 31) + 31 - k + (lane & 32)) & 63;
              const float v = __uint_as_float(__builtin_amdgcn_ds_permute(to * 4, __float_as_uint(p[r])));
              const bool low = (unsigned)(lane - (31 - k)) < 32u;
              lo += low ? v : 0.f;
              hi += low ? 0.f : v;
            }
            lo += __uint_as_float(__builtin_amdgcn_ds_bpermute(((lane + 36) & 63) * 4, __float_as_uint(hi)));
            const int d = dlow + lane;
            const bool outer = d <= -a.range || d >= a.range;
            if (d <= -a.range) left += lo;
            else if (d >= a.range) right += lo;
            const int64_t w = ((int64_t)b * a.heads + head) * wblocks + wblock;
            a.diag[(w * a.near + (t - near0)) * 64 + lane] = outer ? 0.f : lo;
          }
        }
        if constexpr (GEN) {
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] *= slope[r];
        }
        phase();
        add_transposed<T, DP>(dk, cat, 0, p);
      }
    }
    if (diag && gn != g) {  // the head's last step
      for (int o = 32; o > 0; o >>= 1) {
        left += __shfl_xor(left, o, 64);
        right += __shfl_xor(right, o, 64);
      }
      if (lane == 0) {
        float* w = a.tail + 2 * (((int64_t)b * a.heads + kvh * group + g) * wblocks + wblock);
        w[0] = left;
        w[1] = right;
      }
      left = right = 0.f;
    }
    buf ^= 1;
    if (gn < group) store(buf);
    t = tn;
    g = gn;
  }
  if (!in) return;
  if constexpr (WHAT & 1) st_column<T, DP>((T*)a.dv.p + b * a.dv.b + (int64_t)j * a.dv.t + kvh * a.dv.h, a.dim, dv, 1.f);
  if constexpr (WHAT & 2) st_column<T, DP>((T*)a.dk.p + b * a.dk.b + (int64_t)j * a.dk.t + kvh * a.dk.h, a.dim, dk, a.scale);
}

// ---------------------------------------------------------------- launches
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
int padded_dim(int dim) { return dim <= 64 ? 64 : 128; }
int keys_of(int dtype) { return dtype == DT_BF16 ? BN<bf16_t> : BN<float>; }
int dq_keys_of(int dtype, const AttnArgs& a) { return dtype == DT_BF16 && a.dim <= 64 ? BN_DQ<bf16_t, 64> : 32; }

// Few query rows: those of the heads that share keys go into one workgroup, which then reads
// the keys once for all of them.
int rows_packed(const AttnArgs& a) {
  const int group = a.heads / a.kv_heads;
  return (int64_t)a.nq * group <= ROWS ? group : 1;
}

// Parts of the keys where the rows alone do not fill the card (two workgroups a CU): at
// least 4 steps each.
int parts(int dtype, const AttnArgs& a) {
  const int pk = rows_packed(a);
  const int64_t groups = ceil_div((int64_t)a.nq * pk, ROWS) * (a.heads / pk) * a.batch, steps = ceil_div(a.nk, keys_of(dtype));
  if (groups == 0 || groups >= 256) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(512, groups), steps / 4));
}

// whether the forward's waves take 64 query rows each
bool wide(const AttnArgs& a) { return false;
  return a.splits == 1 && ceil_div((int64_t)a.nq * a.pk, 2 * ROWS) * (a.heads / a.pk) * a.batch >= 256;
}

// blocks of 32 queries that hold distances within the range, of 32 keys
int near_blocks(const AttnArgs& a) { return (int)std::min<int64_t>(ceil_div(a.nq, 32), ceil_div(2 * (int64_t)a.range + 62, 32) + 1); }

// Inputs whose rows are not whole, aligned chunks of 16 bytes are copied to such ones first:
// the kernels read nothing else.  Places the copy at `at` in the workspace, with `from` what is to
// be copied (p null: nothing), and returns the workspace's new end.
size_t lay_packed(int dtype, AttnArgs& a, AttnMat& m, int64_t tokens, int64_t heads, char* base, size_t at, AttnMat& from) {
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  a.ldim = (a.dim + chunk - 1) / chunk * chunk;
  from = AttnMat{};
  const int64_t n = a.batch * tokens * heads;
  if (n == 0) return at;
  auto odd = [&](int64_t stride, int64_t count) { return count > 1 && stride % chunk != 0; };
  if (a.ldim == a.dim && (reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && !odd(m.b, a.batch) && !odd(m.t, tokens) && !odd(m.h, heads)) return at;
  from = m;
  m = AttnMat{base ? base + at : nullptr, tokens * heads * a.ldim, heads * a.ldim, a.ldim};
  return at + round256((size_t)n * a.ldim * es);
}

// The workspace's pieces; sets their pointers where base is given.
size_t lay_fwd(int dtype, AttnArgs& a, char* base, AttnMat* from) {
  size_t n = 0;
  auto take = [&](size_t bytes) { size_t at = n; n += round256(bytes); return base ? base + at : nullptr; };
  AttnMat* m[3] = {&a.q, &a.k, &a.v};
  for (int i = 0; i < 3; ++i) n = lay_packed(dtype, a, *m[i], i ? a.nk : a.nq, i ? a.kv_heads : a.heads, base, n, from[i]);
  a.pk = rows_packed(a);
  a.splits = parts(dtype, a);
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq;
  if (a.splits > 1) {
    a.part_o = (float*)take((size_t)rows * a.splits * padded_dim(a.dim) * 4);
    a.part_ml = (float*)take((size_t)rows * a.splits * 8);
  }
  if (a.k_doc) a.k_tab = (int4*)take((size_t)a.batch * ceil_div(a.nk, keys_of(dtype)) * sizeof(int4));
  return n;
}
size_t lay_bwd(int dtype, AttnArgs& a, char* base, AttnMat* from) {
  size_t n = 0;
  auto take = [&](size_t bytes) { size_t at = n; n += round256(bytes); return base ? base + at : nullptr; };
  AttnMat* m[4] = {&a.q, &a.k, &a.v, &a.dout};
  for (int i = 0; i < 4; ++i) {
    const bool keys = i == 1 || i == 2;
    n = lay_packed(dtype, a, *m[i], keys ? a.nk : a.nq, keys ? a.kv_heads : a.heads, base, n, from[i]);
  }
  a.rows = (float*)take((size_t)a.batch * a.heads * ceil_div(a.nq, ROWS) * 4 * ROW_INFO * 4);
  if (a.k_doc) {
    a.k_tab = (int4*)take((size_t)a.batch * ceil_div(a.nk, dq_keys_of(dtype, a)) * sizeof(int4));
    a.q_tab = (int4*)take((size_t)a.batch * ceil_div(a.nq, QT) * sizeof(int4));
  }
  if (a.grad_bias) {
    const int64_t waves = (int64_t)a.batch * a.heads * ceil_div(a.nk, ROWS) * 4;
    a.near = near_blocks(a);
    a.diag = (float*)take((size_t)waves * a.near * 64 * 4);
    a.tail = (float*)take((size_t)waves * 8);
  }
  return n;
}

bool general(const AttnArgs& a) { return a.bias || a.cap > 0.f; }

// documents of the tiles of keys, and of queries
void launch_docs(const int32_t* doc, const int32_t* len, int n, int batch, int tile, int4* tab, hipStream_t s) {
  if (n == 0) return;
  XP_LAUNCH("k_attn_docs", 4.0 * batch * n, k_attn_docs, dim3((unsigned)ceil_div(n, tile), batch), dim3(64), 0, s, doc, len, n, tile, tab);
}

void launch_pack(int dtype, const AttnArgs& a, const AttnMat& from, const AttnMat& to, int64_t tokens, int64_t heads, hipStream_t s) {
  if (!from.p) return;
  const int64_t rows = (int64_t)a.batch * tokens * heads, n = rows * a.ldim;
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(n, 256 * 8), 4096);
  if (dtype == DT_BF16)
    XP_LAUNCH("k_attn_pack<bf16>", 4.0 * n, k_attn_pack<bf16_t>, dim3(blocks), dim3(256), 0, s, from, (bf16_t*)to.p, rows, (int)tokens, (int)heads, a.dim, a.ldim);
  else
    XP_LAUNCH("k_attn_pack<f32>", 8.0 * n, k_attn_pack<float>, dim3(blocks), dim3(256), 0, s, from, (float*)to.p, rows, (int)tokens, (int)heads, a.dim, a.ldim);
}

template <typename T, int DP, bool GEN>
void fwd(const AttnArgs& a, hipStream_t s) {
  const double flops = 4.0 * a.batch * a.heads * a.nq * (double)a.nk * a.dim;
  auto run = [&](auto qb) {
    constexpr int QB = decltype(qb)::value;
    const int64_t groups = ceil_div((int64_t)a.nq * a.pk, ROWS * QB) * (a.heads / a.pk) * a.batch * a.splits;
    XP_LAUNCH(sizeof(T) == 2 ? "k_attn_fwd<bf16>" : "k_attn_fwd<f32>", flops, (k_attn_fwd<T, DP, GEN, QB>), dim3((unsigned)groups), dim3(256), 0, s, a);
  };
  if constexpr (sizeof(T) == 2) {
    if (wide(a)) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 1>{});
  } else {
    run(std::integral_constant<int, 1>{});
  }
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.batch * a.heads * a.nq;
    XP_LAUNCH("k_attn_join", 4.0 * rows * a.splits * DP, (k_attn_join<T, DP>), dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, s, a);
  }
}

template <typename T, int DP, bool GEN>
void bwd(const AttnArgs& a, hipStream_t s) {
  const double pairs = (double)a.batch * a.heads * a.nq * a.nk;
  const int64_t groups = ceil_div(a.nq, ROWS) * a.heads * a.batch, kgroups = ceil_div(a.nk, ROWS) * a.kv_heads * a.batch;
  if (groups > 0)
    XP_LAUNCH(sizeof(T) == 2 ? "k_attn_dq<bf16>" : "k_attn_dq<f32>", 6 * pairs * a.dim, (k_attn_dq<T, DP, GEN>), dim3((unsigned)groups), dim3(256), 0, s, a);
  if (kgroups == 0) {
  } else if constexpr (sizeof(T) == 4 && DP == 128) {
    XP_LAUNCH("k_attn_dv<f32>", 4 * pairs * a.dim, (k_attn_dkv<T, DP, GEN, 1>), dim3((unsigned)kgroups), dim3(256), 0, s, a);
    XP_LAUNCH("k_attn_dk<f32>", 6 * pairs * a.dim, (k_attn_dkv<T, DP, GEN, 2>), dim3((unsigned)kgroups), dim3(256), 0, s, a);
  } else {
    XP_LAUNCH(sizeof(T) == 2 ? "k_attn_dkv<bf16>" : "k_attn_dkv<f32>", 8 * pairs * a.dim, (k_attn_dkv<T, DP, GEN, 3>), dim3((unsigned)kgroups),
              dim3(256), 0, s, a);
  }
  if (a.grad_bias && groups > 0 && kgroups > 0)
    XP_LAUNCH("k_attn_dbias", 4.0 * (2 * a.range + 1) * a.heads, k_attn_dbias, dim3((unsigned)ceil_div(2 * (int64_t)a.range + 1, 64), a.heads), dim3(1024), 0, s, a);
}

// calls f(element type, padded dim, whether scores need more than the scale)
template <typename F>
void by_kind(int dtype, const AttnArgs& a, F&& f) {
  using std::bool_constant;
  using std::integral_constant;
  auto with = [&](auto t, auto d) {
    if (general(a)) f(t, d, bool_constant<true>{});
    else f(t, d, bool_constant<false>{});
  };
  auto dims = [&](auto t) {
    if (a.dim <= 64) with(t, integral_constant<int, 64>{});
    else with(t, integral_constant<int, 128>{});
  };
  if (dtype == DT_BF16) dims(bf16_t{});
  else dims(float{});
}

}  // namespace

size_t attn_fwd_bytes(int dtype, const AttnArgs& a) {
  AttnArgs c = a;
  AttnMat from[3];
  return lay_fwd(dtype, c, nullptr, from);
}
size_t attn_bwd_bytes(int dtype, const AttnArgs& a) {
  AttnArgs c = a;
  AttnMat from[4];
  return lay_bwd(dtype, c, nullptr, from);
}

hipError_t launch_attn_fwd(int dtype, AttnArgs a, void* workspace, hipStream_t s) {
  AttnMat from[3];
  lay_fwd(dtype, a, (char*)workspace, from);
  launch_pack(dtype, a, from[0], a.q, a.nq, a.heads, s);
  launch_pack(dtype, a, from[1], a.k, a.nk, a.kv_heads, s);
  launch_pack(dtype, a, from[2], a.v, a.nk, a.kv_heads, s);
  if (a.k_doc) launch_docs(a.k_doc, a.k_len, a.nk, a.batch, keys_of(dtype), a.k_tab, s);
  by_kind(dtype, a, [&](auto t, auto d, auto g) { fwd<decltype(t), decltype(d)::value, decltype(g)::value>(a, s); });
  return hipGetLastError();
}

hipError_t launch_attn_bwd(int dtype, AttnArgs a, void* workspace, hipStream_t s) {
  AttnMat from[4];
  a.pk = a.splits = 1;
  lay_bwd(dtype, a, (char*)workspace, from);
  launch_pack(dtype, a, from[0], a.q, a.nq, a.heads, s);
  launch_pack(dtype, a, from[1], a.k, a.nk, a.kv_heads, s);
  launch_pack(dtype, a, from[2], a.v, a.nk, a.kv_heads, s);
  launch_pack(dtype, a, from[3], a.dout, a.nq, a.heads, s);
  if (a.k_doc) {
    launch_docs(a.k_doc, a.k_len, a.nk, a.batch, dq_keys_of(dtype, a), a.k_tab, s);
    launch_docs(a.q_doc, a.q_len, a.nq, a.batch, QT, a.q_tab, s);
  }
  by_kind(dtype, a, [&](auto t, auto d, auto g) { bwd<decltype(t), decltype(d)::value, decltype(g)::value>(a, s); });
  return hipGetLastError();
}

}  // namespace xp
