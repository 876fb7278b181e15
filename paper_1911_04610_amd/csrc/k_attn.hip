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
// a bf16 product is; scores, sums and statistics are fp32 throughout.  That leaves results 1.9e-3 to 2.4e-3 of
// their 2-norm off where their own rounding alone is 1.66e-3.  P and dX as two bf16 values everywhere reach that, for half
// of the products again: 16 heads of 8192 tokens, causal and capped, 493 us for 370; 2 x 4096 tokens, prefix, training
// step 1168 for 860.  Two values are taken where they cost little: in k_attn_few, and of dX in k_attn_dq over few keys.
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

template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);
// keys of a step of the forward, and of k_attn_dq
template <typename T> constexpr int BN = sizeof(T) == 2 ? 64 : 32;
template <typename T, int DP> constexpr int BN_DQ = sizeof(T) == 2 && DP == 64 ? 64 : 32;
// queries of a step of k_attn_dkv
template <typename T, int DP> constexpr int QT_ = sizeof(T) == 2 && DP == 64 ? 64 : 32;
// waves of a SIMD that a kernel's registers leave room for: 512 of them a lane, one wave
// where both operands' columns and the results need more than 256.  (Steps of 32 leave bf16 rows of 64 room for three in
// the backward, and cost more than these give: training step of 2 x 4096 tokens, 12 heads, causal 422 us, with steps of 32
// keys and three waves in k_attn_dq 456, and of 32 queries in k_attn_dkv 458; without a mask 619, 598, 558.)
template <typename T, int DP> constexpr int WAVES = sizeof(T) == 4 && DP > 64 ? 1 : 2;

// ---------------------------------------------------------------- tiles in LDS
// Rows of DP elements, chunk c of row r at position c ^ swz(r).  Read along rows, 16
// bytes of 16 rows at a time, and down columns (bf16: the transposing read, 4 rows of 16
// columns for every 16 lanes; fp32: 32 columns of two rows four apart): the swizzle gives
// 16 rows different places, and four neighbouring rows different groups of four chunks.
template <typename T, int DP>
XP_DEV int swz(int r) {
  if constexpr (sizeof(T) == 4) return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
  else if constexpr (DP > 64) return (r & 3) << 2 | ((r >> 2) & 3);
  else return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

template <int DP> constexpr int PITCH = DP == 64 ? 64 : 128;  // elements: rows of 96 lie as those of 128 do
template <typename T, int DP> constexpr int ROW = PITCH<DP> * (int)sizeof(T);  // bytes
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
template <typename T, int DP, int N, int THREADS = 256>
struct Stager {
  static constexpr int CPR = PITCH<DP> / CHUNK<T>, STEP = THREADS / CPR, PER = N / STEP;
  static_assert(N % STEP == 0 && PER >= 1, "whole passes");
  u32x4_t r[PER];
  int off;  // of the lane's chunk in the first rows, in bytes; negative behind dim
  int step;
  XP_DEV Stager(int64_t stride, int dim) {
    const int c = threadIdx.x % CPR, at = threadIdx.x % THREADS / CPR;
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
      const int at = fresh(threadIdx.x) % THREADS / CPR;
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
    const int tid = fresh(threadIdx.x), c = tid & (CPR - 1), at = (tid & (THREADS - 1)) / CPR;
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

// [batch][token][head][dim] with any strides to contiguous rows of ldim elements, zeros behind
// dim: all that a call has of these, one blockIdx.y each
struct PackArgs {
  AttnMat from[4];
  void* to[4];
  int64_t rows[4];
  int tokens[4], heads[4];
  int dim, ldim;
};
template <typename T>
__global__ __launch_bounds__(256) void k_attn_pack(PackArgs a) {
  const int m = blockIdx.y, per = a.ldim / CHUNK<T>;
  const AttnMat from = a.from[m];
  const int64_t n = a.rows[m] * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int c = (int)(i % per) * CHUNK<T>, h = (int)(row % a.heads[m]), t = (int)(row / a.heads[m] % a.tokens[m]);
    const int64_t b = row / a.heads[m] / a.tokens[m];
    const T* p = (const T*)from.p + b * from.b + t * from.t + h * from.h + c;
    *reinterpret_cast<u32x4_t*>((T*)a.to[m] + i * CHUNK<T>) = ld_chunk(p, a.dim - c);
  }
}

// Nothing moves over this line: without it the compiler starts the next product's reads so
// early that the registers do not hold them.
XP_DEV void phase() { __builtin_amdgcn_sched_barrier(0); }

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

// 32 rows of a tile, `more` bytes from it on, times the lanes' columns; at: row_place + tile
template <typename T, int DP>
XP_DEV f32x16_t rows_times(uint32_t at, int more, const u32x4_t (&col)[DP / CHUNK<T> / 2], int dim) {
  f32x16_t c;
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
  for (int s = 0; s < DP / CHUNK<T> / 2; ++s) {
    // (fp32 products take 16 times as long as bf16 ones: those of zeros behind dim are left out)
    if (sizeof(T) == 2 || s * 2 * CHUNK<T> < dim) {
      const u32x4_t row = *lds<u32x4_t>((at ^ (s * 32)) + more);
      c = mma<T>(row, col[s], c);
    }
  }
  return c;
}
// the same with the columns in LDS too, rows of another tile
template <typename T, int DP>
XP_DEV f32x16_t rows_times(uint32_t at, int more, uint32_t col) {
  f32x16_t c;
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
  for (int s = 0; s < DP / CHUNK<T> / 2; ++s) {
    const u32x4_t row = *lds<u32x4_t>((at ^ (s * 32)) + more), mine = *lds<u32x4_t>(col ^ (s * 32));
    c = mma<T>(row, mine, c);
    if (s % 2 == 1) phase();  // (at most four reads ahead: registers)
  }
  return c;
}

// acc[d][lane's column] += sum over 32 rows of tile[row][d] w[row]; at: column_place + tile.
// TWICE: w as two bf16 values, for 16 bits of it.
template <typename T, int DP, bool TWICE = false>
XP_DEV void add_transposed(f32x16_t (&acc)[DP / 32], uint32_t at, int more, const float (&w)[16], int dim) {
  if constexpr (sizeof(T) == 2) {
    typedef short v4i16 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < 2; ++b) {  // 16 rows: 4 lane / 32 + 0 .. 3 of them, and 8 further on
      u32x4_t f, rest;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w0 = w[8 * b + 2 * i], w1 = w[8 * b + 2 * i + 1];
        f[i] = f32x2_to_bf16x2(w0, w1);
        if constexpr (TWICE) rest[i] = f32x2_to_bf16x2(w0 - __uint_as_float(f[i] << 16), w1 - __uint_as_float(f[i] & 0xffff0000u));
      }
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        v4i16 part[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          part[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds<v4i16>((at ^ (d * 64 + k * 32)) + (more + (16 * b + 8 * k) * ROW<T, DP>)));
        const u32x4_t x = __builtin_bit_cast(u32x4_t, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        acc[d] = mma<T>(x, f, acc[d]);
        if constexpr (TWICE) acc[d] = mma<T>(x, rest, acc[d]);
      }
    }
  } else {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      if (d * 32 < dim)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = *lds<float>((at ^ (d * 128 + ((r >> 2) & 1) * 64 + (r & 3) * 16)) + (more + (8 * (r >> 2) + (r & 3)) * ROW<T, DP>));
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w[r], acc[d], 0, 0, 0);
      }
    }
  }
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

// ---------------------------------------------------------------- halves and waves
// What the wave's lanes stored in LDS before, its other lanes read behind this line, and the other way round.  (One
// wave alone: its LDS operations run in order, so this is for the compiler and costs nothing.)
XP_DEV void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
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

// {smallest, largest document, whether the tile holds several or padding, whether padding} of each
// tile of keys and of queries
struct DocArgs {
  const int32_t* doc[2];
  const int32_t* len[2];
  int n[2], tile[2], tiles[2];
  int4* tab[2];
};
__global__ __launch_bounds__(64) void k_attn_docs(DocArgs a) {
  const int w = (int)blockIdx.x >= a.tiles[0], t = blockIdx.x - (w ? a.tiles[0] : 0), b = blockIdx.y, n = a.n[w], tile = a.tile[w];
  const int limit = a.len[w] ? min(max(a.len[w][b], 0), n) : n;
  const int at = t * tile + threadIdx.x;
  const bool in = (int)threadIdx.x < tile && at < limit;
  const int d = in ? a.doc[w][(int64_t)b * n + at] : -1;
  int lo = d >= 0 ? d : INT_MAX, hi = d;
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, 64));
    hi = max(hi, __shfl_xor(hi, o, 64));
  }
  const bool pad = __any((int)threadIdx.x < tile && d < 0);
  if (threadIdx.x == 0) a.tab[w][(int64_t)b * a.tiles[w] + t] = make_int4(lo, hi < 0 ? -1 : hi, lo != hi || pad, pad);
}

// smallest and largest document over a workgroup's rows, and over the wave's; negative ones do not count
struct DocRange { int lo, hi, wlo, whi; };
XP_DEV DocRange doc_range(int doc, int (*sh)[2]) {
  DocRange d;
  d.wlo = doc >= 0 ? doc : INT_MAX;
  d.whi = doc >= 0 ? doc : -1;
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

// `none` in the place of keys that a lane's query does not see, of a block of 32 from k0 on: those
// from kend on, and (docs given) those of other documents.  (Selects, one condition at a time:
// an element of a vector assigned under "a || b" is lost in places with this compiler.)
template <typename V>
XP_DEV void hide_from(V& s, int left, float none) {  // left: kend - k0
  left -= 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) >= left ? none : s[r];
}
template <typename V>
XP_DEV void hide_others(V& s, const int* docs, int doc, float none) {
  docs += 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = docs[8 * (r >> 2) + (r & 3)] != doc ? none : s[r];
}

// ---------------------------------------------------------------- scores
// What the scores are, in units of log 2 (the exponential's):
//   PLAIN  scale q.k; held as the products q.k (c1 = scale log2(e) comes in with the exponential)
//   CAP    cap tanh(scale q.k / cap)
//   BIAS   scale q.k plus a bias
//   BOTH   CAP plus a bias
//   QUICK  CAP, bf16 storage and a cap up to QUICK_CAP
enum { PLAIN = 0, CAP = 1, BIAS = 2, BOTH = 3, QUICK = 5 };
constexpr bool has_cap(int mode) { return mode & CAP; }
constexpr bool has_bias(int mode) { return mode & BIAS; }
// exp(score - base); c1: as above
template <int MODE>
XP_DEV float exp_of(float s, float base, float c1) {
  if constexpr (MODE == PLAIN) return exp2_(s * c1 - base * c1);
  else return exp2_(s - base);
}
// a score, or a difference of two, in units of log 2
template <int MODE>
XP_DEV float log2_of(float d, float c1) { return MODE == PLAIN ? d * c1 : d; }

// Scores of a block of 32 x 32 from its products, in their place; slope: of the cap.  at(r): the bias of
// register r.  For x = scale q.k / cap the capped score is cap tanh(x), a few steps off itself at most whatever the
// cap is: below SMALL from tanh(x) / x = 1 + x^2 p(x^2), p of degree 3 with the least relative error over that
// range (2^-26), times scale q.k, so that a large cap costs no bits; beyond it 1 - 2 q with q = 1 / (1 + exp(2 x)), and
// the slope 4 q (1 - q), off by 2^-22 of 1.  Which of them a score takes depends on itself alone; a block none of whose
// scores is beyond SMALL passes the exponentials over (BOTH_WAYS, in the forward where the
// keys' bytes or the fp32 products bound: none does, for fewer registers).
// QUICK has 1 - 2 q alone: its scores are off by 12 * 2^-24 of the cap, 2^-14 at most, where P itself is rounded by 2^-8;
// with a bias, whose gradient is fp32, there is no such kind.  (16 heads of 8192 tokens, causal, scores of 1: cap 50 404 us, 409 with
// the polynomial; cap 1, where half of the scores are beyond SMALL, 390 and 552.)
constexpr float SMALL = 0.5f, QUICK_CAP = 64.f;
template <int MODE, bool SLOPE, bool BOTH_WAYS, typename F>
XP_DEV void scores(f32x16_t& s, const AttnArgs& a, float (&slope)[16], F&& at) {
  if constexpr (has_cap(MODE)) {
#pragma clang fp contract(off)  // (the bits of a score do not depend on which way its block goes)
    const float c1 = a.scale * LOG2E, k = a.scale / a.cap, top = a.cap * LOG2E;
    auto small = [&](float v, float x, float& d) __attribute__((always_inline)) {
      const float y = x * x;
      const float p = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 0.01724149f, -0.05304549f), 0.13325879f), -0.33333144f), 1.f);
      d = fmaf(-(y * p), p, 1.f);
      return v * c1 * p;
    };
    auto large = [&](float x2, float& d) __attribute__((always_inline)) {  // (2 log2(e) x)
      const float q = __builtin_amdgcn_rcpf(1.f + exp2_(x2));
      d = 4.f * fmaf(-q, q, q);
      return fmaf(-2.f * top, q, top);
    };
    bool any_large = true;
    if constexpr (MODE != QUICK && !BOTH_WAYS) {
      float most = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
      any_large = __any(most * k >= SMALL);
    }
    if constexpr (MODE == QUICK) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float d;
        s[r] = large(s[r] * (2.f * LOG2E * k), d);
        if constexpr (SLOPE) slope[r] = d;
      }
    } else if (any_large) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float d, dl;
        const float x = s[r] * k, v = small(s[r], x, d), vl = large(2.f * LOG2E * x, dl);
        const bool beyond = fabsf(x) >= SMALL;
        s[r] = beyond ? vl : v;
        if constexpr (SLOPE) slope[r] = beyond ? dl : d;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float d;
        s[r] = small(s[r], s[r] * k, d);
        if constexpr (SLOPE) slope[r] = d;
      }
    }
    if constexpr (has_bias(MODE)) {
      phase();
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] += at(r);
    }
  } else if constexpr (has_bias(MODE)) {
    const float c1 = a.scale * LOG2E;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = s[r] * c1 + at(r);
  }
}

// A bias in units of log 2.  The lowest and highest values of fp32 stay finite: a row that holds
// nothing else keeps its softmax of equal scores.
XP_DEV float log2_bias(float v) {
  const float most = 3.402823466e38f, u = v * LOG2E;
  return fabsf(v) <= most ? fminf(fmaxf(u, -most), most) : u;
}

// A head's bias around a tile: WIDTH distances from `low` on, a step ahead like the tiles, in
// LDS (reads from memory among the products would wait for the tiles in flight as well).
template <int WIDTH>
struct BiasWindow {
  static_assert(WIDTH <= 256, "one each thread");
  float reg;
  XP_DEV void load(const AttnArgs& a, int head, int low) {
    if (threadIdx.x < WIDTH)
      reg = a.bias[(int64_t)head * (2 * a.range + 1) + a.range + min(max(low + (int)threadIdx.x, -a.range), a.range)];
  }
  XP_DEV void store(float* sh) const {
    if (threadIdx.x < WIDTH) sh[threadIdx.x] = log2_bias(reg);
  }
};

// ---------------------------------------------------------------- forward
// The largest score with those of n blocks, and everything so far multiplied if it has grown by more than 8
// (base 2) since it last entered the exponentials: P is at most 2^8 then, the sums stay in
// fp32's range, and the results are rarely multiplied.
template <int DP, int MODE>
XP_DEV void softmax_step(const f32x16_t* s, int n, float& m, float& base, float& l, f32x16_t (&acc)[DP / 32], float c1) {
  float top = s[0][0];
  for (int i = 0; i < n; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
  m = fmaxf(m, both_max(top));
  if (__any(log2_of<MODE>(m - base, c1) > 8.f)) {  // (from -inf on: infinite; while there is no key: NaN)
    const float keep = m == NEG_INF ? 1.f : exp2_(log2_of<MODE>(base - m, c1));
    base = m;
    l *= keep;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] *= keep;
  }
}

// A lane's query row at the end: o and the statistics, or (part >= 0) one part of them.
template <typename T, int DP, int MODE>
XP_DEV void write_rows(const AttnArgs& a, int b, int head, int i, int64_t part, int kend, float m, float base, float l, f32x16_t (&acc)[DP / 32]) {
  const float c1 = a.scale * LOG2E;
  const bool low = (threadIdx.x & 63) < 32;
  // (a NaN among the scores leaves l NaN, and the row NaN)
  const float sum = both_sum(l);
  const bool none = kend == 0 || sum == 0.f;
  const float fit = exp2_(log2_of<MODE>(base - m, c1));  // (o and l belong to `base`)
  const float ms = none ? NEG_INF : log2_of<MODE>(m, c1), ls = none ? 0.f : sum * fit;
  if (part >= 0) {  // (a sum of zero leaves the part of o unwritten)
    if (low) {
      a.part_ml[2 * part] = ms;
      a.part_ml[2 * part + 1] = ls;
    }
    st_column<float, DP>(a.part_o + part * DP, none ? 0 : DP, acc, fit);
    return;
  }
  if (a.stats && low) {
    float* st = a.stats + 2 * (((int64_t)b * a.heads + head) * a.nq + i);
    st[0] = ms;
    st[1] = ls;
  }
  if (none)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  st_column<T, DP>((T*)a.o.p + b * a.o.b + (int64_t)i * a.o.t + head * a.o.h, a.dim, acc, none ? 0.f : 1.f / sum);
}

// One workgroup per 128 query rows of a head, and part of the keys.
// Bound by the matrix units and the vector instructions, 512 cycles and some 690 for a block of 32 x 32 of dim 128 (125
// instructions, 16 of them exponentials): a SIMD's waves (two; three for bf16 rows of 64 but with both cap and bias) hardly
// overlap them.  bf16, dim 128: 16 heads of 8192 tokens 564 us (975 Tflop/s), causal 307 us (895); capped and causal
// 371 us; 2 x 4096 tokens, 16 heads over 4 291 us (945), with a prefix 201 us.  dim 64: 2 x 8192 tokens, 16 heads 657 us (835),
// causal 359.  fp32, dim 128: 8 heads of 2048 tokens, causal 141 us.  No LDS bank conflicts.  Causal and prefix masks:
// an XCD takes one head after another, each from its longest block, so the last head's longest blocks start late.
template <typename T, int DP, int MODE>
__global__ __launch_bounds__(256, (WAVES<T, DP>)) void k_attn_fwd(AttnArgs a) {
  constexpr int KEYS = BN<T>, NB = KEYS / 32;
  constexpr int TILE = KEYS * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE];  // keys, values, twice
  __shared__ float sbias[2][has_bias(MODE) ? ROWS + KEYS : 1];
  __shared__ int sdoc[2][KEYS];
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (a.nq + ROWS - 1) / ROWS;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int split = id % a.splits;
  id /= a.splits;
  const int blk = blocks - 1 - id % blocks;  // (causal: the longest first)
  id /= blocks;
  const int head = id % a.heads, b = id / a.heads;
  const int kvh = head / (a.heads / a.kv_heads);
  const Seq seq(a, b);

  // limits of the workgroup's and the wave's rows (of those that count)
  const int last = min((blk + 1) * ROWS, min(a.nq, seq.ql)) - 1, first = blk * ROWS;
  const int kmax = first <= last ? seq.kend(last) : 0;
  const int wfirst = first + wave * 32, wlast = min(wfirst + 31, last);
  const int wmax = wfirst <= wlast ? seq.kend(wlast) : 0, wmin = wfirst <= wlast ? seq.kend(wfirst) : 0;

  const int i = wfirst + (lane & 31);
  const bool in = i < a.nq, live = in && i < seq.ql;
  const int doc = a.q_doc ? (live ? a.q_doc[(int64_t)b * a.nq + i] : -1) : 0;
  const int kend = live && doc >= 0 ? seq.kend(i) : 0;
  u32x4_t q[DP / CHUNK<T> / 2];
  ld_column<T, DP>((const T*)a.q.p + b * a.q.b + (int64_t)i * a.q.t + head * a.q.h, live, a.ldim, q);
  DocRange docs = {0, 0, 0, 0};
  if (a.q_doc) docs = doc_range(doc, sh);
  const T* kp = (const T*)a.k.p + b * a.k.b + kvh * a.k.h;
  const T* vp = (const T*)a.v.p + b * a.v.b + kvh * a.v.h;
  const int32_t* kdoc = a.k_doc ? a.k_doc + (int64_t)b * a.nk : nullptr;

  const int tiles = (kmax + KEYS - 1) / KEYS, per = (tiles + a.splits - 1) / a.splits;
  const int tab_tiles = (a.nk + KEYS - 1) / KEYS;
  Walk walk(a.k_tab ? a.k_tab + (int64_t)b * tab_tiles : nullptr, min(tiles, (split + 1) * per), docs.lo, docs.hi);

  // m: the largest score so far, base: the one in the exponentials; l: this lane's part of the sum
  const float c1 = a.scale * LOG2E;
  float m = NEG_INF, base = NEG_INF, l = 0.f;
  f32x16_t acc[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;

  Stager<T, DP, KEYS> ks(a.k.t, a.ldim), vs(a.v.t, a.ldim);
  BiasWindow<ROWS + KEYS> window;
  const int low = -(first + ROWS - 1) - seq.off;  // the window's smallest distance, of tile 0
  int dreg = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = t * KEYS;
    const int32_t* pad = kdoc && walk.tab[t].w ? kdoc + j0 : nullptr;
    ks.load(kp + (int64_t)j0 * a.k.t, seq.kl - j0, pad);
    vs.load(vp + (int64_t)j0 * a.v.t, seq.kl - j0, pad);
    if constexpr (has_bias(MODE)) window.load(a, head, low + j0);
    if (kdoc && threadIdx.x < KEYS) dreg = j0 + (int)threadIdx.x < seq.kl ? kdoc[j0 + threadIdx.x] : -1;
  };
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  auto store = [&](int buf) __attribute__((always_inline)) {
    ks.store(tile0 + buf * 2 * TILE);
    vs.store(tile0 + buf * 2 * TILE + TILE);
    if constexpr (has_bias(MODE)) window.store(sbias[buf]);
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
      f32x16_t s[NB];
      // (the other wave of the SIMD has its exponentials then)
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int n = 0; n < NB; ++n) s[n] = rows_times<T, DP>(rat, n * 32 * ROW<T, DP>, q, a.ldim);
      __builtin_amdgcn_s_setprio(0);
      if constexpr (MODE != PLAIN) {
        float none[16];
        const float* mine = sbias[buf] + ROWS - 1 - (i - first) + 4 * (lane >> 5);
#pragma unroll
        for (int n = 0; n < NB; ++n)
          scores<MODE, false, sizeof(T) == 4>(s[n], a, none, [&](int r) { return mine[n * 32 + 8 * (r >> 2) + (r & 3)]; });
      }
      if ((t + 1) * KEYS > wmin)
#pragma unroll
        for (int n = 0; n < NB; ++n) hide_from(s[n], kend - t * KEYS - n * 32, NEG_INF);
      if (mixed)
#pragma unroll
        for (int n = 0; n < NB; ++n) hide_others(s[n], sdoc[buf] + n * 32, doc, NEG_INF);
      softmax_step<DP, MODE>(s, NB, m, base, l, acc, c1);
      const float off = base == NEG_INF ? 0.f : base;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = exp_of<MODE>(s[n][r], off, c1);
          l += p[r];
        }
        add_transposed<T, DP>(acc, cat, TILE + n * 32 * ROW<T, DP>, p, a.ldim);
      }
    }
    buf ^= 1;
    if (tn < walk.end) store(buf);
    t = tn;
  }

  if (in) {
    const int64_t row = ((int64_t)b * a.heads + head) * a.nq + i, rows = (int64_t)a.batch * a.heads * a.nq;
    write_rows<T, DP, MODE>(a, b, head, i, a.splits > 1 ? split * rows + row : -1, kend, m, base, l, acc);
  }
}

// The workgroups of k_attn_few that a sequence gets, of `groups` for each block of rows and key
// head: one each, and the others by the sequences' lengths, so that the longest does not decide the
// call's time (up to 64 sequences; more of them even out by their number).  Without lengths equal shares, and the last
// sequence has what is left over.
struct Share {
  int b, first, end;  // the sequence, its workgroups
};
XP_DEV Share share_at(const AttnArgs& a, int group, int seq) {  // the one that `group` is in, or (group < 0) that of sequence seq
  const int groups = a.splits, lane = threadIdx.x & 63;
  if (a.batch > 64 || !a.k_len) {
    const int per = groups / a.batch, b = group < 0 ? seq : min(group / per, a.batch - 1);
    return {b, b * per, b == a.batch - 1 ? groups : (b + 1) * per};
  }
  const int steps = lane < a.batch ? (min(max(a.k_len[lane], 0), a.nk) + 31) / 32 : 0;
  int before = steps;
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(before, o, 64);
    before += lane >= o ? v : 0;
  }
  const int total = __shfl(before, 63, 64);
  before -= steps;
  const int c = lane < a.batch ? lane + (total > 0 ? (int)((int64_t)before * (groups - a.batch) / total) : 0) : groups;
  const int b = group < 0 ? seq : __popcll(__ballot(c <= group)) - 1;
  return {b, __shfl(c, b, 64), b + 1 < a.batch ? __shfl(c, b + 1, 64) : groups};
}

// where a wave's part of a row lies
XP_DEV int64_t few_part(const AttnArgs& a, int kvh, int blk, int wave, int row) {
  const int blocks = (a.nq * a.pk + 31) / 32;
  return (((int64_t)kvh * blocks + blk) * (a.splits * 4) + wave) * 32 + row;
}

// Few query rows (a generation step): a wave takes up to 32 rows of the heads that share keys
// together, row r being query r / pk of head r % pk, and a part of the keys by itself, 32 at a
// time through LDS of its own, the next 32 on their way: four times the bytes in flight
// that the workgroups of k_attn_fwd have, whose other waves would have no rows.  Short
// sequences (splits 0): all of the keys, four waves being four blocks of rows.
// Bound by the keys' and values' bytes (5.2 TB/s, what a copy reaches), so P is two bf16 values: 8 sequences of up to 32768
// tokens, 8 heads of 128, 151.4 us for 150.0, and o 1.66e-3 of its 2-norm off, which is its own rounding, for 2.3e-3.
template <typename T, int DP, int MODE>
__global__ __launch_bounds__(256, (WAVES<T, DP>)) void k_attn_few(AttnArgs a) {
  constexpr int TILE = 32 * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * 2 * TILE];  // of each wave: keys, values
  __shared__ int sdoc[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = a.nq * a.pk, blocks = (rows + 31) / 32, units = a.kv_heads;
  // (nothing is read twice: neighbours, the heads of the same keys, go to different XCDs, and so
  // do the parts of one sequence)
  int id = a.splits > 0 ? blockIdx.x : blockIdx.x * 4 + wave;
  const int kvh = id % units;
  id /= units;
  const int blk = id % blocks, group = id / blocks;
  if (a.splits == 0 && group >= a.batch) return;
  Share share = {group, 0, 0};
  if (a.splits > 0) share = share_at(a, group, 0);
  const int b = __builtin_amdgcn_readfirstlane(share.b);
  const int parts = a.splits > 0 ? (share.end - share.first) * 4 : 1, split = a.splits > 0 ? (group - share.first) * 4 + wave : 0;
  const Seq seq(a, b);

  const int first = blk * 32 / a.pk, last = min((min(rows, (blk + 1) * 32) - 1) / a.pk, seq.ql - 1);
  const int kmax = first <= last ? seq.kend(last) : 0, kmin = first <= last ? seq.kend(first) : 0;
  const int row = blk * 32 + (lane & 31), i = row / a.pk, head = kvh * a.pk + row % a.pk;
  const bool in = row < rows, live = in && i < seq.ql;
  const int doc = a.q_doc ? (live ? a.q_doc[(int64_t)b * a.nq + i] : -1) : 0;
  const int kend = live && doc >= 0 ? seq.kend(i) : 0;
  u32x4_t q[DP / CHUNK<T> / 2];
  ld_column<T, DP>((const T*)a.q.p + b * a.q.b + (int64_t)i * a.q.t + head * a.q.h, live, a.ldim, q);
  const T* kp = (const T*)a.k.p + b * a.k.b + kvh * a.k.h;
  const T* vp = (const T*)a.v.p + b * a.v.b + kvh * a.v.h;
  const int32_t* kdoc = a.k_doc ? a.k_doc + (int64_t)b * a.nk : nullptr;
  const float* bias = has_bias(MODE) ? a.bias + (int64_t)min(head, a.heads - 1) * (2 * a.range + 1) + a.range : nullptr;

  // (documents: every step is looked at, their tiles have no table here)
  const int steps = (kmax + 31) / 32, per = (steps + parts - 1) / parts;
  const int end = min(steps, (split + 1) * per);
  const float c1 = a.scale * LOG2E;
  float m = NEG_INF, base = NEG_INF, l = 0.f;
  f32x16_t acc[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;

  Stager<T, DP, 32, 64> ks(a.k.t, a.ldim), vs(a.v.t, a.ldim);
  int dreg = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = t * 32;
    ks.load(kp + (int64_t)j0 * a.k.t, seq.kl - j0, kdoc ? kdoc + j0 : nullptr);
    vs.load(vp + (int64_t)j0 * a.v.t, seq.kl - j0, kdoc ? kdoc + j0 : nullptr);
    if (kdoc) dreg = lane < 32 && j0 + lane < seq.kl ? kdoc[j0 + lane] : -1;
  };
  const uint32_t tile = lds_address(tiles_) + wave * 2 * TILE, rplace = row_place<T, DP>() + tile, cplace = column_place<T, DP>() + tile;
  int t = min(steps, split * per);
  if (t < end) load(t);
  for (; t < end; ++t) {
    ks.store(tile);
    vs.store(tile + TILE);
    if (kdoc && lane < 32) sdoc[wave][lane] = dreg;
    wave_fence();
    const int next = t + 1;
    if (next < end) load(next);
    const int j0 = t * 32;
    f32x16_t s = rows_times<T, DP>(rplace, 0, q, a.ldim);
    if constexpr (MODE != PLAIN) {
      float none[16];
      const int d0 = j0 - i - seq.off;
      scores<MODE, false, true>(s, a, none, [&](int r) { return log2_bias(bias[min(max(d0 + row_of(r), -a.range), a.range)]); });
    }
    if (j0 + 32 > kmin || blk == blocks - 1) hide_from(s, kend - j0, NEG_INF);
    if (kdoc) hide_others(s, sdoc[wave], doc, NEG_INF);
    float p[16];
    softmax_step<DP, MODE>(&s, 1, m, base, l, acc, c1);
    const float off = base == NEG_INF ? 0.f : base;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = exp_of<MODE>(s[r], off, c1);
      l += p[r];
    }
    add_transposed<T, DP, true>(acc, cplace, TILE, p, a.ldim);
    wave_fence();
  }
  if (in) write_rows<T, DP, MODE>(a, b, head, i, a.splits > 0 ? few_part(a, kvh, blk, group * 4 + wave, lane & 31) : -1, kend, m, base, l, acc);
}

// The parts of the keys joined: one workgroup per query row; for the sums a lane takes every 64th
// part, for o a wave every fourth.  Bound by the launch and the latency of two reads, one after the
// other (256 rows of 128 columns, 32 parts each on average: 8 us).
template <typename T, int DP, bool FEW>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  __shared__ float sh[4][128];
  constexpr int N = (DP + 63) / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq, r = blockIdx.x;
  const int i = (int)(r % a.nq), head = (int)(r / a.nq % a.heads), b = (int)(r / a.nq / a.heads);
  int64_t first = r, step = rows;
  int parts = a.splits;
  if constexpr (FEW) {
    const Share share = share_at(a, -1, b);
    const int row = i * a.pk + head % a.pk;
    first = few_part(a, head / a.pk, row / 32, share.first * 4, row % 32);
    step = 32;
    parts = (share.end - share.first) * 4;
  }
  const f32x2_t* ml = (const f32x2_t*)a.part_ml;
  const f32x2_t mine = lane < parts ? ml[first + lane * step] : (f32x2_t){NEG_INF, 0.f};  // (most calls have no more)
  float m = mine[0];
  for (int p = lane + 64; p < parts; p += 64) m = fmaxf(m, ml[first + p * step][0]);
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  float l = 0.f, o[N];
#pragma unroll
  for (int d = 0; d < N; ++d) o[d] = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int p = p0 + lane;
    const f32x2_t v = p0 == 0 ? mine : p < parts ? ml[first + p * step] : (f32x2_t){NEG_INF, 0.f};
    const float lp = v[1], w = lp == 0.f ? 0.f : exp2_(v[0] - m);
    l += lp * w;
    const int n = min(64, parts - p0);
#pragma unroll 8
    for (int k = wave; k < n; k += 4) {  // (a part whose sum is zero was not written; of one that is NaN, l is)
      const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), k));
#pragma unroll
      for (int d = 0; d < N; ++d) {
        const float v = d * 64 + lane < DP ? a.part_o[(first + (p0 + k) * step) * DP + d * 64 + lane] : 0.f;
        o[d] += wk > 0.f ? wk * v : 0.f;
      }
    }
  }
  for (int k = 32; k > 0; k >>= 1) l += __shfl_xor(l, k, 64);
#pragma unroll
  for (int d = 0; d < N; ++d) sh[wave][d * 64 + lane] = o[d];
  __syncthreads();
  if (a.stats && threadIdx.x == 0) {
    a.stats[2 * r] = m;
    a.stats[2 * r + 1] = l;
  }
  if ((int)threadIdx.x < a.dim) {
    const int d = threadIdx.x;
    const float v = (sh[0][d] + sh[1][d]) + (sh[2][d] + sh[3][d]);
    std_((T*)a.o.p + b * a.o.b + (int64_t)i * a.o.t + head * a.o.h + d, (double)(l == 0.f ? 0.f : v / l));
  }
}

// ---------------------------------------------------------------- statistics of a row
// P = exp2(score - row.a), where row.a has the sum's logarithm in it; BIAS (whose scores may be so
// large that it would be lost there): exp2(score - row.a - row.b).  A row without keys gives 0.
struct RowStat { float a, b; };
template <int MODE>
XP_DEV RowStat row_stat(float m, float l) {
  if (l == 0.f) return {__builtin_inff(), 0.f};
  const float log2l = __builtin_amdgcn_logf(l);
  if constexpr (has_bias(MODE)) return {m, log2l};
  else return {m + log2l, 0.f};
}
template <int MODE>
XP_DEV float weight(float s, float a, float b, float c1) {
  if constexpr (MODE == PLAIN) return exp2_(s * c1 - a);
  else if constexpr (!has_bias(MODE)) return exp2_(s - a);
  else return exp2_((s - a) - b);
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
// TWICE: dX as two bf16 values.  Three roundings reach dq in bf16 storage: its own, dX's, and o's, which the
// sum over n keys of like weight leaves at 1 / sqrt(n) of itself.  Over many keys dq is
// 2.4e-3 of its 2-norm off (its own rounding alone: 1.7e-3); over few it would be 2.6e-3 to
// 2.8e-3, and is 2.3e-3 without dX's (2 x 4096 tokens, 12 heads of 64, documents of 32 to 2048: 100 us for 90).
// Few rows: the keys in `splits` parts, whose sums k_attn_dq_join adds.
// Bound as the forward is, with three products a block.
// 2 sequences of 4096 tokens, 16 heads of 128 over 4, prefix: 332 us; matrix units busy for 30 % of it.
template <typename T, int DP, int MODE, bool TWICE>
__global__ __launch_bounds__(256, (WAVES<T, DP>)) void k_attn_dq(AttnArgs a) {
  constexpr int KEYS = BN_DQ<T, DP>, NB = KEYS / 32;
  constexpr int TILE = KEYS * ROW<T, DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE];  // keys, values, twice
  __shared__ float sbias[2][has_bias(MODE) ? ROWS + KEYS : 1];
  __shared__ int sdoc[2][KEYS];
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (a.nq + ROWS - 1) / ROWS;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int split = id % a.splits;
  id /= a.splits;
  const int blk = blocks - 1 - id % blocks;
  id /= blocks;
  const int head = id % a.heads, b = id / a.heads;
  const int kvh = head / (a.heads / a.kv_heads);
  const Seq seq(a, b);

  const int i = blk * ROWS + wave * 32 + (lane & 31);
  const bool in = i < a.nq, live = in && i < seq.ql;
  const int doc = a.q_doc ? (live ? a.q_doc[(int64_t)b * a.nq + i] : -1) : 0;
  const int kend = live && doc >= 0 ? seq.kend(i) : 0;
  const int last = min((blk + 1) * ROWS, min(a.nq, seq.ql)) - 1, first = blk * ROWS;
  const int kmax = first <= last ? seq.kend(last) : 0;
  const int wfirst = first + wave * 32, wlast = min(wfirst + 31, last);
  const int wmax = wfirst <= wlast ? seq.kend(wlast) : 0, wmin = wfirst <= wlast ? seq.kend(wfirst) : 0;
  DocRange docs = {0, 0, 0, 0};
  if (a.q_doc) docs = doc_range(doc, sh);

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
    st = row_stat<MODE>(a.stats[2 * srow], a.stats[2 * srow + 1]);
  }
  delta = both_sum(delta);
  float exact = 0.f;

  const T* kp = (const T*)a.k.p + b * a.k.b + kvh * a.k.h;
  const T* vp = (const T*)a.v.p + b * a.v.b + kvh * a.v.h;
  const int32_t* kdoc = a.k_doc ? a.k_doc + (int64_t)b * a.nk : nullptr;

  const int tiles = (kmax + KEYS - 1) / KEYS, per = (tiles + a.splits - 1) / a.splits;
  const int tab_tiles = (a.nk + KEYS - 1) / KEYS;
  Walk walk(a.k_tab ? a.k_tab + (int64_t)b * tab_tiles : nullptr, min(tiles, (split + 1) * per), docs.lo, docs.hi);
  const float c1 = a.scale * LOG2E;
  f32x16_t acc[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;

  Stager<T, DP, KEYS> ks(a.k.t, a.ldim), vs(a.v.t, a.ldim);
  BiasWindow<ROWS + KEYS> window;
  const int low = -(first + ROWS - 1) - seq.off;  // the window's smallest distance, of tile 0
  int dreg = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int j0 = t * KEYS;
    const int32_t* pad = kdoc && walk.tab[t].w ? kdoc + j0 : nullptr;
    ks.load(kp + (int64_t)j0 * a.k.t, seq.kl - j0, pad);
    vs.load(vp + (int64_t)j0 * a.v.t, seq.kl - j0, pad);
    if constexpr (has_bias(MODE)) window.load(a, head, low + j0);
    if (kdoc && threadIdx.x < KEYS) dreg = j0 + (int)threadIdx.x < seq.kl ? kdoc[j0 + threadIdx.x] : -1;
  };
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  auto store = [&](int buf) __attribute__((always_inline)) {
    ks.store(tile0 + buf * 2 * TILE);
    vs.store(tile0 + buf * 2 * TILE + TILE);
    if constexpr (has_bias(MODE)) window.store(sbias[buf]);
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
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int k0 = t * KEYS + n * 32;
        f32x16_t s = rows_times<T, DP>(rat, n * 32 * ROW<T, DP>, q, a.ldim);
        phase();
        const f32x16_t dp = rows_times<T, DP>(rat, TILE + n * 32 * ROW<T, DP>, g, a.ldim);
        phase();
        float slope[16], ds[16];
        if constexpr (MODE != PLAIN) {
          const float* mine = sbias[buf] + ROWS - 1 - (wave * 32 + (lane & 31)) + 4 * (lane >> 5) + n * 32;
          scores<MODE, true, false>(s, a, slope, [&](int r) { return mine[8 * (r >> 2) + (r & 3)]; });
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = weight<MODE>(s[r], st.a, st.b, c1);
        if (k0 + 32 > wmin) hide_from(ds, kend - k0, 0.f);
        if (mixed) hide_others(ds, sdoc[buf] + n * 32, doc, 0.f);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          exact += ds[r] * dp[r];
          ds[r] *= dp[r] - delta;
        }
        if constexpr (has_cap(MODE)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] *= slope[r];
        }
        phase();
        add_transposed<T, DP, TWICE>(acc, cat, n * 32 * ROW<T, DP>, ds, a.ldim);
        phase();
      }
    }
    buf ^= 1;
    if (tn < walk.end) store(buf);
    t = tn;
  }
  exact = both_sum(exact);
  if (lane < 32 && split == 0) {
    float* row = a.rows + (((int64_t)b * a.heads + head) * (blocks * 4) + blk * 4 + wave) * ROW_INFO + lane;
    row[0] = st.a;
    row[32] = st.b;
    row[64] = a.splits > 1 ? 0.f : exact;
    row[96] = __int_as_float(kend);
    row[128] = __int_as_float(doc);
  }
  if (!in) return;
  if (a.splits > 1) {
    const int64_t at = split * ((int64_t)a.batch * a.heads * a.nq) + srow;
    st_column<float, DP>(a.part_o + at * DP, DP, acc, a.scale);
    if (lane < 32) a.part_ml[at] = exact;
  } else {
    st_column<T, DP>((T*)a.dq.p + b * a.dq.b + (int64_t)i * a.dq.t + head * a.dq.h, a.dim, acc, a.scale);
  }
}

// The parts' sums of dq, and of P dP for k_attn_dkv, added in their order: four columns a thread.
// Bound by the launch: few rows.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_dq_join(AttnArgs a) {
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq, x = (int64_t)blockIdx.x * 256 + threadIdx.x, r = x / (DP / 4);
  if (r >= rows) return;
  const int d = (int)(x % (DP / 4)) * 4;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, exact = 0.f;
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part_o + (p * rows + r) * DP + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += v[i];
    if (d == 0) exact += a.part_ml[p * rows + r];
  }
  const int i = (int)(r % a.nq), head = (int)(r / a.nq % a.heads), b = (int)(r / a.nq / a.heads), blocks = (a.nq + ROWS - 1) / ROWS;
  T* to = (T*)a.dq.p + b * a.dq.b + (int64_t)i * a.dq.t + head * a.dq.h + d;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (d + k < a.dim) std_(to + k, (double)s[k]);
  if (d == 0) a.rows[(((int64_t)b * a.heads + head) * (blocks * 4) + i / 32) * ROW_INFO + 64 + i % 32] = exact;
}

// grad_bias[head][x] += the sum over sequences and key blocks of the blocks' diagonals at
// that distance: a workgroup takes 64 distances of a head, its 16 waves every 16th (sequence, 32 keys).
// Bound by the latency of those reads, few and scattered (2 x 4096 keys, 12 heads, range 128: 15 us; 64 us with one
// wave a distance group).
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
        if (x < width)
          for (int q = 0; q < a.q_parts; ++q) v0 += a.tail[2 * (at * a.q_parts + q) + (x == 0 ? 0 : 1)];
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
//
// A launch may be cut over the heads that share keys and over the queries (few keys would not
// fill the card): each part then leaves its sums in fp32, which k_attn_dkv_join adds.
// bf16 rows of 128: the values' columns stay in LDS, for 32 registers less.
//
// Bound as the forward is, with four products a block, two of whose operands come out of registers.  2 sequences of 4096
// tokens, 16 heads of 128 over 4, prefix: 386 us and the join 23 us; matrix units busy for 35 % of it, no LDS bank
// conflicts.  The backward as a whole: 16 heads of 8192 tokens 2.0 ms (680 Tflop/s).
template <typename T, int DP, int MODE, int WHAT>
__global__ __launch_bounds__(256, (WAVES<T, DP>)) void k_attn_dkv(AttnArgs a) {
  constexpr int QT = QT_<T, DP>, TILE = QT * ROW<T, DP>;
  constexpr bool V_LDS = sizeof(T) == 2 && DP == 128;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_[4 * TILE + (V_LDS ? ROWS * ROW<T, DP> : 0)];  // q, dout, twice; values
  __shared__ float sbias[2][has_bias(MODE) ? ROWS + QT : 1];
  __shared__ float srow[2][5 * QT];  // five values of 32 queries, then of the next 32
  __shared__ int sh[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (a.nk + ROWS - 1) / ROWS, group = a.heads / a.kv_heads;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int parts = a.head_parts * a.q_parts, part = id % parts;
  id /= parts;
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
    docs = doc_range(doc, sh);
    pad = __any(doc < 0);
  }
  const uint32_t tile0 = lds_address(tiles_), rplace = row_place<T, DP>() + tile0, cplace = column_place<T, DP>() + tile0;
  const uint32_t vplace = rplace + 4 * TILE + wave * 32 * ROW<T, DP>;
  u32x4_t kc[DP / CHUNK<T> / 2], vc[V_LDS ? 1 : DP / CHUNK<T> / 2];
  const bool use = j < seq.kl && doc >= 0;
  ld_column<T, DP>((const T*)a.k.p + b * a.k.b + (int64_t)j * a.k.t + kvh * a.k.h, use, a.ldim, kc);
  if constexpr (V_LDS) {
    Stager<T, DP, ROWS> all(a.v.t, a.ldim);
    all.load((const T*)a.v.p + b * a.v.b + kvh * a.v.h + k0 * a.v.t, seq.kl - k0, a.k_doc ? a.k_doc + (int64_t)b * a.nk + k0 : nullptr);
    all.store(tile0 + 4 * TILE);
  } else if constexpr (WHAT & 2)
    ld_column<T, DP>((const T*)a.v.p + b * a.v.b + (int64_t)j * a.v.t + kvh * a.v.h, use, a.ldim, vc);
  const int32_t* qdoc = a.q_doc ? a.q_doc + (int64_t)b * a.nq : nullptr;

  // queries that see a key of the workgroup: those with kend > k0, from the first such on
  int tiles = (seq.ql + QT - 1) / QT, t0 = 0;
  if (k0 >= seq.kl) tiles = 0;
  else if (seq.causal && seq.prefix <= k0) t0 = min(tiles, max(0, k0 - seq.off) / QT);
  const int h0 = kvh * group + part % a.head_parts * (group / a.head_parts), h1 = h0 + group / a.head_parts;
  const int per = (tiles - t0 + a.q_parts - 1) / a.q_parts;
  t0 = t0 + part / a.head_parts * per;
  tiles = min(tiles, t0 + per);
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

  const bool diag = has_bias(MODE) && (WHAT & 2) && a.grad_bias;
  float left = 0.f, right = 0.f;
  const int near0 = first_near(a, seq, kw);
  const int64_t wblock = blk * 4 + wave, wblocks = blocks * 4;
  const int q_part = part / a.head_parts;
  if (diag) {  // zeros for blocks that no step reaches: this part's, and what lies before the first's and behind the last's
    const int n0 = q_part == 0 ? 0 : max(0, t0 * (QT / 32) - near0);
    const int n1 = q_part == a.q_parts - 1 ? a.near : min(a.near, (t0 + per) * (QT / 32) - near0);
    for (int h = h0; h < h1; ++h) {
      const int64_t w = ((int64_t)b * a.heads + h) * wblocks + wblock;
      for (int n = n0; n < n1; ++n) a.diag[(w * a.near + n) * 64 + lane] = 0.f;
      if (lane == 0) {  // (the lane that writes them again at the head's end)
        a.tail[2 * (w * a.q_parts + q_part)] = 0.f;
        a.tail[2 * (w * a.q_parts + q_part) + 1] = 0.f;
      }
    }
  }

  Stager<T, DP, QT> qs(a.q.t, a.ldim), gs(a.dout.t, a.ldim);
  const int row_tiles = (a.nq + ROWS - 1) / ROWS * 4;
  BiasWindow<ROWS + QT> window;
  const int low = k0 - (QT - 1) - seq.off;  // the window's smallest distance, of tile 0
  float rreg[QT / 32];
  auto load = [&](int t, int head) __attribute__((always_inline)) {
    const int i0 = t * QT;
    const int32_t* pads = qdoc && walk.tab[t].w ? qdoc + i0 : nullptr;
    qs.load((const T*)a.q.p + b * a.q.b + head * a.q.h + i0 * a.q.t, seq.ql - i0, pads);
    gs.load((const T*)a.dout.p + b * a.dout.b + head * a.dout.h + i0 * a.dout.t, seq.ql - i0, pads);
    if constexpr (has_bias(MODE)) window.load(a, head, low - i0);
    if (threadIdx.x < 5 * 32)
#pragma unroll
      for (int n = 0; n < QT / 32; ++n) rreg[n] = a.rows[(((int64_t)b * a.heads + head) * row_tiles + t * (QT / 32) + n) * ROW_INFO + threadIdx.x];
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
    qs.store(tile0 + buf * 2 * TILE);
    gs.store(tile0 + buf * 2 * TILE + TILE);
    if constexpr (has_bias(MODE)) window.store(sbias[buf]);
    if (threadIdx.x < 5 * 32)
#pragma unroll
      for (int n = 0; n < QT / 32; ++n) srow[buf][n * 5 * 32 + threadIdx.x] = rreg[n];
  };
  int head = h0, t = walk.next(t0), buf = 0;
  const int t_first = t;
  const bool any = t < walk.end;
  if (any) {
    load(t, h0);
    store(0);
  }
  while (any && head < h1) {
    int tn = walk.next(t + 1), hn = head;
    if (tn >= walk.end) {
      tn = t_first;
      ++hn;
    }
    if (hn < h1) load(tn, hn);
    __syncthreads();
    bool mixed = false, other = false;
    if (qdoc) {
      const int4 e = walk.tab[t];
      other = e.x > docs.whi || e.y < docs.wlo;
      mixed = e.z || pad || docs.wlo != docs.whi;
    }
    // (a function called for each block: an unrolled loop of one round leaves more values in registers)
    auto block = [&](int n) __attribute__((always_inline)) {
      const int i0 = t * QT + n * 32, i1 = min(i0 + 32, seq.ql) - 1;
      if (other || i0 >= seq.ql || seq.kend(i1) <= kw) return;
      const uint32_t rat = rplace + buf * 2 * TILE, cat = cplace + buf * 2 * TILE;
      f32x16_t s = rows_times<T, DP>(rat, n * 32 * ROW<T, DP>, kc, a.ldim);
      phase();
      float p[16], slope[16];
      if constexpr (MODE != PLAIN) {  // (register r's place in the window: key - query + QT - 1)
        const float* mine = sbias[buf] + (has_bias(MODE) ? (j - k0) + QT - 28 - 4 * (lane >> 5) - n * 32 : 0);
        scores<MODE, (WHAT & 2) != 0, false>(s, a, slope, [&](int r) { return mine[27 - 8 * (r >> 2) - (r & 3)]; });
      }
      auto of = [&](int what, int r) __attribute__((always_inline)) { return srow[buf][n * (5 * 32) + what * 32 + row_of(r)]; };
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = weight<MODE>(s[r], of(0, r), has_bias(MODE) ? of(1, r) : 0.f, c1);
      if (i0 + 32 > seq.ql || seq.kend(i0) < kw + 32)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = j >= __float_as_int(of(3, r)) ? 0.f : p[r];
      if (mixed)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __float_as_int(of(4, r)) != doc ? 0.f : p[r];
      if constexpr (WHAT & 1) {
        phase();
        add_transposed<T, DP>(dv, cat, TILE + n * 32 * ROW<T, DP>, p, a.ldim);
        phase();
      }
      if constexpr (WHAT & 2) {
        f32x16_t dp;
        if constexpr (V_LDS) dp = rows_times<T, DP>(rat, TILE + n * 32 * ROW<T, DP>, (uint32_t)fresh(vplace));
        else dp = rows_times<T, DP>(rat, TILE + n * 32 * ROW<T, DP>, vc, a.ldim);
        phase();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] *= dp[r] - of(2, r);
          if (DP == 128 && r % 4 == 3) phase();
        }
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
            a.diag[(w * a.near + ((i0 >> 5) - near0)) * 64 + lane] = outer ? 0.f : lo;
          }
        }
        if constexpr (has_cap(MODE)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] *= slope[r];
        }
        phase();
        add_transposed<T, DP>(dk, cat, n * 32 * ROW<T, DP>, p, a.ldim);
      }
    };
    block(0);
    if constexpr (QT == 64) block(1);
    if (diag && hn != head) {  // the head's last step
      for (int o = 32; o > 0; o >>= 1) {
        left += __shfl_xor(left, o, 64);
        right += __shfl_xor(right, o, 64);
      }
      if (lane == 0) {
        float* w = a.tail + 2 * ((((int64_t)b * a.heads + head) * wblocks + wblock) * a.q_parts + q_part);
        w[0] = left;
        w[1] = right;
      }
      left = right = 0.f;
    }
    buf ^= 1;
    if (hn < h1) store(buf);
    t = tn;
    head = hn;
  }
  if (!in) return;
  if (parts > 1) {
    float* to = a.part_kv + ((((int64_t)part * a.batch + b) * a.nk + j) * a.kv_heads + kvh) * (2 * DP);
    if constexpr (WHAT & 2) st_column<float, DP>(to, DP, dk, a.scale);
    if constexpr (WHAT & 1) st_column<float, DP>(to + DP, DP, dv, 1.f);
    return;
  }
  if constexpr (WHAT & 1) st_column<T, DP>((T*)a.dv.p + b * a.dv.b + (int64_t)j * a.dv.t + kvh * a.dv.h, a.dim, dv, 1.f);
  if constexpr (WHAT & 2) st_column<T, DP>((T*)a.dk.p + b * a.dk.b + (int64_t)j * a.dk.t + kvh * a.dk.h, a.dim, dk, a.scale);
}

// The parts' sums of dk and dv added, in their order: four columns a thread.  Bound by reading
// the parts (134 MB of 2 x 4096 keys, 4 heads of 128 in four parts: 23 us).
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_dkv_join(AttnArgs a) {
  constexpr int PER = 2 * DP / 4;  // threads a row: dk's and dv's columns side by side
  const int64_t rows = (int64_t)a.batch * a.nk * a.kv_heads, x = (int64_t)blockIdx.x * 256 + threadIdx.x, r = x / PER;
  if (r >= rows) return;
  const int at = (int)(x % PER) * 4, d = at % DP;
  const int parts = a.head_parts * a.q_parts;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part_kv + (p * rows + r) * (2 * DP) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += v[i];
  }
  const int kvh = (int)(r % a.kv_heads), j = (int)(r / a.kv_heads % a.nk), b = (int)(r / a.kv_heads / a.nk);
  const AttnMat& m = at < DP ? a.dk : a.dv;
  T* to = (T*)m.p + b * m.b + (int64_t)j * m.t + kvh * m.h + d;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (d + i < a.dim) std_(to + i, (double)s[i]);
}

// ---------------------------------------------------------------- launches
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }
int keys_of(int dtype) { return dtype == DT_BF16 ? BN<bf16_t> : BN<float>; }
int q_step_of(int dtype, const AttnArgs& a) { return dtype == DT_BF16 && a.dim <= 64 ? QT_<bf16_t, 64> : 32; }
int dq_keys_of(int dtype, const AttnArgs& a) { return dtype == DT_BF16 && a.dim <= 64 ? BN_DQ<bf16_t, 64> : 32; }

// Few query rows (k_attn_few): those of the heads that share keys go together, for keys that are
// read once for all of them.  Up to 64: twice the keys' reads, by then from the L2.
bool few(const AttnArgs& a) { return (int64_t)a.nq * (a.heads / a.kv_heads) <= 64; }

// Parts of the keys where the rows alone do not fill the card.  k_attn_fwd: two workgroups a CU, at
// least 4 steps each (fp32, whose steps are long: 2), 1: none.  k_attn_few: workgroups over all sequences for each key head and block of
// rows, two a CU, of at least 8 steps of 32 keys; 0: up to 4 steps, which a wave does sooner than a
// second launch joins them, and where the rows alone are eight waves a CU.
int parts(int dtype, const AttnArgs& a) {
  if (few(a)) {
    const int64_t units = ceil_div((int64_t)a.nq * a.pk, 32) * a.kv_heads, steps = ceil_div(a.nk, 32);
    if (steps <= 4 || units == 0 || units * a.batch >= 2048) return 0;
    return (int)std::max<int64_t>(a.batch, std::min<int64_t>(ceil_div(512, units), a.batch * ceil_div(steps, 8)));
  }
  const int64_t groups = ceil_div(a.nq, ROWS) * a.heads * a.batch, steps = ceil_div(a.nk, keys_of(dtype));
  if (groups == 0 || groups >= 256) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(512, groups), steps / (dtype == DT_BF16 ? 4 : 2)));
}

// Parts of the keys of k_attn_dq where its rows do not fill the card, of at least 8 steps (fp32, whose steps are
// long: 2).  Not with documents: the parts are cut from all keys, not from those of a block's documents, so most of
// them would be empty.  (Training steps: fp32, 2902 tokens, one head of 33: 207 us, in
// one part 469; bf16, 3840 tokens, 8 heads of 64: 239 and 287.)
int dq_parts(int dtype, const AttnArgs& a) {
  const int64_t groups = ceil_div(a.nq, ROWS) * a.heads * a.batch, steps = ceil_div(a.nk, dq_keys_of(dtype, a));
  if (groups == 0 || groups >= 256 || a.q_doc) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(512, groups), steps / (dtype == DT_BF16 ? 8 : 2)));
}

// Where dq's products keep dX to 16 bits.
bool few_keys(const AttnArgs& a) { return a.k_doc || a.nk <= 2048; }

// blocks of 32 queries that hold distances within the range, of 32 keys
int near_blocks(const AttnArgs& a) { return (int)std::min<int64_t>(ceil_div(a.nq, 32), ceil_div(2 * (int64_t)a.range + 62, 32) + 1); }

// Parts of k_attn_dkv where its blocks of keys do not fill the card twice over (causal, where they
// differ in length: four times): heads that share keys first, then runs of queries, of at least 8 steps
// (fp32, whose steps are long: 2).  Not with documents: the parts are cut from all queries, not from those of a
// block's documents, so most of them would be empty (2 x 4096 tokens, 12 heads of 64, documents of 32 to 2048: 147 us without, 172 with).
void cut_dkv(int dtype, AttnArgs& a, int64_t kgroups) {
  const int group = a.heads / a.kv_heads, want = a.causal ? 1024 : 512;
  a.head_parts = a.q_parts = 1;
  if (kgroups == 0) return;
  for (int d = 1; d <= group && kgroups * a.head_parts < want; ++d)
    if (group % d == 0) a.head_parts = d;
  const int64_t groups = kgroups * a.head_parts;
  if (groups < want && !a.q_doc)
    a.q_parts = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(want, groups), ceil_div(a.nq, q_step_of(dtype, a)) / (dtype == DT_BF16 ? 8 : 2)));
}

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
  a.pk = few(a) ? a.heads / a.kv_heads : 1;
  a.splits = parts(dtype, a);
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq;
  const int64_t count = few(a) ? ceil_div((int64_t)a.nq * a.pk, 32) * a.kv_heads * a.splits * 128 : a.splits > 1 ? rows * a.splits : 0;
  if (count > 0) {
    a.part_o = (float*)take((size_t)count * padded_dim(a.dim) * 4);
    a.part_ml = (float*)take((size_t)count * 8);
  }
  if (a.k_doc && !few(a)) a.k_tab = (int4*)take((size_t)a.batch * ceil_div(a.nk, keys_of(dtype)) * sizeof(int4));
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
  const int64_t kgroups = ceil_div(a.nk, ROWS) * a.kv_heads * a.batch;
  cut_dkv(dtype, a, kgroups);
  a.splits = dq_parts(dtype, a);
  if (a.splits > 1) {
    const int64_t count = (int64_t)a.batch * a.heads * a.nq * a.splits;
    a.part_o = (float*)take((size_t)count * padded_dim(a.dim) * 4);
    a.part_ml = (float*)take((size_t)count * 4);
  }
  if (a.head_parts * a.q_parts > 1)
    a.part_kv = (float*)take((size_t)a.batch * a.nk * a.kv_heads * a.head_parts * a.q_parts * 2 * padded_dim(a.dim) * 4);
  a.rows = (float*)take((size_t)a.batch * a.heads * ceil_div(a.nq, ROWS) * 4 * ROW_INFO * 4);
  if (a.k_doc) {
    a.k_tab = (int4*)take((size_t)a.batch * ceil_div(a.nk, dq_keys_of(dtype, a)) * sizeof(int4));
    a.q_tab = (int4*)take((size_t)a.batch * ceil_div(a.nq, q_step_of(dtype, a)) * sizeof(int4));
  }
  if (a.grad_bias) {
    const int64_t waves = (int64_t)a.batch * a.heads * ceil_div(a.nk, ROWS) * 4;
    a.near = near_blocks(a);
    a.diag = (float*)take((size_t)waves * a.near * 64 * 4);
    a.tail = (float*)take((size_t)waves * a.q_parts * 8);
  }
  return n;
}

// documents of the tiles of keys, and (q_step > 0) of queries
void launch_docs(const AttnArgs& a, int k_step, int q_step, hipStream_t s) {
  DocArgs d{};
  d.doc[0] = a.k_doc;
  d.len[0] = a.k_len;
  d.n[0] = a.nk;
  d.tile[0] = k_step;
  d.tiles[0] = (int)ceil_div(a.nk, k_step);
  d.tab[0] = a.k_tab;
  d.doc[1] = a.q_doc;
  d.len[1] = a.q_len;
  d.n[1] = a.nq;
  d.tile[1] = q_step;
  d.tiles[1] = q_step > 0 ? (int)ceil_div(a.nq, q_step) : 0;
  d.tab[1] = a.q_tab;
  if (d.tiles[0] + d.tiles[1] == 0) return;
  XP_LAUNCH("k_attn_docs", 4.0 * a.batch * (a.nk + (q_step > 0 ? a.nq : 0)), k_attn_docs, dim3(d.tiles[0] + d.tiles[1], a.batch), dim3(64), 0, s, d);
}

void launch_pack(int dtype, const AttnArgs& a, const AttnMat* from, const AttnMat* const* to, int n, hipStream_t s) {
  PackArgs p{};
  p.dim = a.dim;
  p.ldim = a.ldim;
  int count = 0;
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    if (!from[i].p) continue;
    const bool keys = i == 1 || i == 2;
    p.from[count] = from[i];
    p.to[count] = (void*)to[i]->p;
    p.tokens[count] = keys ? a.nk : a.nq;
    p.heads[count] = keys ? a.kv_heads : a.heads;
    p.rows[count] = (int64_t)a.batch * p.tokens[count] * p.heads[count];
    most = std::max(most, p.rows[count++]);
  }
  if (count == 0) return;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(most * a.ldim, 256 * 8), 4096), count);
  if (dtype == DT_BF16) XP_LAUNCH("k_attn_pack<bf16>", 4.0 * most * count * a.ldim, k_attn_pack<bf16_t>, grid, dim3(256), 0, s, p);
  else XP_LAUNCH("k_attn_pack<f32>", 8.0 * most * count * a.ldim, k_attn_pack<float>, grid, dim3(256), 0, s, p);
}

template <typename T, int DP, int MODE>
void fwd(const AttnArgs& a, hipStream_t s) {
  const double flops = 4.0 * a.batch * a.heads * a.nq * (double)a.nk * a.dim;
  const int64_t rows = (int64_t)a.batch * a.heads * a.nq;
  if (few(a)) {
    const int64_t units = ceil_div((int64_t)a.nq * a.pk, 32) * a.kv_heads, groups = a.splits > 0 ? units * a.splits : ceil_div(units * a.batch, 4);
    XP_LAUNCH(sizeof(T) == 2 ? "k_attn_few<bf16>" : "k_attn_few<f32>", flops, (k_attn_few<T, DP, MODE>), dim3((unsigned)groups), dim3(256), 0, s, a);
    if (a.splits > 0)
      XP_LAUNCH("k_attn_join", 512.0 * units * a.splits * DP, (k_attn_join<T, DP, true>), dim3((unsigned)rows), dim3(256), 0, s, a);
    return;
  }
  const int64_t groups = ceil_div(a.nq, ROWS) * a.heads * a.batch * a.splits;
  XP_LAUNCH(sizeof(T) == 2 ? "k_attn_fwd<bf16>" : "k_attn_fwd<f32>", flops, (k_attn_fwd<T, DP, MODE>), dim3((unsigned)groups), dim3(256), 0, s, a);
  if (a.splits > 1)
    XP_LAUNCH("k_attn_join", 4.0 * rows * a.splits * DP, (k_attn_join<T, DP, false>), dim3((unsigned)rows), dim3(256), 0, s, a);
}

template <typename T, int DP, int MODE>
void bwd(const AttnArgs& a, hipStream_t s) {
  const double pairs = (double)a.batch * a.heads * a.nq * a.nk;
  const int64_t parts = (int64_t)a.head_parts * a.q_parts;
  const int64_t groups = ceil_div(a.nq, ROWS) * a.heads * a.batch * a.splits, kgroups = ceil_div(a.nk, ROWS) * a.kv_heads * a.batch * parts;
  if (groups > 0) {
    const double flops = 6 * pairs * a.dim;
    bool done = false;
    if constexpr (sizeof(T) == 2) {
      if (few_keys(a)) {
        XP_LAUNCH("k_attn_dq<bf16>", flops, (k_attn_dq<T, DP, MODE, true>), dim3((unsigned)groups), dim3(256), 0, s, a);
        done = true;
      }
    }
    if (!done) XP_LAUNCH(sizeof(T) == 2 ? "k_attn_dq<bf16>" : "k_attn_dq<f32>", flops, (k_attn_dq<T, DP, MODE, false>), dim3((unsigned)groups), dim3(256), 0, s, a);
    if (a.splits > 1) {
      const int64_t rows = (int64_t)a.batch * a.heads * a.nq;
      XP_LAUNCH("k_attn_dq_join", 4.0 * rows * a.splits * DP, (k_attn_dq_join<T, DP>), dim3((unsigned)ceil_div(rows * (DP / 4), 256)), dim3(256), 0, s, a);
    }
  }
  if (kgroups == 0) return;
  if constexpr (sizeof(T) == 4 && DP > 64) {
    XP_LAUNCH("k_attn_dv<f32>", 4 * pairs * a.dim, (k_attn_dkv<T, DP, MODE, 1>), dim3((unsigned)kgroups), dim3(256), 0, s, a);
    XP_LAUNCH("k_attn_dk<f32>", 6 * pairs * a.dim, (k_attn_dkv<T, DP, MODE, 2>), dim3((unsigned)kgroups), dim3(256), 0, s, a);
  } else {
    XP_LAUNCH(sizeof(T) == 2 ? "k_attn_dkv<bf16>" : "k_attn_dkv<f32>", 8 * pairs * a.dim, (k_attn_dkv<T, DP, MODE, 3>), dim3((unsigned)kgroups),
              dim3(256), 0, s, a);
  }
  if (parts > 1) {
    const int64_t rows = (int64_t)a.batch * a.nk * a.kv_heads;
    XP_LAUNCH("k_attn_dkv_join", 8.0 * rows * parts * DP, (k_attn_dkv_join<T, DP>), dim3((unsigned)ceil_div(rows * (2 * DP / 4), 256)), dim3(256), 0, s, a);
  }
  if (a.grad_bias && groups > 0)
    XP_LAUNCH("k_attn_dbias", 4.0 * (2 * a.range + 1) * a.heads, k_attn_dbias, dim3((unsigned)ceil_div(2 * (int64_t)a.range + 1, 64), a.heads), dim3(1024), 0, s, a);
}

// calls f(element type, padded dim, kind of scores)
template <typename F>
void by_kind(int dtype, const AttnArgs& a, F&& f) {
  using std::integral_constant;
  auto with = [&](auto t, auto d) {
    if (a.bias && a.cap > 0.f) f(t, d, integral_constant<int, BOTH>{});
    else if (a.bias) f(t, d, integral_constant<int, BIAS>{});
    else if (a.cap > 0.f) {
      if constexpr (sizeof(t) == 2) {
        if (a.cap <= QUICK_CAP) return f(t, d, integral_constant<int, QUICK>{});
      }
      f(t, d, integral_constant<int, CAP>{});
    } else f(t, d, integral_constant<int, PLAIN>{});
  };
  auto dims = [&](auto t) {
    if (a.dim <= 64) with(t, integral_constant<int, 64>{});
    else if (a.dim <= 96) with(t, integral_constant<int, 96>{});
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
  const AttnMat* const to[3] = {&a.q, &a.k, &a.v};
  launch_pack(dtype, a, from, to, 3, s);
  if (a.k_tab) launch_docs(a, keys_of(dtype), 0, s);
  by_kind(dtype, a, [&](auto t, auto d, auto g) { fwd<decltype(t), decltype(d)::value, decltype(g)::value>(a, s); });
  return hipGetLastError();
}

hipError_t launch_attn_bwd(int dtype, AttnArgs a, void* workspace, hipStream_t s) {
  AttnMat from[4];
  a.pk = 1;
  lay_bwd(dtype, a, (char*)workspace, from);
  const AttnMat* const to[4] = {&a.q, &a.k, &a.v, &a.dout};
  launch_pack(dtype, a, from, to, 4, s);
  if (a.k_doc) launch_docs(a, dq_keys_of(dtype, a), q_step_of(dtype, a), s);
  by_kind(dtype, a, [&](auto t, auto d, auto g) { bwd<decltype(t), decltype(d)::value, decltype(g)::value>(a, s); });
  return hipGetLastError();
}

}  // namespace xp
