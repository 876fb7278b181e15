// Linear layers outside a stage: y = act(x W^T + b) + residual and its gradients
// (LinearArgs in xp_kernels.h defines the three products), bf16 on bf16 MFMA and
// fp32 on fp32 MFMA, both with fp32 accumulators; each stored value is rounded
// once, from fp32.
#include "xp_device.h"
#include "xp_lds.h"
#include "xp_kernels.h"

#include <algorithm>
#include <cstdio>

namespace xp {

namespace {

// elements of a 16-byte chunk, and of a step's 128 bytes of the reduction
template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);
template <typename T> constexpr int STEP = 128 / (int)sizeof(T);

// ---------------------------------------------------------------- activations
// In fp32: a stored value is rounded to 8 (bf16) or 24 bits from there, and the
// product before it has fp32 sums.  The reciprocal is the hardware's (good to 2^-23), and
// so is the exponential in bf16 storage (2^-23 times the argument's size); in fp32 it
// is expf, good to as much of itself whatever the argument.  The normal distribution
// function shares its exponential with the density in GELU's slope: Phi(-a) = exp(-a^2 / 2) t P(t) with
// t = 1 / (1 + p a), where
//   fp32 storage: P has nine terms, fitted here for the least relative error over
//     0 <= a <= 14.5 (beyond, Phi leaves fp32): good to 8 * 2^-24 of itself, rounding
//     included, and the exponential's argument to a^2 / 2 of them, in the far tail too
//     (xpipe_act_bwd of 2^26 elements 137 us, as ReLU; with erfcf 155).
//   bf16 storage: six terms, fitted to 5e-8 of 1 and to 2^-11 of Phi itself, an eighth of
//     bf16's half step, where that is less (both gradients of 8192x8192x2048 behind a GELU
//     639 us with erff and expf, 559 so).
template <typename T>
XP_DEV float normal_cdf(float z, float& e) {  // and e = exp(-z^2 / 2)
  float tail;
  if constexpr (sizeof(T) == 4) {
    e = expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.28f * fabsf(z));
    tail = e * t * (0.111689358f + t * (0.111959679f + t * (0.101177704f + t * (0.0911249906f + t * (0.0554682483f +
                   t * (0.0176901268f + t * (0.0725002237f + t * (-0.0846662747f + t * 0.0230559717f))))))));
  } else {
    e = __expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.29f * fabsf(z));
    tail = e * t * (0.116616427f + t * (0.102033926f + t * (0.176945863f + t * (-0.0907976066f + t * (0.283885533f -
                   t * 0.0886841861f)))));
  }
  return z >= 0.f ? 1.f - tail : tail;
}
template <typename T>
XP_DEV float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + (sizeof(T) == 4 ? expf(-z) : __expf(-z))); }

template <typename T, int N>
XP_DEV void act_values(float (&z)[N], int act) {
  if (act == LIN_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] > 0.f ? z[i] : (z[i] != z[i] ? z[i] : 0.f);
  } else if (act == LIN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      z[i] *= normal_cdf<T>(z[i], e);
    }
  } else if (act == LIN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= sigmoid<T>(z[i]);
  }
}

// v *= act'(z); 0 at 0 for the ReLU, and then 0 whatever v (an infinite gradient of a
// dead unit is none)
template <typename T, int N>
XP_DEV void act_slopes(float (&v)[N], const float (&z)[N], int act) {
  if (act == LIN_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = z[i] > 0.f ? v[i] : 0.f;
  } else if (act == LIN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      const float c = normal_cdf<T>(z[i], e);
      v[i] *= c + z[i] * 0.39894228040143268f * e;
    }
  } else if (act == LIN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float s = sigmoid<T>(z[i]);
      v[i] *= s * (1.f + z[i] * (1.f - s));
    }
  }
}

// ---------------------------------------------------------------- epilogue
template <typename T> XP_DEV float ldf(const T* p);
template <> XP_DEV float ldf<float>(const float* p) { return *p; }
template <> XP_DEV float ldf<bf16_t>(const bf16_t* p) { return bf16_to_f32(*p); }

// a 16-byte chunk: CHUNK<T> elements
template <typename T>
XP_DEV void unpack(const u32x4_t& u, float (&v)[CHUNK<T>]) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(u[i]);
    else v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  }
}
template <typename T>
XP_DEV u32x4_t pack(const float (&v)[CHUNK<T>]) {
  u32x4_t u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(v[i]);
    else u[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
  }
  return u;
}
// the first n of a chunk's elements, one by one
template <typename T>
XP_DEV u32x4_t ld_some(const T* p, int n) {
  float v[CHUNK<T>];
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) v[i] = i < n ? ldf<T>(p + i) : 0.f;
  return pack<T>(v);  // (bf16 values: no rounding)
}
template <typename T>
XP_DEV void st_some(T* p, int n, const float (&v)[CHUNK<T>]) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i)
    if (i < n) {
      if constexpr (sizeof(T) == 4) p[i] = v[i];
      else p[i] = f32_to_bf16(v[i]);
    }
}
// a chunk with n elements left in its row: vec, aligned (whole chunks only); else of any alignment
template <typename T>
XP_DEV u32x4_t ld_chunk(const T* p, bool vec, int n) {
  if (vec) return *reinterpret_cast<const u32x4_t*>(p);
  if (n < CHUNK<T>) return ld_some<T>(p, n);
  u32x4_t u;
  __builtin_memcpy(&u, p, 16);
  return u;
}
template <typename T>
XP_DEV void st_chunk(T* p, bool vec, int n, const float (&v)[CHUNK<T>]) {
  if (vec) {
    *reinterpret_cast<u32x4_t*>(p) = pack<T>(v);
  } else if (n < CHUNK<T>) {
    st_some<T>(p, n, v);
  } else {
    const u32x4_t u = pack<T>(v);
    __builtin_memcpy(p, &u, 16);
  }
}

// The arguments with the epilogue's pointers moved to row m0 and column n0, and N the
// columns from there: rows and offsets below then are 32 bits wide (256 rows at most,
// XPIPE_LINEAR_MAX_LD elements apart).
template <typename T>
XP_DEV LinearArgs from(LinearArgs a, int64_t m0, int n0) {
  const auto move = [&](const void* p, int64_t ld) __attribute__((always_inline)) -> void* {
    return p ? (void*)((T*)p + m0 * ld + n0) : nullptr;
  };
  a.res = move(a.res, a.ldr);
  a.z_in = move(a.z_in, a.ldz);
  a.z_out = move(a.z_out, a.ldz);
  a.y = move(a.y, a.ldy);
  if (a.grad) a.grad += m0 * a.ldg + n0;
  if (a.bias) a.bias += n0;
  a.N -= n0;
  return a;
}
XP_DEV uint32_t at(int row, int64_t ld, int n) { return (uint32_t)row * (uint32_t)ld + (uint32_t)n; }

// What the epilogue of columns n .. n + CHUNK<T> of row m reads: the residual and the
// pre-activation, or (LIN_GRAD) the accumulators
struct Fetched {
  u32x4_t r, z;
};
template <typename T, int EPI>
XP_DEV Fetched fetch(const LinearArgs& a, int m, int n) {
  const int left = a.N - n;
  const bool vec = a.vec && left >= CHUNK<T>;
  Fetched f;
  if constexpr (EPI == LIN_GRAD) {
    const float* g = a.grad + at(m, a.ldg, n);
    f.r = ld_chunk<float>(g, vec, left);
    if constexpr (sizeof(T) == 2) f.z = ld_chunk<float>(g + 4, vec, left - 4);
  } else {
    if (a.res) f.r = ld_chunk<T>((const T*)a.res + at(m, a.ldr, n), vec, left);
    if (EPI == LIN_DATA && a.z_in) f.z = ld_chunk<T>((const T*)a.z_in + at(m, a.ldz, n), vec, left);
  }
  return f;
}
// the bias of columns n ..
template <typename T, int EPI>
XP_DEV void fetch_bias(const LinearArgs& a, int n, float (&b)[CHUNK<T>]) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) b[i] = EPI == LIN_FWD && a.bias && n + i < a.N ? a.bias[n + i] : 0.f;
}

// The product's epilogue; v: the sums
template <typename T, int EPI>
XP_DEV void finish(const LinearArgs& a, int m, int n, float (&v)[CHUNK<T>], const float (&b)[CHUNK<T>], const Fetched& f) {
  constexpr int C = CHUNK<T>;
  const int left = a.N - n;
  const bool vec = a.vec && left >= C;
  if constexpr (EPI == LIN_GRAD) {
    // fp32 accumulators whatever T
    float* g = a.grad + at(m, a.ldg, n);
#pragma unroll
    for (int h = 0; h < C / 4; ++h) {
      float o[4];
      unpack<float>(h ? f.z : f.r, o);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += v[4 * h + i];
      st_chunk<float>(g + 4 * h, vec, left - 4 * h, o);
    }
    return;
  }
  if constexpr (EPI == LIN_FWD) {
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += b[i];
    if (a.z_out) st_chunk<T>((T*)a.z_out + at(m, a.ldz, n), vec, left, v);
    act_values<T>(v, a.act);
  } else if (a.z_in) {
    float z[C];
    unpack<T>(f.z, z);
    act_slopes<T>(v, z, a.act);
  }
  if (a.res) {
    float r[C];
    unpack<T>(f.r, r);
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += r[i];
  }
  st_chunk<T>((T*)a.y + at(m, a.ldy, n), vec, left, v);
}

// The same for one element of a forward: what it reads, and its end
struct Fetched1 {
  float r, b;
};
template <typename T>
XP_DEV Fetched1 fetch1(const LinearArgs& a, int m, int n) {
  return Fetched1{a.res ? ldf<T>((const T*)a.res + at(m, a.ldr, n)) : 0.f, a.bias ? a.bias[n] : 0.f};
}
template <typename T>
XP_DEV void finish1(const LinearArgs& a, int m, int n, float sum, const Fetched1& f) {
  const auto st = [&](void* p, int64_t ld, float v) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 4) ((float*)p)[at(m, ld, n)] = v;
    else ((bf16_t*)p)[at(m, ld, n)] = f32_to_bf16(v);
  };
  float v[1] = {sum + f.b};
  if (a.z_out) st(a.z_out, a.ldz, v[0]);
  act_values<T>(v, a.act);
  st(a.y, a.ldy, a.res ? v[0] + f.r : v[0]);
}

// ---------------------------------------------------------------- product
// LDS tile of an operand, one step deep.  Stored with the reduction along its
// rows in memory (TR false): one 128-byte row of 8 chunks per tile row, chunk c
// of row r at position c ^ (r / 2 & 7): two rows span the banks, and the 16 rows
// that a fragment read takes at a time then lie in different ones.  Stored with the reduction down its rows (TR true): one row of
// W elements per reduction index; chunk c of row k at c ^ tr_swz(k), which moves
// the rows that one fragment read touches to different banks.
template <typename T, int W>
XP_DEV int tr_swz(int k) {
  if constexpr (sizeof(T) == 4) return ((k >> 2) & 1) << 3;
  else return W >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
}

// Transposing LDS reads of N bf16 fragments (16 of the reduction, 32 columns), in one
// block with their wait.  In each group of 16 lanes, output e (0..3) of lane i is
// element i % 4 of the 8 bytes that lane 4 e + i / 4 addressed; a fragment is two
// reads, HI bytes (four rows) apart.  As builtins they would each wait for every
// copy into LDS that is in flight (the compiler does not see which array they read).
template <int N, int OFF, int HI>
XP_DEV void read_tr(const uint32_t (&at)[N], u32x4_t (&out)[N]) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  static_assert(N == 1 || N == 2 || N == 4 || N == 6, "blocks written out");
  static_assert(OFF + HI < 65536, "16-bit offsets");
  u32x2_t lo[N], hi[N];
#define XP_TR(A, D) "ds_read_b64_tr_b16 %" #D ", %" #A " offset:%c[o]\n\t"
#define XP_TRH(A, D) "ds_read_b64_tr_b16 %" #D ", %" #A " offset:%c[h]\n\t"
#define XP_WAIT "s_waitcnt lgkmcnt(0)"
  if constexpr (N == 1)
    asm volatile(XP_TR(2, 0) XP_TRH(2, 1) XP_WAIT
                 : "=&v"(lo[0]), "=&v"(hi[0]) : "v"(at[0]), [o] "n"(OFF), [h] "n"(OFF + HI) : "memory");
  else if constexpr (N == 2)
    asm volatile(XP_TR(4, 0) XP_TRH(4, 1) XP_TR(5, 2) XP_TRH(5, 3) XP_WAIT
                 : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1])
                 : "v"(at[0]), "v"(at[1]), [o] "n"(OFF), [h] "n"(OFF + HI) : "memory");
  else if constexpr (N == 4)
    asm volatile(XP_TR(8, 0) XP_TRH(8, 1) XP_TR(9, 2) XP_TRH(9, 3) XP_TR(10, 4) XP_TRH(10, 5) XP_TR(11, 6) XP_TRH(11, 7) XP_WAIT
                 : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1]), "=&v"(lo[2]), "=&v"(hi[2]), "=&v"(lo[3]), "=&v"(hi[3])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), [o] "n"(OFF), [h] "n"(OFF + HI) : "memory");
  else
    asm volatile(XP_TR(12, 0) XP_TRH(12, 1) XP_TR(13, 2) XP_TRH(13, 3) XP_TR(14, 4) XP_TRH(14, 5) XP_TR(15, 6) XP_TRH(15, 7)
                 XP_TR(16, 8) XP_TRH(16, 9) XP_TR(17, 10) XP_TRH(17, 11) XP_WAIT
                 : "=&v"(lo[0]), "=&v"(hi[0]), "=&v"(lo[1]), "=&v"(hi[1]), "=&v"(lo[2]), "=&v"(hi[2]), "=&v"(lo[3]), "=&v"(hi[3]),
                   "=&v"(lo[4]), "=&v"(hi[4]), "=&v"(lo[5]), "=&v"(hi[5])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), [o] "n"(OFF), [h] "n"(OFF + HI)
                 : "memory");
#undef XP_TR
#undef XP_TRH
#undef XP_WAIT
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = __builtin_shufflevector(lo[i], hi[i], 0, 1, 2, 3);
}

// The same for fp32: of N columns (a lane each) four rows, PITCH bytes apart.
template <int N, int OFF, int PITCH>
XP_DEV void read_col(const uint32_t (&at)[N], u32x4_t (&out)[N]) {
  static_assert(N == 1 || N == 2 || N == 4, "blocks written out");
  static_assert(OFF + 3 * PITCH < 65536, "16-bit offsets");
  uint32_t v[4 * N];
#define XP_C4(A, D0, D1, D2, D3)                                                                        \
  "ds_read_b32 %" #D0 ", %" #A " offset:%c[p0]\n\tds_read_b32 %" #D1 ", %" #A " offset:%c[p1]\n\t"      \
  "ds_read_b32 %" #D2 ", %" #A " offset:%c[p2]\n\tds_read_b32 %" #D3 ", %" #A " offset:%c[p3]\n\t"
#define XP_O4(I) "=&v"(v[4 * I]), "=&v"(v[4 * I + 1]), "=&v"(v[4 * I + 2]), "=&v"(v[4 * I + 3])
#define XP_OFFS [p0] "n"(OFF), [p1] "n"(OFF + PITCH), [p2] "n"(OFF + 2 * PITCH), [p3] "n"(OFF + 3 * PITCH)
#define XP_WAIT "s_waitcnt lgkmcnt(0)"
  if constexpr (N == 1)
    asm volatile(XP_C4(4, 0, 1, 2, 3) XP_WAIT : XP_O4(0) : "v"(at[0]), XP_OFFS : "memory");
  else if constexpr (N == 2)
    asm volatile(XP_C4(8, 0, 1, 2, 3) XP_C4(9, 4, 5, 6, 7) XP_WAIT : XP_O4(0), XP_O4(1) : "v"(at[0]), "v"(at[1]), XP_OFFS : "memory");
  else
    asm volatile(XP_C4(16, 0, 1, 2, 3) XP_C4(17, 4, 5, 6, 7) XP_C4(18, 8, 9, 10, 11) XP_C4(19, 12, 13, 14, 15) XP_WAIT
                 : XP_O4(0), XP_O4(1), XP_O4(2), XP_O4(3)
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), XP_OFFS : "memory");
#undef XP_C4
#undef XP_O4
#undef XP_OFFS
#undef XP_WAIT
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = (u32x4_t){v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}

// bytes of a step's two tiles
template <int BM, int BN> constexpr int STAGE = (BM + BN) * 128;

// One workgroup per BM x BN tile of the product and part of the reduction, WM x
// WN waves of 32x32 MFMA results.  Both operands are copied from memory
// straight into LDS, one step (128 bytes of the reduction) at a time, with NS
// buffers: NS - 1 steps are in flight while one is multiplied.
// Measured (256x256 tiles, the library's plain product in turn on the same card in
// brackets): forward 8192x16384x4096 0.83 ms (0.68), 1.33 PFLOP/s (1.61); 8192x8192x8192 0.82
// (0.67).  By counters the matrix units are busy for two thirds of the cycles, at the
// 1.7 GHz that power leaves: the last third is the waves' wait for each step's barrier,
// copies and fragments (0.38 of their cycles), which one tile of two waves per SIMD does not
// cover.  8192x8192x2048 dx 233 us (222), behind a GELU 286: the epilogue's own
// traffic, which nothing overlaps with one tile on a CU (128x128 tiles, two on a CU, 289
// and 319); weight gradient 252 (237).  fp32 8192x8192x8192 7.4 ms, 148 TFLOP/s (154);
// 4096x4096x2048 dx and weight gradient 0.49 ms each, 140 (149): the fp32 matrix rate.
template <typename T, int BM, int BN, int WM, int WN, int NS, bool TA, bool TB, int EPI>
XP_DEV void linear_tile(const LinearArgs& a, int tiles_m, int tiles_n, int lin, unsigned char* st0, unsigned char* st1,
                        unsigned char* st2, unsigned char* st3) {
  constexpr int NW = WM * WN, ES = (int)sizeof(T), C = CHUNK<T>, BK = STEP<T>;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static_assert(WTM % 32 == 0 && WTN % 32 == 0, "wave tile");
  constexpr int A_I = BM / 8 / NW, B_I = BN / 8 / NW;  // copies of 1 KB per wave and step
  static_assert(A_I * NW * 8 == BM && B_I * NW * 8 == BN, "whole copies per wave");
  static_assert(NS >= 2 && NS <= 4, "stages");
  auto stage = [&](auto I) __attribute__((always_inline)) -> unsigned char* {
    constexpr int i = decltype(I)::value;
    if constexpr (i == 0) return st0;
    else if constexpr (i == 1) return st1;
    else if constexpr (i == 2) return st2;
    else return st3;
  };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // tile order: runs of 8 tile rows, so that the tiles that one XCD holds at a
  // time share rows of both operands in its L2
  const int split = lin / (tiles_m * tiles_n), tile = lin - split * tiles_m * tiles_n;
  const int grp = tile / (8 * tiles_n), gm = min(8, tiles_m - grp * 8), in = tile - grp * 8 * tiles_n;
  const int tm = grp * 8 + in % gm, tn = in / gm;
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;
  const int64_t kbeg = (int64_t)split * a.kper;
  const int64_t kend = min((int64_t)a.K, kbeg + a.kper);
  const int nk = (int)((kend - kbeg + BK - 1) / BK);

  // Per copy the lane's byte offset from the step's base, ~0 where its row (TR:
  // its column chunk) is past the operand; the base moves by one step at a time, and
  // reduction indices past the end are masked step by step.  So every chunk that
  // is copied holds an element of the operand (a 16-byte chunk never leaves that
  // element's page).
  const char* abase = (const char*)a.A + (TA ? kbeg * a.lda + m0 : m0 * a.lda + kbeg) * ES;
  const char* bbase = (const char*)a.B + (TB ? kbeg * a.ldb + n0 : n0 * a.ldb + kbeg) * ES;
  const int64_t astep = TA ? (int64_t)BK * a.lda * ES : 128, bstep = TB ? (int64_t)BK * a.ldb * ES : 128;
  uint32_t a_off[A_I], b_off[B_I];
  int a_k[A_I], b_k[B_I];  // the reduction index (of the step) that the copy reads
  auto place = [&](auto TR, auto W, int i, int64_t r0, int64_t rows, int64_t ld, uint32_t& off, int& k) __attribute__((always_inline)) {
    constexpr int w = decltype(W)::value;
    if constexpr (decltype(TR)::value) {
      constexpr int CPR = w / C;  // chunks per row
      const int pos = i * 64 + lane;
      k = pos / CPR;
      const int col = ((pos % CPR) ^ tr_swz<T, w>(k)) * C;
      off = r0 + col < rows ? (uint32_t)((k * ld + col) * ES) : ~0u;
    } else {
      const int r = i * 8 + (lane >> 3), c = (lane & 7) ^ (r >> 1 & 7);
      k = c * C;
      off = r0 + r < rows ? (uint32_t)((r * ld + k) * ES) : ~0u;
    }
  };
#pragma unroll
  for (int i = 0; i < A_I; ++i)
    place(std::bool_constant<TA>{}, std::integral_constant<int, BM>{}, wave * A_I + i, m0, a.M, a.lda, a_off[i], a_k[i]);
#pragma unroll
  for (int i = 0; i < B_I; ++i)
    place(std::bool_constant<TB>{}, std::integral_constant<int, BN>{}, wave * B_I + i, n0, a.N, a.ldb, b_off[i], b_k[i]);

  int left = (int)(kend - kbeg);  // reduction indices not copied yet
  // the copies [from, to) of a step's A_I + B_I (past the last step: zeros)
  auto copy = [&](auto I, int from, int to) __attribute__((always_inline)) {
    unsigned char* sa = stage(I);
    unsigned char* sb = stage(I) + BM * 128;
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void*)abase, (short)0, 0x7ffffff0, 0x00020000);
    const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc((void*)bbase, (short)0, 0x7ffffff0, 0x00020000);
#pragma unroll
    for (int q = from; q < to; ++q) {
      const int i = q < A_I ? q : q - A_I;
      if (q < A_I) load_lds16(ar, (bf16_t*)(sa + (wave * A_I + i) * 1024), a_k[i] < left ? (int)a_off[i] : -1, 0);
      else load_lds16(br, (bf16_t*)(sb + (wave * B_I + i) * 1024), b_k[i] < left ? (int)b_off[i] : -1, 0);
    }
    if (to == A_I + B_I) {
      abase += astep;
      bbase += bstep;
      left -= BK;
    }
  };

  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  // Fragments of 32 rows (columns of the product), 16 bytes of the reduction per
  // lane: lane l holds row l % 32 and the chunk l / 32 of the pair kk (bf16: 8
  // elements for one 32x32x16 product; fp32: 4, one for each of four 32x32x2
  // products, whose reduction indices then are 4 (l / 32) + q in both operands).
  const int fr = lane & 31, fh = lane >> 5;
  // (One offset into the stage's array per read: the compiler then sees which array
  // it reads, and waits for no copies into the others.)
  auto frag = [&](auto I, int base, int row0, int kk) __attribute__((always_inline)) -> u32x4_t {
    return *reinterpret_cast<const u32x4_t*>(stage(I) + (base + (row0 + fr) * 128 + (((kk * 2 + fh) ^ (fr >> 1 & 7)) << 4)));
  };
  // Two sets of fragments: while the products of one quarter of a step run, the next
  // quarter's fragments are read.
  u32x4_t fa[2][TM], fb[2][TN];
  // where the lane's reads of columns start (in the first quarter, from the stage's array on)
  constexpr int TRN = (TA ? TM : 0) + (TB ? TN : 0);
  uint32_t tr_at[TRN > 0 ? TRN : 1];
  if constexpr (TRN > 0) {
    static_assert(BM == BN, "one offset for both operands' rows");
    auto at = [&](int base, int row0) __attribute__((always_inline)) -> uint32_t {
      // the first read's row (the swizzle is the same for all of the lane's rows) and column
      const int k = ES == 2 ? 8 * fh + ((lane & 15) >> 2) : 4 * fh;
      const int c = ES == 2 ? row0 + 16 * (fr >> 4) + 4 * (lane & 3) : row0 + fr;
      return base + k * (BM * ES) + (((c / C) ^ tr_swz<T, BM>(k)) << 4) + c % C * ES;
    };
    if constexpr (TB) {
#pragma unroll
      for (int j = 0; j < TN; ++j) tr_at[j] = at(BM * 128, wn * WTN + j * 32);
    }
    if constexpr (TA) {
#pragma unroll
      for (int i = 0; i < TM; ++i) tr_at[TRN - TM + i] = at(0, wm * WTM + i * 32);
    }
  }
  auto read = [&](auto I, auto KK, int set) __attribute__((always_inline)) {
    constexpr int kk = decltype(KK)::value;
    // (B's first: the next quarter's first products take all of them and one of A's)
    if constexpr (!TB) {
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[set][j] = frag(I, BM * 128, wn * WTN + j * 32, kk);
    }
    if constexpr (!TA) {
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[set][i] = frag(I, 0, wm * WTM + i * 32, kk);
    }
    if constexpr (TRN > 0) {
      const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)stage(I);
      uint32_t at[TRN];
      u32x4_t out[TRN];
#pragma unroll
      for (int i = 0; i < TRN; ++i) at[i] = lds + tr_at[i];
      if constexpr (ES == 2) read_tr<TRN, kk * 16 * BM * 2, 4 * BM * 2>(at, out);
      else read_col<TRN, kk * 8 * BM * 4, BM * 4>(at, out);
      if constexpr (TB) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[set][j] = out[j];
      }
      if constexpr (TA) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[set][i] = out[TRN - TM + i];
      }
    }
  };
  auto multiply = [&](int set, int from, int to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = from; i < to; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        if constexpr (ES == 2) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fa[set][i]),
                                                              __builtin_bit_cast(bf16x8_t, fb[set][j]), acc[i][j], 0, 0, 0);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa[set][i][q]), __uint_as_float(fb[set][j][q]),
                                                             acc[i][j], 0, 0, 0);
        }
      }
  };
  // Reads one quarter's fragments and multiplies another's.  Reads that the
  // compiler can move are spread over the products; a block of column reads
  // comes between them (the other wave of the SIMD multiplies while it waits).
  auto overlap = [&](auto I, auto KK, int into, int set) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (TRN > 0) {
      multiply(set, 0, (TM + 1) / 2);
      __builtin_amdgcn_sched_barrier(0);
      read(I, KK, into);
      __builtin_amdgcn_sched_barrier(0);
      multiply(set, (TM + 1) / 2, TM);
    } else {
      constexpr int PER = TM * TN * (ES == 2 ? 1 : 4), READS = TM + TN;
      constexpr int SLOTS = READS < PER ? READS : PER;
      read(I, KK, into);
      multiply(set, 0, TM);
      static_for<0, SLOTS>([&](auto S) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        constexpr int r = (s + 1) * READS / SLOTS - s * READS / SLOTS, m = (s + 1) * PER / SLOTS - s * PER / SLOTS;
        __builtin_amdgcn_sched_group_barrier(0x100, r, 0);  // LDS reads
        __builtin_amdgcn_sched_group_barrier(0x008, m, 0);  // products
      });
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // The last quarter of a step: the copies into its buffer I are issued, and the first
  // fragments of the next step read, between the products.
  auto turn = [&](auto I, auto NEXT) __attribute__((always_inline)) {
    constexpr std::integral_constant<int, 0> Q0{};
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, TM>([&](auto R) __attribute__((always_inline)) {
      constexpr int r = decltype(R)::value;
      if constexpr (r == (TRN > 0 ? TM / 2 : 0)) read(NEXT, Q0, 0);
      multiply(1, r, r + 1);
      copy(I, r * (A_I + B_I) / TM, (r + 1) * (A_I + B_I) / TM);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The bias gradient is the sum of A's rows over the reduction: the first wave
  // column of the first tile column adds the elements of its fragments, a quarter in
  // fp32 (at most 8 of them) and the quarters in fp64.
  const bool sums = EPI == LIN_GRAD && a.grad_b && tn == 0 && wn == 0;
  double bsum[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) bsum[i] = 0.0;
  auto add_rows = [&](int set) __attribute__((always_inline)) {
    if constexpr (EPI == LIN_GRAD) {
      if (sums) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          float e[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if constexpr (ES == 4) e[q] = __uint_as_float(fa[set][i][q]);
            else e[q] = __uint_as_float(fa[set][i][q] << 16) + __uint_as_float(fa[set][i][q] & 0xffff0000u);
          }
          bsum[i] += (double)((e[0] + e[1]) + (e[2] + e[3]));
        }
      }
    }
  };

  // Step k from buffer k % NS.  By its last quarter all of the step's fragments
  // are in registers: past the barrier there the buffer takes the copies of step
  // k + NS, and the first fragments of step k + 1, whose copies have had NS - 1 steps'
  // time to land, are read while the last quarter is multiplied.
  constexpr std::integral_constant<int, 0> B0{};
  static_for<0, NS>([&](auto I) __attribute__((always_inline)) { copy(I, 0, A_I + B_I); });
  wait_step<(NS - 1) * (A_I + B_I)>();
  read(B0, B0, 0);
  int k = 0;
  auto quarters = [&](auto I) __attribute__((always_inline)) {
    static_for<0, 3>([&](auto KK) __attribute__((always_inline)) {
      constexpr int kk = decltype(KK)::value;
      add_rows(kk & 1);
      overlap(I, std::integral_constant<int, kk + 1>{}, (kk + 1) & 1, kk & 1);
    });
    add_rows(1);
  };
  quarters(B0);
  bool more = ++k < nk;
  while (more) {
    static_for<0, NS>([&](auto I) __attribute__((always_inline)) {
      if (more) {
        constexpr std::integral_constant<int, (decltype(I)::value + 1) % NS> NEXT{};
        // this wave's copies of step k have landed and its reads of step k - 1
        // returned; past the barrier so have the others'
        wait_step<(NS - 2) * (A_I + B_I)>();
        turn(I, NEXT);
        quarters(NEXT);
        more = ++k < nk;
      }
    });
  }
  multiply(1, 0, TM);
  wait_step<0>();

  if constexpr (EPI == LIN_GRAD) {
    if (sums) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const double total = bsum[i] + __shfl_xor(bsum[i], 32, 64);
        const int64_t m = m0 + wm * WTM + i * 32 + fr;
        if (fh == 0 && m < a.M) {
          if (a.part) a.part_b[(int64_t)split * a.M + m] = total;
          else a.grad_b[m] = (float)((double)a.grad_b[m] + total);
        }
      }
    }
  }

  // Each wave finishes its tile in strips of 16 rows through its own part of LDS
  // (no barrier), so that memory is accessed by rows, 16 bytes a lane; what a
  // strip's epilogue reads is loaded before the strip before it is finished.  32x32
  // result: lane l, register r holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32.
  constexpr int PITCH = WTN + 4;
  static_assert(NW * 16 * PITCH * 4 <= STAGE<BM, BN>, "strips");
  float* strip = reinterpret_cast<float*>(st0) + wave * 16 * PITCH;
  const int64_t rows = a.M - m0;  // of the tile and below
  const LinearArgs t = from<T>(a, m0, n0);
  auto to_strip = [&](auto S) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 8; ++r)
        strip[(8 * (r >> 2) + 4 * fh + (r & 3)) * PITCH + j * 32 + fr] = acc[s >> 1][j][(s & 1) * 8 + r];
    __builtin_amdgcn_wave_barrier();
  };
  constexpr int CW = WTN / C, RP = 64 / CW, PASS = 16 / RP;  // chunks per strip row, rows per part
  const int ch = lane % CW, c = wn * WTN + ch * C, lr = wm * WTM + lane / CW;
  const bool direct = !a.part;
  float bias[C];
  fetch_bias<T, EPI>(t, c, bias);
  Fetched next[PASS];
  auto prefetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const int row = lr + s * 16 + p * RP;
      if (direct && row < rows && c < t.N) next[p] = fetch<T, EPI>(t, row, c);
    }
  };
  prefetch(0);
  static_for<0, TM * 2>([&](auto S) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
    Fetched now[PASS];
#pragma unroll
    for (int p = 0; p < PASS; ++p) now[p] = next[p];
    if constexpr (s + 1 < TM * 2) prefetch(s + 1);
    to_strip(S);
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const int row = lr + s * 16 + p * RP;
      float v[C];
#pragma unroll
      for (int q = 0; q < C / 4; ++q) {
        const f32x4_t g = *reinterpret_cast<const f32x4_t*>(strip + (p * RP + lane / CW) * PITCH + ch * C + q * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[q * 4 + i] = g[i];
      }
      if (row >= rows || c >= t.N) continue;
      if (direct) {
        finish<T, EPI>(t, row, c, v, bias, now[p]);
      } else {
        // partial sums, rows of N rounded up to whole chunks
        float* out = a.part + ((int64_t)split * a.M + m0 + row) * a.ldpart + n0 + c;
#pragma unroll
        for (int q = 0; q < C / 4; ++q)
          *reinterpret_cast<f32x4_t*>(out + 4 * q) = (f32x4_t){v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      }
    }
    __builtin_amdgcn_wave_barrier();
  });
}

// (separate arrays: see frag)
#define XP_STAGES(BM, BN, NS)                                                   \
  __shared__ __align__(16) unsigned char st0[STAGE<BM, BN>];                    \
  __shared__ __align__(16) unsigned char st1[STAGE<BM, BN>];                    \
  __shared__ __align__(16) unsigned char st2[NS > 2 ? STAGE<BM, BN> : 16];      \
  __shared__ __align__(16) unsigned char st3[NS > 3 ? STAGE<BM, BN> : 16]

template <typename T, int BM, int BN, int WM, int WN, int NS, bool TA, bool TB, int EPI>
__global__ __launch_bounds__(WM * WN * 64) void k_linear(LinearArgs a, int tiles_m, int tiles_n) {
  XP_STAGES(BM, BN, NS);
  linear_tile<T, BM, BN, WM, WN, NS, TA, TB, EPI>(a, tiles_m, tiles_n, xcd_tile(blockIdx.x, gridDim.x), st0, st1, st2, st3);
}

// Both products of a backward in one launch: the first `first` workgroups are the
// data gradient's (grad_first: the weight gradient's).  They depend on nothing of each
// other's, and small ones alone leave most of the GPU idle.
template <typename T, int B, int NS>
__global__ __launch_bounds__(256) void k_linear_bwd(LinearArgs d, int tiles_md, int tiles_nd, int first, int grad_first,
                                                    LinearArgs g, int tiles_mg, int tiles_ng) {
  XP_STAGES(B, B, NS);
  const int b = blockIdx.x;
  const int t = b < first ? xcd_tile(b, first) : xcd_tile(b - first, gridDim.x - first);
  if ((b < first) != (grad_first != 0))
    linear_tile<T, B, B, 2, 2, NS, false, true, LIN_DATA>(d, tiles_md, tiles_nd, t, st0, st1, st2, st3);
  else
    linear_tile<T, B, B, 2, 2, NS, true, true, LIN_GRAD>(g, tiles_mg, tiles_ng, t, st0, st1, st2, st3);
}

// the splits' partial sums added in order, and the epilogue (4 us for 777x515)
template <typename T, int EPI>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  constexpr int C = CHUNK<T>;
  const int cpr = (a.N + C - 1) / C;
  const int64_t total = a.M * cpr;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / cpr;
    const int n = (int)(i - m * cpr) * C;
    const LinearArgs t = from<T>(a, m, 0);
    const Fetched f = fetch<T, EPI>(t, 0, n);
    float v[C], b[C];
    fetch_bias<T, EPI>(t, n, b);
#pragma unroll
    for (int q = 0; q < C; ++q) v[q] = 0.f;
    const float* p = a.part + m * a.ldpart + n;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s, p += a.M * a.ldpart) {
#pragma unroll
      for (int q = 0; q < C / 4; ++q) {
        const f32x4_t g = *reinterpret_cast<const f32x4_t*>(p + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] += g[e];
      }
    }
    finish<T, EPI>(t, 0, n, v, b, f);
  }
  if constexpr (EPI == LIN_GRAD) {
    if (!a.grad_b) return;
    for (int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x; m < a.M; m += (int64_t)gridDim.x * 256) {
      double t = 0.0;
      for (int s = 0; s < a.splits; ++s) t += a.part_b[(int64_t)s * a.M + m];
      a.grad_b[m] = (float)((double)a.grad_b[m] + t);
    }
  }
}

// The first n >= 1 of CHUNK<T> elements at p, of any alignment, zeros behind them: made
// from the aligned 16 bytes that the first lies in and, where they reach past
// those, the next.
template <typename T>
XP_DEV u32x4_t ld_any(const char* p, int n) {
  const int bytes = min(n, CHUNK<T>) * (int)sizeof(T);
  const int mis = (int)(reinterpret_cast<uintptr_t>(p) & 15);
  const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p - mis);
  const u32x4_t lo = q[0];
  u32x4_t hi = {0u, 0u, 0u, 0u};
  if (mis + bytes > 16) hi = q[1];
  uint32_t w[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  if (mis & 8) {
#pragma unroll
    for (int e = 0; e < 6; ++e) w[e] = w[e + 2];
  }
  if (mis & 4) {
#pragma unroll
    for (int e = 0; e < 5; ++e) w[e] = w[e + 1];
  }
  if (mis & 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __funnelshift_r(w[e], w[e + 1], 16);
  }
  u32x4_t out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int have = bytes - 4 * e;
    out[e] = have >= 4 ? w[e] : have == 2 ? w[e] & 0xffffu : 0u;
  }
  return out;
}

// ---------------------------------------------------------------- few rows
// The forward of a few rows, 16 MT of them per workgroup: bound by reading W once, so
// every wave streams its part of the reduction of 16 rows of W from memory
// straight into registers (16x16 products, W the columns, the rows of x the rows,
// empty ones zeros).  The eight waves of a workgroup take the reduction's 128-byte
// steps in turn and add their results through LDS in the order of the waves: no
// workspace, one launch.  ANY: operands of any alignment.  bf16 1x4096x4096 7.1 to 7.8
// us, 4.3 to 4.7 TB/s of W.
constexpr int FEW_WAVES = 8, FEW_STEPS = 4;  // steps in flight per wave
template <typename T, int MT, bool ANY>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_linear_few(LinearArgs a) {
  constexpr int C = CHUNK<T>, ES = (int)sizeof(T), BK = STEP<T>;
  constexpr int EACH = (MT * 256 + FEW_WAVES * 64 - 1) / (FEW_WAVES * 64);  // results per thread
  __shared__ float red[FEW_WAVES][MT][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, fr = lane & 15, fg = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int rows = (int)min((int64_t)(16 * MT), a.M - m0);
  const LinearArgs t = from<T>(a, m0, n0);
  auto result = [&](int e, int& m, int& n) __attribute__((always_inline)) -> bool {
    const int i = e * FEW_WAVES * 64 + tid;
    m = i / 16;
    n = i % 16;
    return i < MT * 256 && m < rows && n < t.N;
  };
  Fetched1 f[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    int m, n;
    if (result(e, m, n)) f[e] = fetch1<T>(t, m, n);
  }
  const char* xr[MT];  // the lane's rows (null: none)
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = i * 16 + fr < rows ? (const char*)a.A + (m0 + i * 16 + fr) * a.lda * ES : nullptr;
  const char* wr = n0 + fr < a.N ? (const char*)a.B + (int64_t)(n0 + fr) * a.ldb * ES : nullptr;
  auto chunk = [&](const char* row, int k) __attribute__((always_inline)) -> u32x4_t {
    const int n = a.K - k;
    u32x4_t u = {0u, 0u, 0u, 0u};
    if (row && n > 0) {
      if constexpr (ANY) u = ld_any<T>(row + (int64_t)k * ES, n);
      else u = *reinterpret_cast<const u32x4_t*>(row + (int64_t)k * ES);  // (K is whole chunks)
    }
    return u;
  };
  f32x4_t acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  const int steps = (a.K + BK - 1) / BK;
  for (int s0 = wave; s0 < steps; s0 += FEW_WAVES * FEW_STEPS) {
    // 16 x 16 x (4 chunks): lane l holds row l % 16 and chunk l / 16, in both operands
    u32x4_t x[FEW_STEPS][2][MT], w[FEW_STEPS][2];
#pragma unroll
    for (int u = 0; u < FEW_STEPS; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (s0 + u * FEW_WAVES) * BK + (h * 4 + fg) * C;
        w[u][h] = chunk(wr, k);
#pragma unroll
        for (int i = 0; i < MT; ++i) x[u][h][i] = chunk(xr[i], k);
      }
#pragma unroll
    for (int u = 0; u < FEW_STEPS; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if constexpr (ES == 2) {
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x[u][h][i]),
                                                             __builtin_bit_cast(bf16x8_t, w[u][h]), acc[i], 0, 0, 0);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[u][h][i][q]), __uint_as_float(w[u][h][q]),
                                                            acc[i], 0, 0, 0);
          }
        }
  }
  // 16x16 result: lane l, register r holds row 4 (l / 16) + r, column l % 16
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) red[wave][i][(4 * fg + r) * 16 + fr] = acc[i][r];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    int m, n;
    if (!result(e, m, n)) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) v += red[w][m >> 4][(m & 15) * 16 + n];
    finish1<T>(t, m, n, v, f[e]);
  }
}

// ---------------------------------------------------------------- packing
// Operands whose rows do not start at multiples of 16 bytes, or end inside a
// chunk of the reduction, are copied to rows of whole chunks (zeros behind the
// columns), all of a call's in one launch.  Loads of 16 unaligned bytes straight
// into the products took four times an aligned product's time (2001x2001x2001 98 us, packed 38, aligned 25).
struct PackArgs {
  int count;
  const void* src[3];
  void* dst[3];
  int64_t ld[3], rows[3];           // source pitch (elements), rows
  int cols[3], per_row[3], log[3];  // columns, chunks per packed row, log2 of the lanes that take a row
  int first[3], blocks;             // first workgroup, and their number
};
// Bound by its launch at the sizes where it counts (1001x999x1333 backward, 15 MB read
// and written: 6.3 to 8.1 us).
template <typename T>
__global__ __launch_bounds__(256) void k_linear_pack(PackArgs a) {
  constexpr int C = CHUNK<T>, ES = (int)sizeof(T);
  int m = 0;
#pragma unroll
  for (int q = 1; q < 3; ++q)
    if (q < a.count && (int)blockIdx.x >= a.first[q]) m = q;
  // 2^log lanes take a row
  const int log = a.log[m], per = a.per_row[m], cols = a.cols[m];
  const int64_t r = ((int64_t)((int)blockIdx.x - a.first[m]) * 256 + threadIdx.x) >> log;
  if (r >= a.rows[m]) return;
  const char* row = (const char*)a.src[m] + r * a.ld[m] * ES;
  u32x4_t* dst = reinterpret_cast<u32x4_t*>(a.dst[m]) + r * per;
#pragma unroll 2
  for (int j = threadIdx.x & ((1 << log) - 1); j < per; j += 1 << log) {
    const int c = j * C, n = min(C, cols - c);
    const char* p = row + (int64_t)c * ES;
    dst[j] = ld_any<T>(p, n);
  }
}

// ---------------------------------------------------------------- activation gradient
// dz may be dy or z: no pointer is __restrict__.
// Bound by memory: 2^26 elements behind a GELU 70 us in bf16, 5.8 TB/s, 137 in fp32, 5.9.
template <typename T>
__global__ __launch_bounds__(256) void k_act_bwd(const T* dy, const T* z, T* dz, int64_t n, int act, int vec) {
  constexpr int C = CHUNK<T>;
  const int64_t chunks = (n + C - 1) / C;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int left = (int)min((int64_t)C, n - i * C);
    const bool v = vec && left == C;
    float g[C], zz[C];
    unpack<T>(ld_chunk<T>(dy + i * C, v, left), g);
    unpack<T>(ld_chunk<T>(z + i * C, v, left), zz);
    act_slopes<T>(g, zz, act);
    st_chunk<T>(dz + i * C, v, left, g);
  }
}

int grid_of(int64_t items) { return (int)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 1 << 16)); }

// ---------------------------------------------------------------- plan
// What a launch costs, in us, fitted to 500 timed products of 76 shapes (MI355X; a
// step is 128 bytes of the reduction): per step and workgroup alone on its CU, per
// step of two that share a CU (one 256x256 tile fills it), and the rest of a
// workgroup (prologue and epilogue).  Products of up to a few workgroups per CU
// are bound by the length of their chains, not by rates.  The choice by these
// costs was on average 3% (bf16) and 1% (fp32) slower than the fastest of all
// tiles and splits timed: e.g. 512x1024x4096 64x64 9.2 us, 128x128 13.2, 64x64
// in two splits 24; 4096x2048x4096 256x256 68, 128x128 73; weight gradient
// 8192x1024x1024 128x128 in eight splits 36, in one 66.
struct TileCost {
  int tile;
  double alone, pair, alone_rest, pair_rest;
};
constexpr TileCost COST_BF16[] = {{64, 0.29, 0.41, 2.1, 2.1}, {128, 0.63, 0.93, 3.1, 5.8}, {256, 1.46, 2.92, 8.2, 16.4}};
constexpr TileCost COST_F32[] = {{64, 0.56, 1.05, 0.0, 1.3}, {128, 2.0, 3.7, 3.5, 3.9}};
// the join of splits: its launch, and the partial sums' traffic per MB of fp32 results
constexpr double JOIN_US = 4.6, JOIN_US_PER_MB = 0.134;
constexpr int MAX_SPLITS = 16;

double pick(int dtype, int64_t M, int N, int64_t steps, int* tile, int* splits) {
  const TileCost* cost = dtype == DT_BF16 ? COST_BF16 : COST_F32;
  const int tiles = dtype == DT_BF16 ? 3 : 2;
  double best = 0.0;
  *tile = 0;
  for (int i = 0; i < tiles; ++i) {
    const int b = cost[i].tile;
    const int64_t count = ((M + b - 1) / b) * ((N + b - 1) / b);
    for (int s = 1; s <= MAX_SPLITS && (s == 1 || 2 * s <= steps); s *= 2) {
      const int64_t per = (steps + s - 1) / s, blocks = (count * ((steps + per - 1) / per) + 255) / 256;
      if (blocks >= 1 << 15 && i + 1 < tiles) continue;  // a launch has fewer than 2^32 threads
      double t = (double)(blocks / 2) * (cost[i].pair * per + cost[i].pair_rest) +
                 (double)(blocks % 2) * (cost[i].alone * per + cost[i].alone_rest);
      if (s > 1) t += JOIN_US + JOIN_US_PER_MB * 4e-6 * (double)M * N * (2 * s + 1);
      if (*tile == 0 || t < best) {
        best = t;
        *tile = b;
        *splits = s;
      }
    }
  }
  return best;
}

template <typename T, int EPI>
hipError_t join(const LinearArgs& a, hipStream_t s) {
  XP_LAUNCH("k_linear_join", 4.0 * a.M * a.N * a.splits, (k_linear_join<T, EPI>),
            dim3(grid_of(a.M * ((a.N + CHUNK<T> - 1) / CHUNK<T>))), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int BM, int BN, int WM, int WN, int NS, bool TA, bool TB, int EPI>
hipError_t go(const LinearArgs& a, hipStream_t s) {
  const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  static const struct Name {
    char s[64];
    Name() { snprintf(s, sizeof s, "k_linear<%s,%d,%d,%s>", sizeof(T) == 2 ? "bf16" : "f32", BM, BN,
                      EPI == LIN_FWD ? "fwd" : EPI == LIN_DATA ? "data" : "grad"); }
  } name;
  XP_LAUNCH(name.s, 2.0 * a.M * a.N * a.K, (k_linear<T, BM, BN, WM, WN, NS, TA, TB, EPI>),
            dim3((unsigned)(tm * tn * a.splits)), dim3(WM * WN * 64), 0, s, a, (int)tm, (int)tn);
  hipError_t e = hipGetLastError();
  return e != hipSuccess || !a.part ? e : join<T, EPI>(a, s);
}

template <typename T, int B, int NS>
hipError_t go_bwd(const LinearArgs& d, const LinearArgs& g, hipStream_t s) {
  const int64_t tmd = (d.M + B - 1) / B, tnd = (d.N + B - 1) / B, tmg = (g.M + B - 1) / B, tng = (g.N + B - 1) / B;
  // the product with more of the reduction per workgroup first: at the end the short ones fill the CUs evenly
  const int64_t nd = tmd * tnd * d.splits, ng = tmg * tng * g.splits;
  const bool grad_first = g.kper > d.kper;
  static const struct Name {
    char s[64];
    Name() { snprintf(s, sizeof s, "k_linear_bwd<%s,%d>", sizeof(T) == 2 ? "bf16" : "f32", B); }
  } name;
  XP_LAUNCH(name.s, 2.0 * d.M * d.N * d.K + 2.0 * g.M * g.N * g.K, (k_linear_bwd<T, B, NS>),
            dim3((unsigned)(nd + ng)), dim3(256), 0, s, d, (int)tmd, (int)tnd, (int)(grad_first ? ng : nd), (int)grad_first,
            g, (int)tmg, (int)tng);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && d.part) e = join<T, LIN_DATA>(d, s);
  if (e == hipSuccess && g.part) e = join<T, LIN_GRAD>(g, s);
  return e;
}

// Buffers: two, which leaves room for two 128x128 or four 64x64 tiles on a CU.
// 128x128: four buffers and one tile were 0 to 5% slower.  64x64 in bf16: with up to
// two tiles per CU and more than a few steps there is nothing else to hide the copies'
// time behind, and four are faster (over 200 timed products: 16 to 32 steps 1.10 to
// 1.20 of four's time with two, more steps 1.26 to 1.32; up to 8 steps the same; more
// than two tiles per CU 0.86 to 0.97).
constexpr int NS_128 = 2;
template <typename T>
bool deep(int64_t groups, int64_t k) { return sizeof(T) == 2 && groups <= 512 && k > 8 * STEP<T>; }
template <typename T, bool TA, bool TB, int EPI>
hipError_t by_tile(const LinearArgs& a, int tile, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (tile == 256) return go<T, 256, 256, 2, 4, 2, TA, TB, EPI>(a, s);
  }
  if (tile == 128) return go<T, 128, 128, 2, 2, NS_128, TA, TB, EPI>(a, s);
  if constexpr (sizeof(T) == 2) {
    if (deep<T>((a.M + 63) / 64 * ((a.N + 63) / 64) * a.splits, a.kper)) return go<T, 64, 64, 2, 2, 4, TA, TB, EPI>(a, s);
  }
  return go<T, 64, 64, 2, 2, 2, TA, TB, EPI>(a, s);
}

template <typename T>
hipError_t both(const LinearArgs& d, const LinearArgs& g, int tile, hipStream_t s) {
  return tile == 128 ? go_bwd<T, 128, NS_128>(d, g, s) : go_bwd<T, 64, 2>(d, g, s);
}

template <typename T>
hipError_t by_kind(const LinearArgs& a, int tile, hipStream_t s) {
  if (a.epi == LIN_FWD) return by_tile<T, false, false, LIN_FWD>(a, tile, s);
  if (a.epi == LIN_DATA) return by_tile<T, false, true, LIN_DATA>(a, tile, s);
  return by_tile<T, true, true, LIN_GRAD>(a, tile, s);
}

struct Plan {
  int tile, splits;
  double us;
  int64_t kper, ldpart;
  size_t part_b, bytes;  // offset of the bias gradient's partial sums, workspace
};
Plan plan(int dtype, const LinearArgs& a) {
  Plan p{};
  const int bk = dtype == DT_BF16 ? STEP<bf16_t> : STEP<float>;
  const int64_t steps = ((int64_t)a.K + bk - 1) / bk;
  p.us = pick(dtype, a.M, a.N, steps, &p.tile, &p.splits);
  p.kper = (steps + p.splits - 1) / p.splits * bk;
  p.splits = (int)(((int64_t)a.K + p.kper - 1) / p.kper);  // those that hold something
  if (p.splits == 1) return p;
  p.ldpart = (a.N + 7) / 8 * 8;
  p.part_b = ((size_t)p.splits * a.M * p.ldpart * sizeof(float) + 255) / 256 * 256;
  p.bytes = p.part_b + (a.grad_b ? (size_t)p.splits * a.M * sizeof(double) : 0);
  return p;
}

// The forwards that k_linear_few takes: those for which it costs less than the
// tiles (and, where operands are not aligned, packing them).  Its cost, in us: sets of
// four workgroups per CU, in each of which the waves take 32 steps at a time, with a
// time for them that grows with the rows; what the workgroups read through L2 (twice
// where chunks are put together from two; half as much again where rows cross
// cache lines); W from memory.  Packing reads and writes both operands.  A call's host
// time is a floor under both sides: one launch, or two and a workspace.
// Measured, tiles in brackets: bf16 1x4096x4096 7.6 (13.3), 16x4096x4096 10.0 (13.2),
// 32x4096x4096 13.6 (14.8), 16x8192x2048 16.6 (13.7), 32x8192x8192 45.5 (26.3),
// 1x8192x8192 26.4 (25.1); fp32 1x8192x8192 53 (72), 32x8192x8192 111 (77);
// with packing 137x57x128 7.8 (12.4), 300x300x300 8.2 (14.5), 500x4097x100 30.6 (18.0),
// fp32 777x1030x515 53.5 (25.6); bf16 16x1003x16384 18 (24), 24x1003x16384 37 (25),
// 8x4099x2048 19 (21), 8x4099x8192 29 (42), 8x12815x2048 67 (38), 8x12815x16384 172 (258),
// fp32 8x4099x2048 40 (32), 8x12815x16384 333 (554).
// Next to where both sides cost the same the estimates (off by up to 10% each) choose
// wrongly: bf16 8x12815x4096 is taken at 68 (59), 32x4096x4096 left at 14.8 for 13.6.
constexpr double FEW_US = 2.0, FEW_ROUND_US = 2.3, FEW_ROW_US = 0.1, FEW_L2_MB_PER_US = 8.8, FEW_W_MB_PER_US = 5.3;
constexpr double FEW_ANY_SET_US[2] = {9.5, 11.0}, FEW_ANY_ROWS[2] = {13.0, 48.0};  // up to 16 rows, 32
constexpr double PACK_US = 6.0, PACK_MB_PER_US = 5.0, ONE_LAUNCH_US = 7.5, TWO_LAUNCHES_US = 13.0;
bool takes_few(const LinearArgs& a, int es, bool any, const Plan& tiles) {
  if (a.epi != LIN_FWD || (!any && a.M > 32) || (a.M + 31) / 32 > 65535) return false;
  const double steps = ((int64_t)a.K * es + 127) / 128, groups = (double)((a.M + 31) / 32) * ((a.N + 15) / 16);
  const double rows = any ? FEW_ANY_ROWS[a.M > 16] : a.M <= 16 ? (double)a.M : 32.0, row_mb = (double)a.K * es * 1e-6;
  const double set = any ? FEW_ANY_SET_US[a.M > 16] : FEW_ROUND_US + FEW_ROW_US * rows;
  const double lines = any ? 2.0 : (a.lda * es | a.ldb * es) % 128 ? 1.5 : 1.0;
  const double chain = (FEW_US + steps / (FEW_WAVES * FEW_STEPS) * set) * (double)(((int64_t)groups + 1023) / 1024);
  const double read = FEW_US + std::max(groups * (16.0 + rows) * row_mb * lines / FEW_L2_MB_PER_US, a.N * row_mb / FEW_W_MB_PER_US);
  // packing: both operands (of few rows nearly all is W), read and written
  const double pack = any ? PACK_US + 2.0 * (double)(a.M + a.N) * row_mb / PACK_MB_PER_US : 0.0;
  const bool two = any || tiles.splits > 1;
  return std::max({chain, read, ONE_LAUNCH_US}) <=
         std::max(tiles.us + pack, two ? TWO_LAUNCHES_US : ONE_LAUNCH_US);
}
template <typename T, int MT, bool ANY>
hipError_t go_few(const LinearArgs& a, hipStream_t s) {
  XP_LAUNCH(sizeof(T) == 2 ? "k_linear_few<bf16>" : "k_linear_few<f32>", 2.0 * a.M * a.N * a.K, (k_linear_few<T, MT, ANY>),
            dim3((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), dim3(FEW_WAVES * 64), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t few(const LinearArgs& a, bool any, hipStream_t s) {
  if (a.M <= 16) return any ? go_few<T, 1, true>(a, s) : go_few<T, 1, false>(a, s);
  return any ? go_few<T, 2, true>(a, s) : go_few<T, 2, false>(a, s);
}

bool chunked(const void* p, int64_t ld, int chunk) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % chunk == 0;
}

// a forward's operands: a reduction along their rows has to end with a chunk
bool unaligned(const LinearArgs& a, int chunk) {
  return !chunked(a.A, a.lda, chunk) || !chunked(a.B, a.ldb, chunk) || a.K % chunk != 0;
}

}  // namespace

// A call's products with their packed operands: where those and the products' partial
// sums lie in the workspace.
namespace {
struct Call {
  LinearArgs p[2];
  PackArgs pack;
  size_t parts[2], bytes;
  bool few;
};
Call lay_out(int dtype, const LinearArgs* in, int n, char* ws) {
  Call c{};
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  c.few = in[0].M > 0 && takes_few(in[0], es, unaligned(in[0], chunk), plan(dtype, in[0]));
  if (c.few) {
    c.p[0] = in[0];
    return c;
  }
  auto operand = [&](const void*& ptr, int64_t& ld, int64_t rows, int cols, bool must) {
    PackArgs& k = c.pack;
    int at = 0;
    while (at < k.count && !(k.src[at] == ptr && k.ld[at] == ld && k.cols[at] == cols && k.rows[at] == rows)) ++at;
    if (at == k.count) {
      if (!must) return;
      k.rows[at] = rows;
      k.src[at] = ptr;
      k.ld[at] = ld;
      k.cols[at] = cols;
      k.per_row[at] = (cols + chunk - 1) / chunk;
      // (a launch has fewer than 2^32 threads)
      while (k.log[at] < 8 && 1 << k.log[at] < k.per_row[at] && rows << k.log[at] < (int64_t)1 << 29) ++k.log[at];
      k.first[at] = k.blocks;
      k.blocks += (int)(((rows << k.log[at]) + 255) / 256);
      k.dst[at] = ws + c.bytes;
      c.bytes += ((size_t)rows * k.per_row[at] * 16 + 255) / 256 * 256;
      ++k.count;
    }
    ptr = k.dst[at];
    ld = (int64_t)k.per_row[at] * chunk;
  };
  for (int i = 0; i < n; ++i) {
    LinearArgs& a = c.p[i];
    a = in[i];
    if (a.M <= 0) continue;
    const bool ta = a.epi == LIN_GRAD, tb = a.epi != LIN_FWD, tail = a.K % chunk != 0;
    // a reduction along an operand's rows has to end with a chunk
    operand(a.A, a.lda, ta ? a.K : a.M, ta ? (int)a.M : a.K, !chunked(a.A, a.lda, chunk) || (!ta && tail));
    operand(a.B, a.ldb, tb ? a.K : a.N, tb ? a.N : a.K, !chunked(a.B, a.ldb, chunk) || (!tb && tail));
  }
  for (int i = 0; i < n; ++i) {
    c.parts[i] = c.bytes;
    if (c.p[i].M > 0) c.bytes += (plan(dtype, c.p[i]).bytes + 255) / 256 * 256;
  }
  return c;
}
}  // namespace

size_t linear_bytes(int dtype, const LinearArgs* products, int n) { return lay_out(dtype, products, n, nullptr).bytes; }

hipError_t launch_linear(int dtype, const LinearArgs* products, int n, void* workspace, hipStream_t s) {
  const Call c = lay_out(dtype, products, n, (char*)workspace);
  const int chunk = dtype == DT_BF16 ? CHUNK<bf16_t> : CHUNK<float>;
  if (c.few) {
    const LinearArgs& a = c.p[0];
    const bool any = unaligned(a, chunk);
    return dtype == DT_BF16 ? few<bf16_t>(a, any, s) : few<float>(a, any, s);
  }
  if (c.pack.count > 0) {
    const dim3 grid((unsigned)c.pack.blocks);
    const double bytes = 2.0 * c.parts[0];
    if (dtype == DT_BF16) XP_LAUNCH("k_linear_pack<bf16>", bytes, k_linear_pack<bf16_t>, grid, dim3(256), 0, s, c.pack);
    else XP_LAUNCH("k_linear_pack<f32>", bytes, k_linear_pack<float>, grid, dim3(256), 0, s, c.pack);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  LinearArgs a[2];
  int tile[2] = {0, 0};
  for (int i = 0; i < n; ++i) {
    if (c.p[i].M <= 0) continue;
    LinearArgs& q = a[i];
    q = c.p[i];
    const Plan p = plan(dtype, q);
    char* parts = (char*)workspace + c.parts[i];
    tile[i] = p.tile;
    q.splits = p.splits;
    q.kper = p.kper;
    q.ldpart = p.ldpart;
    q.ldg = q.N;
    q.part = p.splits > 1 ? (float*)parts : nullptr;
    q.part_b = p.splits > 1 ? (double*)(parts + p.part_b) : nullptr;
    q.vec = q.epi == LIN_GRAD
                ? chunked(q.grad, q.N, 4)
                : chunked(q.y, q.ldy, chunk) && (!q.res || chunked(q.res, q.ldr, chunk)) &&
                      (!q.z_in || chunked(q.z_in, q.ldz, chunk)) && (!q.z_out || chunked(q.z_out, q.ldz, chunk));
  }
  // (256x256 tiles fill the GPU by themselves)
  if (tile[0] == tile[1] && tile[0] > 0 && tile[0] <= 128)
    return dtype == DT_BF16 ? both<bf16_t>(a[0], a[1], tile[0], s) : both<float>(a[0], a[1], tile[0], s);
  for (int i = 0; i < n; ++i) {
    if (tile[i] == 0) continue;
    hipError_t e = dtype == DT_BF16 ? by_kind<bf16_t>(a[i], tile[i], s) : by_kind<float>(a[i], tile[i], s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_act_bwd(int dtype, const void* dy, const void* z, void* dz, int64_t n, int act, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int chunk = dtype == DT_BF16 ? 8 : 4;
  const int vec = chunked(dy, 0, 1) && chunked(z, 0, 1) && chunked(dz, 0, 1);
  if (dtype == DT_BF16)
    XP_LAUNCH("k_act_bwd<bf16>", 6.0 * n, k_act_bwd<bf16_t>, dim3(grid_of((n + chunk - 1) / chunk)), dim3(256), 0, s,
              (const bf16_t*)dy, (const bf16_t*)z, (bf16_t*)dz, n, act, vec);
  else
    XP_LAUNCH("k_act_bwd<f32>", 12.0 * n, k_act_bwd<float>, dim3(grid_of((n + chunk - 1) / chunk)), dim3(256), 0, s,
              (const float*)dy, (const float*)z, (float*)dz, n, act, vec);
  return hipGetLastError();
}

}  // namespace xp
