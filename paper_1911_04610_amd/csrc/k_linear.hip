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
// product before it has fp32 sums.  erff and expf are correct to a few 2^-24.
template <int N>
XP_DEV void act_values(float (&z)[N], int act) {
  if (act == LIN_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] > 0.f ? z[i] : (z[i] != z[i] ? z[i] : 0.f);
  } else if (act == LIN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = 0.5f * z[i] * (1.f + erff(z[i] * 0.70710678118654752f));
  } else if (act == LIN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] / (1.f + expf(-z[i]));
  }
}

// v *= act'(z); 0 at 0 for the ReLU
template <int N>
XP_DEV void act_slopes(float (&v)[N], const float (&z)[N], int act) {
  if (act == LIN_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= z[i] > 0.f ? 1.f : 0.f;
  } else if (act == LIN_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] *= 0.5f * (1.f + erff(z[i] * 0.70710678118654752f)) + z[i] * 0.39894228040143268f * expf(-0.5f * z[i] * z[i]);
  } else if (act == LIN_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float s = 1.f / (1.f + expf(-z[i]));
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
// the same element by element, the first n of them
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
template <typename T>
XP_DEV u32x4_t ld_chunk(const T* p, bool vec, int n) {
  return vec ? *reinterpret_cast<const u32x4_t*>(p) : ld_some<T>(p, n);
}
template <typename T>
XP_DEV void st_chunk(T* p, bool vec, int n, const float (&v)[CHUNK<T>]) {
  if (vec) *reinterpret_cast<u32x4_t*>(p) = pack<T>(v);
  else st_some<T>(p, n, v);
}

// What the epilogue of columns n .. n + CHUNK<T> of row m reads: the residual and the
// pre-activation, or (LIN_GRAD) the accumulators
struct Fetched {
  u32x4_t r, z;
};
template <typename T, int EPI>
XP_DEV Fetched fetch(const LinearArgs& a, int64_t m, int n) {
  const int left = a.N - n;
  const bool vec = a.vec && left >= CHUNK<T>;
  Fetched f;
  if constexpr (EPI == LIN_GRAD) {
    const float* g = a.grad + m * a.N + n;
    f.r = ld_chunk<float>(g, vec, left);
    if constexpr (sizeof(T) == 2) f.z = ld_chunk<float>(g + 4, vec, left - 4);
  } else {
    if (a.res) f.r = ld_chunk<T>((const T*)a.res + m * a.ldr + n, vec, left);
    if (EPI == LIN_DATA && a.z_in) f.z = ld_chunk<T>((const T*)a.z_in + m * a.ldz + n, vec, left);
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
XP_DEV void finish(const LinearArgs& a, int64_t m, int n, float (&v)[CHUNK<T>], const float (&b)[CHUNK<T>], const Fetched& f) {
  constexpr int C = CHUNK<T>;
  const int left = a.N - n;
  const bool vec = a.vec && left >= C;
  if constexpr (EPI == LIN_GRAD) {
    // fp32 accumulators whatever T
    float* g = a.grad + m * a.N + n;
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
    if (a.z_out) st_chunk<T>((T*)a.z_out + m * a.ldz + n, vec, left, v);
    act_values(v, a.act);
  } else if (a.z_in) {
    float z[C];
    unpack<T>(f.z, z);
    act_slopes(v, z, a.act);
  }
  if (a.res) {
    float r[C];
    unpack<T>(f.r, r);
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += r[i];
  }
  st_chunk<T>((T*)a.y + m * a.ldy + n, vec, left, v);
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

// One workgroup per BM x BN tile of the product and part of the reduction, WM x
// WN waves of 32x32 MFMA results.  Both operands are copied from memory
// straight into LDS, one step (128 bytes of the reduction) at a time, with two
// buffers: one step is in flight while one is multiplied.
template <typename T, int BM, int BN, int WM, int WN, bool TA, bool TB, int EPI>
__global__ __launch_bounds__(WM * WN * 64) void k_linear(LinearArgs a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, ES = (int)sizeof(T), C = CHUNK<T>, BK = STEP<T>;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static_assert(WTM % 32 == 0 && WTN % 32 == 0, "wave tile");
  constexpr int A_I = BM / 8 / NW, B_I = BN / 8 / NW;  // copies of 1 KB per wave and step
  static_assert(A_I * NW * 8 == BM && B_I * NW * 8 == BN, "whole copies per wave");
  constexpr int SZ = (BM + BN) * 128;
  __shared__ __align__(16) unsigned char st0[SZ];
  __shared__ __align__(16) unsigned char st1[SZ];
  auto stage = [&](auto I) __attribute__((always_inline)) -> unsigned char* {
    if constexpr (decltype(I)::value == 0) return st0;
    else return st1;
  };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // tile order: runs of 8 tile rows, so that the tiles that one XCD holds at a
  // time share rows of both operands in its L2
  const int lin = xcd_tile(blockIdx.x, gridDim.x);
  const int split = lin / (tiles_m * tiles_n), t = lin - split * tiles_m * tiles_n;
  const int grp = t / (8 * tiles_n), gm = min(8, tiles_m - grp * 8), in = t - grp * 8 * tiles_n;
  const int tm = grp * 8 + in % gm, tn = in / gm;
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;
  const int64_t kbeg = (int64_t)split * a.kper;
  const int64_t kend = min((int64_t)a.K, kbeg + a.kper);
  const int nk = (int)((kend - kbeg + BK - 1) / BK);

  // Per copy the lane's byte offset from the step's base, ~0 where its row (TR:
  // its column chunk) is past the operand; the base moves by one step at a time, and
  // reduction indices past the end are masked step by step.  So every chunk that
  // is read holds an element of the operand (a 16-byte chunk never leaves that
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
  auto copy = [&](auto I) __attribute__((always_inline)) {  // past the last step: zeros
    unsigned char* sa = stage(I);
    unsigned char* sb = stage(I) + BM * 128;
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void*)abase, (short)0, 0x7ffffff0, 0x00020000);
    const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc((void*)bbase, (short)0, 0x7ffffff0, 0x00020000);
#pragma unroll
    for (int i = 0; i < A_I; ++i)
      load_lds16(ar, (bf16_t*)(sa + (wave * A_I + i) * 1024), a_k[i] < left ? (int)a_off[i] : -1, 0);
#pragma unroll
    for (int i = 0; i < B_I; ++i)
      load_lds16(br, (bf16_t*)(sb + (wave * B_I + i) * 1024), b_k[i] < left ? (int)b_off[i] : -1, 0);
    abase += astep;
    bbase += bstep;
    left -= BK;
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
  // it reads, and waits for no copies into the other.)
  auto frag = [&](auto I, auto TR, auto W, int base, int row0, int kk) __attribute__((always_inline)) -> u32x4_t {
    constexpr int w = decltype(W)::value;
    const unsigned char* lds = stage(I);
    if constexpr (!decltype(TR)::value) {
      return *reinterpret_cast<const u32x4_t*>(lds + (base + (row0 + fr) * 128 + (((kk * 2 + fh) ^ (fr >> 1 & 7)) << 4)));
    } else {
      u32x4_t v;
      const int k = 4 * fh, c = row0 + fr;
      const int at = base + (kk * 8 + k) * (w * 4) + (((c >> 2) ^ tr_swz<T, w>(k)) << 4) + (c & 3) * 4;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const uint32_t*>(lds + (at + q * w * 4));
      return v;
    }
  };
  // Two sets of fragments: while the products of one quarter of a step run, the next
  // quarter's fragments are read.
  u32x4_t fa[2][TM], fb[2][TN];
  // where the lane's transposing reads of a quarter start (of the first quarter, in the first stage's array)
  constexpr int TRN = ES == 2 ? (TA ? TM : 0) + (TB ? TN : 0) : 0;
  uint32_t tr_at[TRN > 0 ? TRN : 1];
  if constexpr (TRN > 0) {
    static_assert(BM == BN, "one offset for both operands' rows");
    auto at = [&](int base, int row0) __attribute__((always_inline)) -> uint32_t {
      const int k = 8 * fh + ((lane & 15) >> 2);  // the first read's row (the swizzle takes it modulo 4)
      const int c = row0 + 16 * (fr >> 4) + 4 * (lane & 3);
      return base + k * (BM * 2) + (((c >> 3) ^ tr_swz<T, BM>(k)) << 4) + (c & 7) * 2;
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
    if constexpr (!(ES == 2 && TB)) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
        fb[set][j] = frag(I, std::bool_constant<TB>{}, std::integral_constant<int, BN>{}, BM * 128, wn * WTN + j * 32, kk);
    }
    if constexpr (!(ES == 2 && TA)) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
        fa[set][i] = frag(I, std::bool_constant<TA>{}, std::integral_constant<int, BM>{}, 0, wm * WTM + i * 32, kk);
    }
    if constexpr (TRN > 0) {
      const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)stage(I);
      uint32_t at[TRN];
      u32x4_t out[TRN];
#pragma unroll
      for (int i = 0; i < TRN; ++i) at[i] = lds + tr_at[i];
      read_tr<TRN, kk * 16 * BM * 2, 4 * BM * 2>(at, out);
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
  // compiler can move are spread over the products; a block of transposing reads
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
      constexpr int PER = TM * TN * (ES == 2 ? 1 : 4), READS = TM * (TA ? 4 : 1) + TN * (TB ? 4 : 1);
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

  // Step k from buffer k % 2.  By its last quarter all of the step's fragments
  // are in registers: past the barrier there the buffer takes the copies of step
  // k + 2, and the first fragments of step k + 1, whose copies have had a step's time
  // to land, are read while the last quarter is multiplied.
  constexpr std::integral_constant<int, 0> B0{};
  copy(B0);
  copy(std::integral_constant<int, 1>{});
  wait_step<A_I + B_I>();
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
  while (++k < nk) {
    bool done = false;
    static_for<0, 2>([&](auto I) __attribute__((always_inline)) {
      if (!done) {
        constexpr std::integral_constant<int, 1 - decltype(I)::value> NEXT{};
        // this wave's copies of step k have landed and its reads of step k - 1
        // returned; past the barrier so have the others'
        wait_step<0>();
        copy(I);
        overlap(NEXT, B0, 0, 1);
        quarters(NEXT);
        if (decltype(I)::value == 0) done = ++k == nk;
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
  static_assert(NW * 16 * PITCH * 4 <= SZ, "strips");
  float* strip = reinterpret_cast<float*>(st0) + wave * 16 * PITCH;
  constexpr int CW = WTN / C, RP = 64 / CW, PASS = 16 / RP;  // chunks per strip row, rows per pass
  const int ch = lane % CW;
  const int n = n0 + wn * WTN + ch * C;
  const bool direct = !a.part;
  float bias[C];
  fetch_bias<T, EPI>(a, n, bias);
  auto row_of = [&](int s, int p) __attribute__((always_inline)) -> int64_t {
    const int64_t m = m0 + wm * WTM + s * 16 + p * RP + lane / CW;
    return m < a.M && n < a.N ? m : -1;
  };
  Fetched next[PASS];
  auto prefetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const int64_t m = row_of(s, p);
      if (direct && m >= 0) next[p] = fetch<T, EPI>(a, m, n);
    }
  };
  prefetch(0);
  static_for<0, TM * 2>([&](auto S) __attribute__((always_inline)) {
    constexpr int s = decltype(S)::value;
    Fetched now[PASS];
#pragma unroll
    for (int p = 0; p < PASS; ++p) now[p] = next[p];
    if constexpr (s + 1 < TM * 2) prefetch(s + 1);
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 8; ++r)
        strip[(8 * (r >> 2) + 4 * fh + (r & 3)) * PITCH + j * 32 + fr] = acc[s >> 1][j][(s & 1) * 8 + r];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const int64_t m = row_of(s, p);
      float v[C];
#pragma unroll
      for (int q = 0; q < C / 4; ++q) {
        const f32x4_t f = *reinterpret_cast<const f32x4_t*>(strip + (p * RP + lane / CW) * PITCH + ch * C + q * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[q * 4 + i] = f[i];
      }
      if (m < 0) continue;
      if (direct) {
        finish<T, EPI>(a, m, n, v, bias, now[p]);
      } else {
        // partial sums, rows of N rounded up to whole chunks
        float* out = a.part + ((int64_t)split * a.M + m) * a.ldpart + n;
#pragma unroll
        for (int q = 0; q < C / 4; ++q)
          *reinterpret_cast<f32x4_t*>(out + 4 * q) = (f32x4_t){v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      }
    }
    __builtin_amdgcn_wave_barrier();
  });
}

// the splits' partial sums added in order, and the epilogue
template <typename T, int EPI>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  constexpr int C = CHUNK<T>;
  const int cpr = (a.N + C - 1) / C;
  const int64_t total = a.M * cpr;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / cpr;
    const int n = (int)(i - m * cpr) * C;
    float v[C];
#pragma unroll
    for (int q = 0; q < C; ++q) v[q] = 0.f;
    const float* p = a.part + m * a.ldpart + n;
    for (int s = 0; s < a.splits; ++s, p += a.M * a.ldpart) {
#pragma unroll
      for (int q = 0; q < C / 4; ++q) {
        const f32x4_t f = *reinterpret_cast<const f32x4_t*>(p + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] += f[e];
      }
    }
    float b[C];
    fetch_bias<T, EPI>(a, n, b);
    finish<T, EPI>(a, m, n, v, b, fetch<T, EPI>(a, m, n));
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

// ---------------------------------------------------------------- packing
// Rows whose chunks do not start at multiples of 16 bytes, or end inside a
// chunk of the reduction, are copied to rows of whole chunks, zeros behind.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_pack(const T* __restrict__ src, int64_t ld, int64_t rows, int cols,
                                                     T* __restrict__ dst, int cols_out) {
  const int64_t total = rows * cols_out;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cols_out;
    const int c = (int)(i - r * cols_out);
    dst[i] = c < cols ? src[r * ld + c] : T(0);
  }
}

// ---------------------------------------------------------------- activation gradient
template <typename T>
__global__ __launch_bounds__(256) void k_act_bwd(const T* __restrict__ dy, const T* __restrict__ z, T* __restrict__ dz,
                                                 int64_t n, int act, int vec) {
  constexpr int C = CHUNK<T>;
  const int64_t chunks = (n + C - 1) / C;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int left = (int)min((int64_t)C, n - i * C);
    const bool v = vec && left == C;
    float g[C], zz[C];
    unpack<T>(ld_chunk<T>(dy + i * C, v, left), g);
    unpack<T>(ld_chunk<T>(z + i * C, v, left), zz);
    act_slopes(g, zz, act);
    st_chunk<T>(dz + i * C, v, left, g);
  }
}

int grid_of(int64_t items) { return (int)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 1 << 16)); }

// ---------------------------------------------------------------- plan
struct Tile {
  int bm, bn;
};

// tile and splits of a product of M x N results over K
void pick(int dtype, int64_t M, int N, int K, Tile* t, int* splits) {
  const int bk = dtype == DT_BF16 ? STEP<bf16_t> : STEP<float>;
  const int64_t big = ((M + 255) / 256) * ((N + 255) / 256), mid = ((M + 127) / 128) * ((N + 127) / 128);
  if (dtype == DT_BF16 && big >= 192) *t = Tile{256, 256};
  else if (mid >= 128) *t = Tile{128, 128};
  else *t = Tile{64, 64};
  const int64_t tiles = ((M + t->bm - 1) / t->bm) * ((N + t->bn - 1) / t->bn);
  const int steps = (K + bk - 1) / bk;
  int64_t s = 1;
  if (tiles < 256) s = std::min<int64_t>(512 / tiles, steps / 4);
  *splits = (int)std::max<int64_t>(1, s);
}

template <typename T, int BM, int BN, int WM, int WN, bool TA, bool TB, int EPI>
hipError_t go(const LinearArgs& a, hipStream_t s) {
  const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  static const struct Name {
    char s[64];
    Name() { snprintf(s, sizeof s, "k_linear<%s,%d,%d,%s>", sizeof(T) == 2 ? "bf16" : "f32", BM, BN,
                      EPI == LIN_FWD ? "fwd" : EPI == LIN_DATA ? "data" : "grad"); }
  } name;
  XP_LAUNCH(name.s, 2.0 * a.M * a.N * a.K, (k_linear<T, BM, BN, WM, WN, TA, TB, EPI>), dim3((unsigned)(tm * tn * a.splits)),
            dim3(WM * WN * 64), 0, s, a, (int)tm, (int)tn);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  XP_LAUNCH("k_linear_join", 4.0 * a.M * a.N * a.splits, (k_linear_join<T, EPI>),
            dim3(grid_of(a.M * ((a.N + CHUNK<T> - 1) / CHUNK<T>))), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool TA, bool TB, int EPI>
hipError_t by_tile(const LinearArgs& a, const Tile& t, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (t.bm == 256) return go<T, 256, 256, 2, 4, TA, TB, EPI>(a, s);
  }
  if (t.bm == 128) return go<T, 128, 128, 2, 2, TA, TB, EPI>(a, s);
  return go<T, 64, 64, 2, 2, TA, TB, EPI>(a, s);
}

template <typename T>
hipError_t by_kind(const LinearArgs& a, const Tile& t, hipStream_t s) {
  if (a.epi == LIN_FWD) return by_tile<T, false, false, LIN_FWD>(a, t, s);
  if (a.epi == LIN_DATA) return by_tile<T, false, true, LIN_DATA>(a, t, s);
  return by_tile<T, true, true, LIN_GRAD>(a, t, s);
}

bool chunked(const void* p, int64_t ld, int chunk) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % chunk == 0;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

}  // namespace

// Where the operands and the results lie: what a call needs of its workspace.
LinearPlan linear_plan(int dtype, const LinearArgs& a) {
  LinearPlan p{};
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  const bool ta = a.epi == LIN_GRAD, tb = a.epi != LIN_FWD;
  // a reduction along the rows has to end with a chunk
  p.pack_a = !chunked(a.A, a.lda, chunk) || (!ta && a.K % chunk != 0);
  p.pack_b = !chunked(a.B, a.ldb, chunk) || (!tb && a.K % chunk != 0);
  auto cols = [&](bool tr, int64_t n) { return (tr ? n : (int64_t)a.K + chunk - 1) / chunk * chunk; };
  p.a_cols = (int)(ta ? (a.M + chunk - 1) / chunk * chunk : cols(false, 0));
  p.b_cols = (int)(tb ? ((int64_t)a.N + chunk - 1) / chunk * chunk : cols(false, 0));
  Tile t;
  pick(dtype, a.M, a.N, a.K, &t, &p.splits);
  p.bm = t.bm;
  const int bk = 128 / es;
  const int64_t steps = ((int64_t)a.K + bk - 1) / bk;
  p.kper = (steps + p.splits - 1) / p.splits * bk;
  p.splits = (int)(((int64_t)a.K + p.kper - 1) / p.kper);  // those that hold something
  p.ldpart = (a.N + 7) / 8 * 8;
  size_t off = 0;
  if (p.pack_a) {
    p.a_off = off;
    off += up256((size_t)(ta ? a.K : a.M) * p.a_cols * es);
  }
  if (p.pack_b) {
    p.b_off = off;
    off += up256((size_t)(tb ? a.K : a.N) * p.b_cols * es);
  }
  if (p.splits > 1) {
    p.part_off = off;
    off += up256((size_t)p.splits * a.M * p.ldpart * sizeof(float));
    p.part_b_off = off;
    if (a.grad_b) off += up256((size_t)p.splits * a.M * sizeof(double));
  }
  p.bytes = off;
  return p;
}

hipError_t launch_linear(int dtype, const LinearArgs& in, void* workspace, hipStream_t s) {
  if (in.M <= 0 || in.N <= 0) return hipSuccess;
  LinearArgs a = in;
  const LinearPlan p = linear_plan(dtype, a);
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  const bool ta = a.epi == LIN_GRAD, tb = a.epi != LIN_FWD;
  char* ws = (char*)workspace;
  auto pack = [&](const void*& ptr, int64_t& ld, int64_t rows, int cols, int cols_out, size_t off) -> hipError_t {
    void* dst = ws + off;
    const double bytes = (double)rows * (cols + cols_out) * es;
    if (dtype == DT_BF16)
      XP_LAUNCH("k_linear_pack<bf16>", bytes, k_linear_pack<bf16_t>, dim3(grid_of(rows * cols_out)), dim3(256), 0, s,
                (const bf16_t*)ptr, ld, rows, cols, (bf16_t*)dst, cols_out);
    else
      XP_LAUNCH("k_linear_pack<f32>", bytes, k_linear_pack<float>, dim3(grid_of(rows * cols_out)), dim3(256), 0, s,
                (const float*)ptr, ld, rows, cols, (float*)dst, cols_out);
    ptr = dst;
    ld = cols_out;
    return hipGetLastError();
  };
  if (p.pack_a) {
    hipError_t e = pack(a.A, a.lda, ta ? a.K : a.M, ta ? (int)a.M : a.K, p.a_cols, p.a_off);
    if (e != hipSuccess) return e;
  }
  if (p.pack_b) {
    hipError_t e = pack(a.B, a.ldb, tb ? a.K : a.N, tb ? a.N : a.K, p.b_cols, p.b_off);
    if (e != hipSuccess) return e;
  }
  a.splits = p.splits;
  a.kper = p.kper;
  a.ldpart = p.ldpart;
  a.part = p.splits > 1 ? (float*)(ws + p.part_off) : nullptr;
  a.part_b = p.splits > 1 ? (double*)(ws + p.part_b_off) : nullptr;
  a.vec = a.epi == LIN_GRAD
              ? chunked(a.grad, a.N, 4)
              : chunked(a.y, a.ldy, chunk) && (!a.res || chunked(a.res, a.ldr, chunk)) &&
                    (!a.z_in || chunked(a.z_in, a.ldz, chunk)) && (!a.z_out || chunked(a.z_out, a.ldz, chunk));
  const Tile t{p.bm, p.bm};
  return dtype == DT_BF16 ? by_kind<bf16_t>(a, t, s) : by_kind<float>(a, t, s);
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
