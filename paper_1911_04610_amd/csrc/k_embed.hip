// Embedding lookup, and its gradient by sorted tokens.
//
// The gradient of a table row is the sum over the positions that hold its token.
// The positions are sorted by token (stable, so a row's terms are added in the
// order of their positions: the same bits every time, no atomics on sums), and
// every row of dy is then read once.  Tokens outside [0, vocab) are padding:
// zero rows forwards, nothing backwards; the sort puts them last, as `vocab`.
#include "xp_device.h"
#include "xp_lds.h"
#include "xp_kernels.h"

#include <algorithm>

namespace xp {

namespace {

template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);

int grid_of(int64_t items, int per) {
  return (int)std::max<int64_t>(1, std::min<int64_t>((items + per - 1) / per, (int64_t)1 << 20));
}

template <typename T>
XP_DEV void unpack(const u32x4_t& u, float (&v)[CHUNK<T>]) {
#pragma unroll
  for (int i = 0; i < CHUNK<T>; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(u[i]);
    else v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  }
}

// ---------------------------------------------------------------- lookup
// One 16-byte chunk of one position per thread (VEC), else one element.  The
// product is formed in fp64 and rounded to fp32 (for bf16, from there).  Bound by
// memory: 65536 rows of 2048 bf16 103 us, 16384 of 4096 43 us, 5.2 and 6.3 TB/s read and
// written.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_embed_fwd(EmbedArgs a) {
  constexpr int C = VEC ? CHUNK<T> : 1;
  const int64_t cpr = a.dim / C, total = a.n * cpr;
  const T* table = (const T*)a.table;
  T* y = (T*)a.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cpr, c = (i - r * cpr) * C;
    const int t = a.tokens[r];
    const bool live = t >= 0 && t < a.vocab;
    if constexpr (VEC) {
      u32x4_t u = {0u, 0u, 0u, 0u};
      if (live) {
        float v[C];
        unpack<T>(*reinterpret_cast<const u32x4_t*>(table + (int64_t)t * a.dim + c), v);
#pragma unroll
        for (int q = 0; q < C; ++q) v[q] = (float)((double)v[q] * a.scale);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (sizeof(T) == 4) u[q] = __float_as_uint(v[q]);
          else u[q] = f32x2_to_bf16x2(v[2 * q], v[2 * q + 1]);
        }
      }
      *reinterpret_cast<u32x4_t*>(y + r * a.dim + c) = u;
    } else {
      std_(y + r * a.dim + c, live ? ldd(table + (int64_t)t * a.dim + c) * a.scale : 0.0);
    }
  }
}

// ---------------------------------------------------------------- sort
XP_DEV uint32_t sort_key(int t, int vocab) { return (uint32_t)t < (uint32_t)vocab ? (uint32_t)t : (uint32_t)vocab; }

// Few positions: a position's place is the number of positions before it in the
// order.  Sixteen positions per workgroup; the sixteen waves go through all keys in
// LDS, and each quarter of a wave takes every fourth four of the wave's own.  Bound by
// the LDS reads: 8192 keys 8 to 10 us (64 positions per workgroup, all lanes reading the same
// key, 20; the radix sort's four launches 23).
constexpr int RANK_MAX = 8192, RANK_POS = 16;
__global__ __launch_bounds__(1024) void k_embed_rank(const int32_t* __restrict__ tokens, int n, int vocab,
                                                      uint32_t* __restrict__ keys, uint32_t* __restrict__ pos) {
  __shared__ __align__(16) uint32_t sk[RANK_MAX];
  __shared__ int sums[16][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pad = (n + 15) / 16 * 16;
  for (int j = tid; j < pad; j += 1024) sk[j] = j < n ? sort_key(tokens[j], vocab) : ~0u;
  __syncthreads();
  const int i0 = blockIdx.x * RANK_POS, i = i0 + (lane & 15);
  const uint32_t key = i < n ? sk[i] : 0u;
  int rank = 0;
  // before the workgroup's own positions equal keys count, after them they do not
#pragma unroll 4
  for (int j0 = wave * 16; j0 < pad; j0 += 256) {
    const int j = j0 + (lane >> 4) * 4;
    const u32x4_t k = *reinterpret_cast<const u32x4_t*>(sk + j);
    if (j0 < i0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) rank += k[q] <= key;
    } else if (j0 > i0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) rank += k[q] < key;
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) rank += k[q] < key || (k[q] == key && j + q < i);
    }
  }
  sums[wave][lane] = rank;
  __syncthreads();
  if (wave == 0) {
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) at += sums[w][lane];
    at += __shfl_xor(at, 16, 64);
    at += __shfl_xor(at, 32, 64);
    if (lane < RANK_POS && i < n) {
      keys[at] = key;
      pos[at] = (uint32_t)i;
    }
  }
}

// More positions: a stable radix sort, eight bits of the token at a time.  A
// workgroup takes `per` consecutive positions (a multiple of 256), each of its
// four waves a quarter of them.
constexpr int RADIX = 256, SORT_BLOCKS = 256;
XP_DEV uint32_t first_key(const uint32_t* keys, const int32_t* tokens, int vocab, int64_t i) {
  return tokens ? sort_key(tokens[i], vocab) : keys[i];
}

__global__ __launch_bounds__(256) void k_embed_hist(const uint32_t* __restrict__ keys, const int32_t* __restrict__ tokens,
                                                    int vocab, int64_t n, int64_t per, int shift,
                                                    uint32_t* __restrict__ hist) {
  __shared__ uint32_t cnt[RADIX];
  const int tid = threadIdx.x;
  cnt[tid] = 0;
  __syncthreads();
  const int64_t beg = blockIdx.x * per, end = min(n, beg + per);
  for (int64_t i = beg + tid; i < end; i += 256)
    atomicAdd(&cnt[(first_key(keys, tokens, vocab, i) >> shift) & (RADIX - 1)], 1u);  // a count: any order
  __syncthreads();
  hist[(int64_t)blockIdx.x * RADIX + tid] = cnt[tid];
}

__global__ __launch_bounds__(256) void k_embed_scatter(const uint32_t* __restrict__ keys, const int32_t* __restrict__ tokens,
                                                       int vocab, const uint32_t* __restrict__ pos, int64_t n, int64_t per,
                                                       int shift, const uint32_t* __restrict__ hist,
                                                       uint32_t* __restrict__ keys_out, uint32_t* __restrict__ pos_out) {
  __shared__ uint32_t off[4][RADIX];
  __shared__ __align__(16) uint32_t sums[4][2][RADIX];
  __shared__ uint32_t wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int w = 0; w < 4; ++w) off[w][tid] = 0;
  __syncthreads();
  const int64_t beg = blockIdx.x * per + wave * (per / 4), end = min(n, beg + per / 4);
  for (int64_t i = beg + lane; i < end; i += 64)
    atomicAdd(&off[wave][(first_key(keys, tokens, vocab, i) >> shift) & (RADIX - 1)], 1u);
  // how many positions all workgroups, and the ones before this one, hold of each
  // digit: a wave adds every fourth workgroup's counts, a lane four digits
  {
    u32x4_t sa = {0u, 0u, 0u, 0u}, sb = {0u, 0u, 0u, 0u};
#pragma unroll 16
    for (int b = wave; b < (int)gridDim.x; b += 4) {
      const u32x4_t h = *reinterpret_cast<const u32x4_t*>(hist + (int64_t)b * RADIX + lane * 4);
      sa += h;
      sb += b < (int)blockIdx.x ? h : (u32x4_t){0u, 0u, 0u, 0u};
    }
    *reinterpret_cast<u32x4_t*>(&sums[wave][0][lane * 4]) = sa;
    *reinterpret_cast<u32x4_t*>(&sums[wave][1][lane * 4]) = sb;
  }
  __syncthreads();
  uint32_t all = 0, before = 0;  // of digit tid
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    all += sums[w][0][tid];
    before += sums[w][1][tid];
  }
  uint32_t scan = all;  // inclusive over the wave's digits, then the waves
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(scan, d, 64);
    scan += lane >= d ? up : 0u;
  }
  if (lane == 63) wsum[wave] = scan;
  __syncthreads();
  uint32_t at = scan - all + before;
  for (int w = 0; w < wave; ++w) at += wsum[w];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t c = off[w][tid];
    off[w][tid] = at;
    at += c;
  }
  __syncthreads();
  // 64 positions at a time; the lanes of one digit take their places in lane order
  volatile uint32_t* mine = off[wave];
  for (int64_t i0 = beg; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool live = i < end;
    const uint32_t key = live ? first_key(keys, tokens, vocab, i) : 0u;
    const int digit = (key >> shift) & (RADIX - 1);
    uint64_t peers = __ballot(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t m = __ballot((digit >> b) & 1);
      peers &= (digit >> b) & 1 ? m : ~m;
    }
    const int rank = __popcll(peers & (((uint64_t)1 << lane) - 1));
    if (live) {
      const uint32_t to = mine[digit] + rank;
      keys_out[to] = key;
      pos_out[to] = tokens ? (uint32_t)i : pos[i];
    }
    __builtin_amdgcn_wave_barrier();
    if (live && rank == 0) mine[digit] = mine[digit] + __popcll(peers);
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------- gradient
// A wave takes `span` consecutive sorted positions and 64 chunks of columns, and
// adds the rows of each run of equal tokens in fp64.  Runs inside the span go
// straight into the accumulator; what a run has in this span that started before
// it (part 0) or goes on behind it (part 1) is left as an fp32 partial for
// k_embed_join; a run that does both is part 0.  Rows are taken GROUP at a
// time, with the accumulators' rows that they end in, so that the loads of a
// group are in flight together.  Bound by memory: 65536 rows of 2048 bf16 into a table
// of 50000 111 to 120 us, 4.4 to 4.7 TB/s of rows and accumulators.
constexpr int GROUP = 4;
template <typename T, bool VEC>
__global__ __launch_bounds__(64) void k_embed_bwd(EmbedArgs a, const uint32_t* __restrict__ keys,
                                                  const uint32_t* __restrict__ pos, int span, float* __restrict__ part) {
  constexpr int C = VEC ? CHUNK<T> : 1;
  const int64_t beg = (int64_t)blockIdx.x * span, end = min(a.n, beg + span);
  const int64_t col = ((int64_t)blockIdx.y * 64 + threadIdx.x) * C;
  if (col >= a.dim) return;
  const T* dy = (const T*)a.dy + col;
  float* grad = a.grad + col;
  double acc[C];
#pragma unroll
  for (int q = 0; q < C; ++q) acc[q] = 0.0;
  bool head = beg > 0 && keys[beg - 1] == keys[beg];  // the present run started before the span
  for (int64_t g = beg; g < end; g += GROUP) {
    uint32_t key[GROUP];
    bool last[GROUP], whole[GROUP];
    u32x4_t v[GROUP];  // (not VEC: one element)
    float o[GROUP][C];
    bool h = head;
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      const int64_t i = g + j;
      const bool in = i < end;
      key[j] = in ? keys[i] : (uint32_t)a.vocab;
      const bool live = in && key[j] < (uint32_t)a.vocab;
      const bool more = i + 1 < a.n && keys[min(i + 1, a.n - 1)] == key[j];  // the run goes on behind i
      last[j] = live && (!more || i + 1 == end);
      whole[j] = last[j] && !more && !h;
      if (in && !more) h = false;
      if (!live) continue;
      const T* row = dy + (int64_t)pos[i] * a.dim;
      if constexpr (VEC) v[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row));
      else v[j][0] = __float_as_uint((float)ldd(row));
      if (whole[j]) {
        const float* gr = grad + (int64_t)key[j] * a.dim;
#pragma unroll
        for (int q = 0; q < C; ++q) o[j][q] = gr[q];
      }
    }
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      if (key[j] >= (uint32_t)a.vocab) continue;
      if constexpr (VEC) {
        float e[C];
        unpack<T>(v[j], e);
#pragma unroll
        for (int q = 0; q < C; ++q) acc[q] += (double)e[q];
      } else {
        acc[0] += (double)__uint_as_float(v[j][0]);
      }
      if (!last[j]) continue;
      if (whole[j]) {
        float* gr = grad + (int64_t)key[j] * a.dim;
#pragma unroll
        for (int q = 0; q < C; ++q) gr[q] = (float)((double)o[j][q] + a.scale * acc[q]);
      } else {
        // from before the span, or (whole runs aside) on behind it
        float* p = part + ((int64_t)blockIdx.x * 2 + (head ? 0 : 1)) * a.dim + col;
#pragma unroll
        for (int q = 0; q < C; ++q) p[q] = (float)acc[q];
      }
      head = false;
#pragma unroll
      for (int q = 0; q < C; ++q) acc[q] = 0.0;
    }
  }
}

// The runs that pass a span's end: the span that a run starts in adds its
// partials.  JOIN_WAVES waves take consecutive parts of the run's spans, 64 JOIN_COLS
// columns each, and their sums are added in order.  Most workgroups find no run to
// join and end: eight waves each were 10 us slower for 65536 positions, and one
// wave 9, where the four take 17 (and the longest run bounds it).
constexpr int JOIN_COLS = 4, JOIN_WAVES = 4;
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_embed_join(EmbedArgs a, const uint32_t* __restrict__ keys, int span,
                                                     const float* __restrict__ part) {
  __shared__ double sums[JOIN_WAVES - 1][64][JOIN_COLS];
  const int64_t c = blockIdx.x, beg = c * span, next = beg + span;
  if (next >= a.n) return;
  const uint32_t key = keys[next - 1], kn = keys[next], kb = keys[beg], kp = keys[beg > 0 ? beg - 1 : 0];
  if (key >= (uint32_t)a.vocab || kn != key) return;  // no run passes the end
  if (beg > 0 && kb == key && kp == key) return;       // it started before this span
  const int64_t spans = (a.n + span - 1) / span;
  // the run's last span: the next as many as there are threads are looked at together, then, of a longer run,
  // every stride-th of those behind
  int64_t lo = c;
  auto look = [&](int64_t stride) __attribute__((always_inline)) {
    const int64_t at = lo + (threadIdx.x + 1) * stride;
    const int more = __syncthreads_count(at < spans && keys[at * span] == key);
    lo += more * stride;
    return more;
  };
  if (look(1) == 64 * JOIN_WAVES)
    for (int64_t stride = (int64_t)1 << 24; stride > 0; stride >>= 8)
      if (lo + stride < spans) look(stride);
  const int64_t cnt = lo - c;  // spans behind the first one
  const int g = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t per = max((int64_t)4, (cnt + JOIN_WAVES - 1) / JOIN_WAVES), s0 = c + 1 + g * per, s1 = min(lo + 1, s0 + per);
  for (int64_t col = ((int64_t)blockIdx.y * 64 + lane) * JOIN_COLS; col - lane * JOIN_COLS < a.dim;
       col += (int64_t)gridDim.y * 64 * JOIN_COLS) {
    const int cols = (int)max((int64_t)0, min((int64_t)JOIN_COLS, a.dim - col));
    const bool vec = cols == JOIN_COLS && a.dim % JOIN_COLS == 0;  // (the partials' rows are 16-byte aligned then)
    double t[JOIN_COLS];
#pragma unroll
    for (int q = 0; q < JOIN_COLS; ++q) t[q] = 0.0;
    auto add = [&](const float* p) __attribute__((always_inline)) {
      if (vec) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
        for (int q = 0; q < JOIN_COLS; ++q) t[q] += (double)v[q];
      } else {
#pragma unroll
        for (int q = 0; q < JOIN_COLS; ++q)
          if (q < cols) t[q] += (double)p[q];
      }
    };
    if (g == 0) add(part + (c * 2 + 1) * a.dim + col);
#pragma unroll 16
    for (int64_t s = s0; s < s1; ++s) add(part + s * 2 * a.dim + col);
    if (g > 0) {
#pragma unroll
      for (int q = 0; q < JOIN_COLS; ++q) sums[g - 1][lane][q] = t[q];
    }
    __syncthreads();
    if (g == 0) {
      float* o = a.grad + (int64_t)key * a.dim + col;
#pragma unroll
      for (int q = 0; q < JOIN_COLS; ++q) {
        if (q >= cols) continue;
        double v = t[q];
#pragma unroll
        for (int w = 0; w < JOIN_WAVES - 1; ++w) v += sums[w][lane][q];
        o[q] = (float)((double)o[q] + a.scale * v);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- few positions
// Without a sort: the workgroup of the first position that holds a token adds all
// of its positions' rows, 64 chunks of columns a wave, each of its four waves a
// consecutive part of them; the others find an earlier one and end.  One launch: 1024
// positions of 1024 bf16 10.6 us, 1025 sorted 15.5; every workgroup reads all tokens, so
// the sort takes over there.  256 positions of 256 fp32 4.4 us, its launch.
constexpr int SMALL_MAX = 1024;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_embed_bwd_small(EmbedArgs a) {
  constexpr int C = VEC ? CHUNK<T> : 1;
  __shared__ uint64_t mask[SMALL_MAX / 64];
  __shared__ int list[SMALL_MAX];
  __shared__ double sums[3][64][C];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = blockIdx.x;
  const int t = a.tokens[i], n = (int)a.n;
  if (t < 0 || t >= a.vocab) return;
#pragma unroll
  for (int q = 0; q < SMALL_MAX / 256; ++q) {
    const int j = q * 256 + tid;
    const uint64_t m = __ballot(j < n && a.tokens[min(j, n - 1)] == t);
    if (lane == 0) mask[q * 4 + wave] = m;
  }
  __syncthreads();
  // the token's positions in order, and whether i is the first
  int count = 0;
  bool first = true;
#pragma unroll
  for (int w = 0; w < SMALL_MAX / 64; ++w) {
    const uint64_t m = mask[w];
    const uint64_t low = i >= (w + 1) * 64 ? ~(uint64_t)0 : i <= w * 64 ? 0 : ((uint64_t)1 << (i - w * 64)) - 1;
    first = first && (m & low) == 0;
    if (w % 4 == wave && (m >> lane & 1))
      list[count + __popcll(m & (((uint64_t)1 << lane) - 1))] = w * 64 + lane;
    count += __popcll(m);
  }
  if (!first) return;
  __syncthreads();
  const int per = max(8, (count + 3) / 4), s0 = min(count, wave * per), s1 = min(count, s0 + per);
  const int64_t col = ((int64_t)blockIdx.y * 64 + lane) * C;
  const bool live = col < a.dim;
  double acc[C];
#pragma unroll
  for (int q = 0; q < C; ++q) acc[q] = 0.0;
  float* o = a.grad + (int64_t)t * a.dim + col;
  float old[C];
  if (live && wave == 0) {
#pragma unroll
    for (int q = 0; q < C; ++q) old[q] = o[q];
  }
  if (live) {
    const T* dy = (const T*)a.dy + col;
#pragma unroll 8
    for (int s = s0; s < s1; ++s) {
      const T* row = dy + (int64_t)list[s] * a.dim;
      if constexpr (VEC) {
        float e[C];
        unpack<T>(*reinterpret_cast<const u32x4_t*>(row), e);
#pragma unroll
        for (int q = 0; q < C; ++q) acc[q] += (double)e[q];
      } else {
        acc[0] += ldd(row);
      }
    }
  }
  if (count > per) {  // (the same for the whole workgroup)
    if (wave > 0) {
#pragma unroll
      for (int q = 0; q < C; ++q) sums[wave - 1][lane][q] = acc[q];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int q = 0; q < C; ++q) acc[q] += sums[w][lane][q];
    }
  }
  if (live && wave == 0) {
#pragma unroll
    for (int q = 0; q < C; ++q) o[q] = (float)((double)old[q] + a.scale * acc[q]);
  }
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }
bool aligned(const void* p, int64_t dim, int chunk) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && dim % chunk == 0; }

// sorted positions per wave of the gradient: as many as leave some 2048 waves (the
// fewer spans, the fewer partials), 8 to 64
int span_of(int64_t n, int64_t dim) {
  const int64_t waves = n * ((dim + 511) / 512);
  int span = 8;
  while (span < 64 && waves > (int64_t)2048 * span) span *= 2;
  return span;
}

int64_t sort_per(int64_t n) { return std::max<int64_t>(1024, ((n + SORT_BLOCKS - 1) / SORT_BLOCKS + 255) / 256 * 256); }

struct Layout {
  size_t keys[2], pos[2], hist, part, bytes;
};
Layout layout(int64_t n, int64_t dim) {
  Layout l{};
  size_t off = 0;
  auto take = [&](size_t b) {
    const size_t at = off;
    off += up256(b);
    return at;
  };
  const int sides = n <= RANK_MAX ? 1 : 2;
  for (int s = 0; s < sides; ++s) {
    l.keys[s] = take((size_t)n * 4);
    l.pos[s] = take((size_t)n * 4);
  }
  if (n > RANK_MAX) l.hist = take((size_t)SORT_BLOCKS * RADIX * 4);
  l.part = take((size_t)((n + span_of(n, dim) - 1) / span_of(n, dim)) * 2 * dim * sizeof(float));
  l.bytes = off;
  return l;
}

}  // namespace

hipError_t launch_embed_fwd(int dtype, const EmbedArgs& a, hipStream_t s) {
  if (a.n <= 0 || a.dim <= 0) return hipSuccess;
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  const bool vec = aligned(a.table, a.dim, chunk) && aligned(a.y, a.dim, chunk);
  const dim3 grid(grid_of(a.n * (vec ? a.dim / chunk : a.dim), 256));
  const double bytes = 2.0 * a.n * a.dim * es;
  if (dtype == DT_BF16) {
    if (vec) XP_LAUNCH("k_embed_fwd<bf16>", bytes, (k_embed_fwd<bf16_t, true>), grid, dim3(256), 0, s, a);
    else XP_LAUNCH("k_embed_fwd<bf16>", bytes, (k_embed_fwd<bf16_t, false>), grid, dim3(256), 0, s, a);
  } else {
    if (vec) XP_LAUNCH("k_embed_fwd<f32>", bytes, (k_embed_fwd<float, true>), grid, dim3(256), 0, s, a);
    else XP_LAUNCH("k_embed_fwd<f32>", bytes, (k_embed_fwd<float, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

size_t embed_bwd_bytes(int64_t n, int64_t dim) { return n <= SMALL_MAX ? 0 : layout(n, dim).bytes; }

hipError_t launch_embed_bwd(int dtype, const EmbedArgs& a, void* workspace, hipStream_t s) {
  if (a.n <= 0 || a.dim <= 0) return hipSuccess;
  const int es = dtype == DT_BF16 ? 2 : 4, chunk = 16 / es;
  // (the accumulator's rows need no alignment of their own: their elements are 4 bytes wide)
  const bool vec = aligned(a.dy, a.dim, chunk);
  const double bytes = (double)a.n * a.dim * es;
  const unsigned col_blocks = (unsigned)(((vec ? a.dim / chunk : a.dim) + 63) / 64);
  if (a.n <= SMALL_MAX) {
    const dim3 grid((unsigned)a.n, col_blocks);
    if (dtype == DT_BF16) {
      if (vec) XP_LAUNCH("k_embed_bwd_small<bf16>", bytes, (k_embed_bwd_small<bf16_t, true>), grid, dim3(256), 0, s, a);
      else XP_LAUNCH("k_embed_bwd_small<bf16>", bytes, (k_embed_bwd_small<bf16_t, false>), grid, dim3(256), 0, s, a);
    } else {
      if (vec) XP_LAUNCH("k_embed_bwd_small<f32>", bytes, (k_embed_bwd_small<float, true>), grid, dim3(256), 0, s, a);
      else XP_LAUNCH("k_embed_bwd_small<f32>", bytes, (k_embed_bwd_small<float, false>), grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
  }
  char* ws = (char*)workspace;
  const Layout l = layout(a.n, a.dim);
  uint32_t *keys = (uint32_t*)(ws + l.keys[0]), *pos = (uint32_t*)(ws + l.pos[0]);
  hipError_t e;
  if (a.n <= RANK_MAX) {
    XP_LAUNCH("k_embed_rank", 12.0 * a.n, k_embed_rank, dim3((unsigned)((a.n + RANK_POS - 1) / RANK_POS)), dim3(1024), 0, s, a.tokens,
              (int)a.n, a.vocab, keys, pos);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  } else {
    int bits = 1;  // of the largest key, vocab
    while ((int64_t)a.vocab >> bits) ++bits;
    const int64_t per = sort_per(a.n);
    const unsigned blocks = (unsigned)((a.n + per - 1) / per);
    uint32_t* hist = (uint32_t*)(ws + l.hist);
    int side = 0;
    for (int shift = 0; shift < bits; shift += 8) {
      const int32_t* tokens = shift == 0 ? a.tokens : nullptr;  // the first pass reads the tokens themselves
      XP_LAUNCH("k_embed_hist", 4.0 * a.n, k_embed_hist, dim3(blocks), dim3(256), 0, s, keys, tokens, a.vocab, a.n, per,
                shift, hist);
      uint32_t *ko = (uint32_t*)(ws + l.keys[1 - side]), *po = (uint32_t*)(ws + l.pos[1 - side]);
      XP_LAUNCH("k_embed_scatter", 16.0 * a.n, k_embed_scatter, dim3(blocks), dim3(256), 0, s, keys, tokens, a.vocab, pos,
                a.n, per, shift, hist, ko, po);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      side = 1 - side;
      keys = ko;
      pos = po;
    }
  }
  const int span = span_of(a.n, a.dim);
  const unsigned spans = (unsigned)((a.n + span - 1) / span);
  const dim3 grid(spans, col_blocks);
  float* part = (float*)(ws + l.part);
  if (dtype == DT_BF16) {
    if (vec) XP_LAUNCH("k_embed_bwd<bf16>", bytes, (k_embed_bwd<bf16_t, true>), grid, dim3(64), 0, s, a, keys, pos, span, part);
    else XP_LAUNCH("k_embed_bwd<bf16>", bytes, (k_embed_bwd<bf16_t, false>), grid, dim3(64), 0, s, a, keys, pos, span, part);
  } else {
    if (vec) XP_LAUNCH("k_embed_bwd<f32>", bytes, (k_embed_bwd<float, true>), grid, dim3(64), 0, s, a, keys, pos, span, part);
    else XP_LAUNCH("k_embed_bwd<f32>", bytes, (k_embed_bwd<float, false>), grid, dim3(64), 0, s, a, keys, pos, span, part);
  }
  e = hipGetLastError();
  if (e != hipSuccess || spans < 2) return e;
  XP_LAUNCH("k_embed_join", 0.0, k_embed_join, dim3(spans - 1, (unsigned)std::min<int64_t>(16, (a.dim + 64 * JOIN_COLS - 1) / (64 * JOIN_COLS))),
            dim3(64 * JOIN_WAVES), 0, s, a, keys, span, part);
  return hipGetLastError();
}

}  // namespace xp
