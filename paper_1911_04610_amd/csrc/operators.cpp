// C ABI of the operators around a stage: linear layers, the embedding and the
// gradient norm.  Each entry point checks its arguments on the host and then
// only enqueues kernels on the caller's stream; none keeps anything between calls.
#include "xp_host.h"

#include <algorithm>
#include <cmath>

using namespace xp;

namespace {

bool known_dtype(int32_t d) { return d == XPIPE_F32 || d == XPIPE_BF16; }
int esize(int32_t dtype) { return dtype == XPIPE_BF16 ? 2 : 4; }

bool at_multiple(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// a matrix argument: present, aligned to its element, rows at least as far apart as long
xpipe_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, int es) {
  if (!p) return fail(XPIPE_EINVAL, std::string("null ") + name);
  if (!at_multiple(p, es)) return fail(XPIPE_EINVAL, std::string(name) + " is not aligned to its element");
  if (ld < cols) return fail(XPIPE_EINVAL, std::string(name) + ": rows closer than they are long");
  if (ld > XPIPE_LINEAR_MAX_LD)
    return fail(XPIPE_EUNSUPPORTED, std::string(name) + ": rows further apart than XPIPE_LINEAR_MAX_LD elements");
  return XPIPE_OK;
}

xpipe_status check_sizes(int64_t rows, int32_t cin, int32_t cout, int32_t dtype, int32_t act) {
  if (rows < 0 || cin < 1 || cout < 1) return fail(XPIPE_EINVAL, "rows must be >= 0, cin and cout >= 1");
  if (!known_dtype(dtype)) return fail(XPIPE_EINVAL, "unknown dtype");
  if (act < XPIPE_ACT_NONE || act > XPIPE_ACT_SILU) return fail(XPIPE_EINVAL, "unknown activation");
  // (a launch's tiles are counted in 32 bits)
  if (rows >= (int64_t)1 << 30 || rows / 64 * (std::max(cin, cout) / 64) >= (int64_t)1 << 30)
    return fail(XPIPE_EUNSUPPORTED, "2^30 rows or 2^42 results or more");
  return XPIPE_OK;
}

#define XP_TRY(call)                        \
  do {                                      \
    xpipe_status r_ = (call);               \
    if (r_ != XPIPE_OK) return r_;          \
  } while (0)

xpipe_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return XPIPE_OK;
  if (!ws) return fail(XPIPE_EINVAL, "null workspace");
  if (bytes < need) return fail(XPIPE_EINVAL, "workspace too small");
  if (!at_multiple(ws, 256)) return fail(XPIPE_EINVAL, "workspace must be 256-byte aligned");
  return XPIPE_OK;
}

// the forward's product
xpipe_status fwd_product(const xpipe_linear_fwd_args* q, LinearArgs* a) {
  if (!q) return fail(XPIPE_EINVAL, "null arguments");
  XP_TRY(check_sizes(q->rows, q->cin, q->cout, q->dtype, q->act));
  *a = LinearArgs{};
  if (q->rows == 0) return XPIPE_OK;
  const int es = esize(q->dtype);
  XP_TRY(check_matrix("x", q->x, q->ldx, q->cin, es));
  XP_TRY(check_matrix("W", q->W, q->ldw, q->cin, es));
  XP_TRY(check_matrix("y", q->y, q->ldy, q->cout, es));
  if (q->residual) XP_TRY(check_matrix("residual", q->residual, q->ldr, q->cout, es));
  if (q->preact) XP_TRY(check_matrix("preact", q->preact, q->ldz, q->cout, es));
  if (q->bias && !at_multiple(q->bias, 4)) return fail(XPIPE_EINVAL, "bias is not aligned to its element");
  if (q->y == q->x || q->y == q->W || q->y == (const void*)q->bias || (q->preact && (q->preact == q->y || q->preact == q->x ||
      q->preact == q->W || q->preact == q->residual || q->preact == (const void*)q->bias)))
    return fail(XPIPE_EINVAL, "an output is an input's or another output's buffer");
  if (q->y == q->residual && q->ldy != q->ldr) return fail(XPIPE_EINVAL, "residual in y's buffer with another ld");
  a->epi = LIN_FWD;
  a->act = q->act;
  a->M = q->rows;
  a->N = q->cout;
  a->K = q->cin;
  a->A = q->x;
  a->lda = q->ldx;
  a->B = q->W;
  a->ldb = q->ldw;
  a->bias = q->bias;
  a->res = q->residual;
  a->ldr = q->ldr;
  a->z_out = q->preact;
  a->ldz = q->ldz;
  a->y = q->y;
  a->ldy = q->ldy;
  return XPIPE_OK;
}

// the backward's two products (M = 0 for one that is not asked for)
xpipe_status bwd_products(const xpipe_linear_bwd_args* q, LinearArgs (&p)[2]) {
  LinearArgs *data = &p[0], *grad = &p[1];
  if (!q) return fail(XPIPE_EINVAL, "null arguments");
  XP_TRY(check_sizes(q->rows, q->cin, q->cout, q->dtype, q->act));
  *data = LinearArgs{};
  *grad = LinearArgs{};
  if (q->grad_b && !q->grad_W) return fail(XPIPE_EINVAL, "grad_b without grad_W");
  if (q->rows == 0 || (!q->dx && !q->grad_W)) return XPIPE_OK;
  const int es = esize(q->dtype);
  XP_TRY(check_matrix("dz", q->dz, q->lddz, q->cout, es));
  if (q->dx) {
    XP_TRY(check_matrix("dx", q->dx, q->lddx, q->cin, es));
    XP_TRY(check_matrix("W", q->W, q->ldw, q->cin, es));
    if (q->act != XPIPE_ACT_NONE) XP_TRY(check_matrix("preact", q->preact, q->ldz, q->cin, es));
    else if (q->preact) return fail(XPIPE_EINVAL, "preact without an activation");
    if (q->residual) XP_TRY(check_matrix("residual", q->residual, q->ldr, q->cin, es));
    if (q->dx == q->dz || q->dx == q->x || q->dx == q->W) return fail(XPIPE_EINVAL, "dx is an input's buffer");
    if ((q->dx == q->residual && q->lddx != q->ldr) || (q->dx == q->preact && q->lddx != q->ldz))
      return fail(XPIPE_EINVAL, "residual or preact in dx's buffer with another ld");
    data->epi = LIN_DATA;
    data->act = q->act;
    data->M = q->rows;
    data->N = q->cin;
    data->K = q->cout;
    data->A = q->dz;
    data->lda = q->lddz;
    data->B = q->W;
    data->ldb = q->ldw;
    data->res = q->residual;
    data->ldr = q->ldr;
    data->z_in = q->act != XPIPE_ACT_NONE ? q->preact : nullptr;
    data->ldz = q->ldz;
    data->y = q->dx;
    data->ldy = q->lddx;
  }
  if (q->grad_W) {
    XP_TRY(check_matrix("x", q->x, q->ldx, q->cin, es));
    if (!at_multiple(q->grad_W, 4) || !at_multiple(q->grad_b, 4))
      return fail(XPIPE_EINVAL, "grad_W or grad_b is not aligned to its element");
    if (q->grad_W == q->grad_b) return fail(XPIPE_EINVAL, "grad_W and grad_b are one buffer");
    const void* g[2] = {q->grad_W, q->grad_b};
    for (const void* p : g)
      if (p && (p == q->dz || p == q->x || p == q->W || p == q->dx || p == q->preact || p == q->residual))
        return fail(XPIPE_EINVAL, "a gradient accumulator is another argument's buffer");
    grad->epi = LIN_GRAD;
    grad->M = q->cout;
    grad->N = q->cin;
    grad->K = (int)q->rows;
    grad->A = q->dz;
    grad->lda = q->lddz;
    grad->B = q->x;
    grad->ldb = q->ldx;
    grad->grad = q->grad_W;
    grad->grad_b = q->grad_b;
  }
  return XPIPE_OK;
}

xpipe_status check_embedding_sizes(int64_t n, int32_t vocab, int32_t dim) {
  if (n < 0 || vocab < 1 || dim < 1) return fail(XPIPE_EINVAL, "n_tokens must be >= 0, vocab and dim >= 1");
  if (n >= (int64_t)1 << 30 || vocab >= 1 << 30 || dim > 1 << 20)
    return fail(XPIPE_EUNSUPPORTED, "2^30 tokens or vocabulary entries or more, or more than 2^20 columns");
  return XPIPE_OK;
}

xpipe_status check_embedding(const void* rows, const char* name, const int32_t* tokens, int64_t n, int32_t vocab,
                             int32_t dim, double scale, int32_t dtype) {
  if (!known_dtype(dtype)) return fail(XPIPE_EINVAL, "unknown dtype");
  if (!std::isfinite(scale)) return fail(XPIPE_EINVAL, "scale must be finite");
  XP_TRY(check_embedding_sizes(n, vocab, dim));
  if (n == 0) return XPIPE_OK;
  if (!rows) return fail(XPIPE_EINVAL, std::string("null ") + name);
  if (!tokens) return fail(XPIPE_EINVAL, "null tokens");
  if (!at_multiple(rows, esize(dtype)) || !at_multiple(tokens, 4))
    return fail(XPIPE_EINVAL, std::string(name) + " or tokens not aligned to their element");
  return XPIPE_OK;
}

// partial sums that a norm over the tensors leaves in its workspace (0: small, none)
xpipe_status check_tensors(const xpipe_tensor* t, int32_t n, int64_t* blocks) {
  if (n < 0 || (n > 0 && !t)) return fail(XPIPE_EINVAL, "bad tensor list");
  int64_t b = 0, units = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].n < 0) return fail(XPIPE_EINVAL, "negative length");
    if (t[i].n > 0 && !t[i].p) return fail(XPIPE_EINVAL, "null tensor");
    if (t[i].n >= (int64_t)1 << 40) return fail(XPIPE_EUNSUPPORTED, "a tensor of 2^40 elements or more");
    b += norm_blocks(t[i].n);
    units += (t[i].n + NORM_SMALL_PER - 1) / NORM_SMALL_PER;
  }
  *blocks = units <= NORM_SMALL_UNITS ? 0 : b;
  return XPIPE_OK;
}

}  // namespace

hipError_t xp::grad_norm(const xpipe_tensor* tensors, int32_t n, int32_t dtype, double max_norm, double* sumsq,
                         float* norm_coef, double* part, int64_t blocks, hipStream_t s) {
  NormArgs a{};
  if (blocks == 0) {  // (at most NORM_SMALL_UNITS tensors hold something)
    int units = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (tensors[i].n == 0) continue;
      a.p[a.count] = tensors[i].p;
      a.n[a.count] = tensors[i].n;
      a.first[a.count++] = units;
      units += (int)((tensors[i].n + NORM_SMALL_PER - 1) / NORM_SMALL_PER);
    }
    return launch_grad_norm_small(dtype, a, units, max_norm, sumsq, norm_coef, s);
  }
  a.part = part;
  int64_t first = 0;
  auto flush = [&]() -> hipError_t {
    hipError_t e = launch_grad_sumsq(dtype, a, (int)first, s);
    a.part += first;
    a.count = 0;
    first = 0;
    return e;
  };
  // tensors in batches of NORM_BATCH, long ones in pieces of 2^30 elements (whole
  // workgroups: norm_blocks counts the same partial sums)
  constexpr int64_t PIECE = (int64_t)1 << 30, MOST = (int64_t)1 << 30;
  for (int32_t i = 0; i < n; ++i) {
    const char* p = (const char*)tensors[i].p;
    for (int64_t left = tensors[i].n; left > 0; left -= PIECE, p += PIECE * esize(dtype)) {
      const int64_t take = std::min(left, PIECE);
      if (a.count == NORM_BATCH || first + norm_blocks(take) > MOST) {
        hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      a.p[a.count] = p;
      a.n[a.count] = take;
      a.first[a.count++] = (int)first;
      first += norm_blocks(take);
    }
  }
  hipError_t e = flush();
  return e != hipSuccess ? e : launch_clip_coef(part, blocks, max_norm, sumsq, norm_coef, s);
}

extern "C" {

xpipe_status xpipe_grad_norm_query(const xpipe_tensor* tensors, int32_t n_tensors, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  int64_t blocks = 0;
  XP_TRY(check_tensors(tensors, n_tensors, &blocks));
  *workspace_bytes = (size_t)blocks * sizeof(double);
  return XPIPE_OK;
}

xpipe_status xpipe_grad_norm(const xpipe_tensor* tensors, int32_t n_tensors, int32_t dtype, double max_norm,
                             double* sumsq, float* norm_coef, void* workspace, size_t workspace_bytes,
                             void* hip_stream) {
  int64_t blocks = 0;
  XP_TRY(check_tensors(tensors, n_tensors, &blocks));
  if (!known_dtype(dtype)) return fail(XPIPE_EINVAL, "unknown dtype");
  if (!sumsq && !norm_coef) return fail(XPIPE_EINVAL, "nothing to write");
  if (norm_coef && !(max_norm > 0)) return fail(XPIPE_EINVAL, "max_norm must be > 0");
  if (!at_multiple(sumsq, 8) || !at_multiple(norm_coef, 4)) return fail(XPIPE_EINVAL, "misaligned output");
  for (int32_t i = 0; i < n_tensors; ++i)
    if (!at_multiple(tensors[i].p, esize(dtype))) return fail(XPIPE_EINVAL, "a tensor is not aligned to its element");
  if (blocks > 0) {
    if (!workspace) return fail(XPIPE_EINVAL, "null workspace");
    if (workspace_bytes < (size_t)blocks * sizeof(double)) return fail(XPIPE_EINVAL, "workspace too small");
    if (!at_multiple(workspace, 8)) return fail(XPIPE_EINVAL, "workspace must be 8-byte aligned");
  }
  XP_HIP(grad_norm(tensors, n_tensors, dtype, max_norm, sumsq, norm_coef, (double*)workspace, blocks, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_clip_coef(const double* sumsq, int64_t n, double max_norm, float* norm_coef, void* hip_stream) {
  if (n < 0) return fail(XPIPE_EINVAL, "negative length");
  if (n > 0 && !sumsq) return fail(XPIPE_EINVAL, "null sumsq");
  if (!norm_coef) return fail(XPIPE_EINVAL, "null norm_coef");
  if (!(max_norm > 0)) return fail(XPIPE_EINVAL, "max_norm must be > 0");
  if (!at_multiple(sumsq, 8) || !at_multiple(norm_coef, 4)) return fail(XPIPE_EINVAL, "misaligned buffer");
  XP_HIP(launch_clip_coef(sumsq, n, max_norm, nullptr, norm_coef, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_linear_fwd_query(const xpipe_linear_fwd_args* args, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  LinearArgs a;
  XP_TRY(fwd_product(args, &a));
  *workspace_bytes = linear_bytes(args->dtype, &a, 1);
  return XPIPE_OK;
}

xpipe_status xpipe_linear_bwd_query(const xpipe_linear_bwd_args* args, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  LinearArgs p[2];
  XP_TRY(bwd_products(args, p));
  *workspace_bytes = linear_bytes(args->dtype, p, 2);
  return XPIPE_OK;
}

xpipe_status xpipe_linear_fwd(const xpipe_linear_fwd_args* args, void* workspace, size_t workspace_bytes,
                              void* hip_stream) {
  LinearArgs a;
  XP_TRY(fwd_product(args, &a));
  if (a.M == 0) return XPIPE_OK;
  XP_TRY(check_workspace(workspace, workspace_bytes, linear_bytes(args->dtype, &a, 1)));
  XP_HIP(launch_linear(args->dtype, &a, 1, workspace, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_linear_bwd(const xpipe_linear_bwd_args* args, void* workspace, size_t workspace_bytes,
                              void* hip_stream) {
  LinearArgs p[2];
  XP_TRY(bwd_products(args, p));
  XP_TRY(check_workspace(workspace, workspace_bytes, linear_bytes(args->dtype, p, 2)));
  XP_HIP(launch_linear(args->dtype, p, 2, workspace, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_act_bwd(const void* dy, const void* z, void* dz, int64_t n, int32_t act, int32_t dtype,
                           void* hip_stream) {
  if (n < 0) return fail(XPIPE_EINVAL, "negative length");
  if (!known_dtype(dtype)) return fail(XPIPE_EINVAL, "unknown dtype");
  if (act < XPIPE_ACT_NONE || act > XPIPE_ACT_SILU) return fail(XPIPE_EINVAL, "unknown activation");
  if (n == 0) return XPIPE_OK;
  if (!dy || !z || !dz) return fail(XPIPE_EINVAL, "null buffer");
  const int es = esize(dtype);
  if (!at_multiple(dy, es) || !at_multiple(z, es) || !at_multiple(dz, es))
    return fail(XPIPE_EINVAL, "a buffer is not aligned to its element");
  XP_HIP(launch_act_bwd(dtype, dy, z, dz, n, act, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_embedding_fwd(const void* table, const int32_t* tokens, int64_t n_tokens, int32_t vocab, int32_t dim,
                                 double scale, int32_t dtype, void* y, void* hip_stream) {
  XP_TRY(check_embedding(table, "table", tokens, n_tokens, vocab, dim, scale, dtype));
  if (n_tokens == 0) return XPIPE_OK;
  if (!y) return fail(XPIPE_EINVAL, "null y");
  if (!at_multiple(y, esize(dtype))) return fail(XPIPE_EINVAL, "y is not aligned to its element");
  if (y == table || y == (const void*)tokens) return fail(XPIPE_EINVAL, "y is an input's buffer");
  EmbedArgs a{};
  a.n = n_tokens;
  a.dim = dim;
  a.vocab = vocab;
  a.tokens = tokens;
  a.scale = scale;
  a.table = table;
  a.y = y;
  XP_HIP(launch_embed_fwd(dtype, a, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_embedding_bwd_query(int64_t n_tokens, int32_t vocab, int32_t dim, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  XP_TRY(check_embedding_sizes(n_tokens, vocab, dim));
  *workspace_bytes = embed_bwd_bytes(n_tokens, dim);
  return XPIPE_OK;
}

xpipe_status xpipe_embedding_bwd(const void* dy, const int32_t* tokens, int64_t n_tokens, int32_t vocab, int32_t dim,
                                 double scale, int32_t dtype, float* grad, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  XP_TRY(check_embedding(dy, "dy", tokens, n_tokens, vocab, dim, scale, dtype));
  if (n_tokens == 0) return XPIPE_OK;
  if (!grad) return fail(XPIPE_EINVAL, "null grad");
  if (!at_multiple(grad, 4)) return fail(XPIPE_EINVAL, "grad is not aligned to its element");
  if ((const void*)grad == dy || (const void*)grad == (const void*)tokens)
    return fail(XPIPE_EINVAL, "grad is an input's buffer");
  XP_TRY(check_workspace(workspace, workspace_bytes, embed_bwd_bytes(n_tokens, dim)));
  EmbedArgs a{};
  a.n = n_tokens;
  a.dim = dim;
  a.vocab = vocab;
  a.tokens = tokens;
  a.scale = scale;
  a.dy = dy;
  a.grad = grad;
  XP_HIP(launch_embed_bwd(dtype, a, workspace, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

}  // extern "C"
