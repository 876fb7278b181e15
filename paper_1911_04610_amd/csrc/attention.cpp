// C ABI of attention: every argument is checked on the host, then kernels are
// enqueued on the caller's stream; nothing is kept between calls.
#include "xp_host.h"

#include <algorithm>
#include <cmath>

using namespace xp;

namespace {

// a matrix [batch][tokens][heads][dim]
xpipe_status check_heads(const char* name, const xpipe_heads& m, int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int es,
                         bool written) {
  if (batch * tokens * heads == 0) return XPIPE_OK;
  if (!m.p) return fail(XPIPE_EINVAL, std::string("null ") + name);
  if (!at_multiple(m.p, es)) return fail(XPIPE_EINVAL, std::string(name) + " is not aligned to its element");
  if (m.batch < 0 || m.token < 0 || m.head < 0) return fail(XPIPE_EINVAL, std::string(name) + ": negative stride");
  if ((tokens > 1 && m.token > XPIPE_ATTENTION_MAX_STRIDE) || (heads > 1 && m.head >= (int64_t)1 << 40) ||
      (batch > 1 && m.batch >= (int64_t)1 << 40))
    return fail(XPIPE_EUNSUPPORTED, std::string(name) + ": a stride too large");
  if (written) {  // each stride at least as long as what the smaller ones span
    std::pair<int64_t, int64_t> d[3] = {{m.batch, batch}, {m.token, tokens}, {m.head, heads}};
    std::sort(d, d + 3);
    int64_t span = dim;
    for (const auto& [stride, n] : d) {
      if (n <= 1) continue;
      if (stride < span) return fail(XPIPE_EINVAL, std::string(name) + ": elements of an output fall together");
      span += (n - 1) * stride;
    }
  }
  return XPIPE_OK;
}

AttnMat matrix(const xpipe_heads& m) { return {m.p, m.batch, m.token, m.head}; }

xpipe_status check_inputs(const xpipe_attention_inputs& q, AttnArgs* a) {
  *a = AttnArgs{};
  if (q.batch < 0 || q.nq < 0 || q.nk < 0 || q.heads < 1 || q.kv_heads < 1 || q.head_dim < 1)
    return fail(XPIPE_EINVAL, "batch, nq and nk must be >= 0, heads, kv_heads and head_dim >= 1");
  if (q.heads % q.kv_heads != 0) return fail(XPIPE_EINVAL, "heads must be a multiple of kv_heads");
  if (!known_dtype(q.dtype)) return fail(XPIPE_EINVAL, "unknown dtype");
  if (!(q.scale > 0) || !std::isfinite((float)q.scale) || !((float)q.scale > 0)) return fail(XPIPE_EINVAL, "scale must be > 0 and finite");
  if (!(q.cap >= 0) || !std::isfinite((float)q.cap) || (q.cap > 0 && !((float)q.cap > 0)))
    return fail(XPIPE_EINVAL, "cap must be >= 0 and finite");
  // (factors that a kernel forms of them)
  if (!std::isfinite(4.f * (float)q.scale) || !std::isfinite(4.f * (float)q.cap) || (q.cap > 0 && !std::isfinite(4.f * (float)q.scale / (float)q.cap)))
    return fail(XPIPE_EINVAL, "scale, cap or their quotient too large for fp32");
  if (q.head_dim > ATTN_MAX_DIM) return fail(XPIPE_EUNSUPPORTED, "head_dim beyond 128");
  // (a launch has less than 2^32 threads)
  if (q.nq >= 1 << 24 || q.nk >= 1 << 24 || (int64_t)q.batch * q.heads >= 1 << 23 ||
      (int64_t)q.batch * q.heads * (q.nq / 128 + 1) >= 1 << 23 || (int64_t)q.batch * q.heads * (q.nk / 128 + 1) >= 1 << 23)
    return fail(XPIPE_EUNSUPPORTED, "2^24 tokens of a sequence, or 2^23 blocks of 128 rows, or more");
  if (q.batch > 65535) return fail(XPIPE_EUNSUPPORTED, "more than 65535 sequences");
  if (q.heads > 65535) return fail(XPIPE_EUNSUPPORTED, "more than 65535 heads");
  if (q.prefix && !q.causal) return fail(XPIPE_EINVAL, "prefix without causal");
  // (documents of nothing may be null; no pair is left to hide then)
  const bool pairs = (int64_t)q.batch * q.nq > 0 && (int64_t)q.batch * q.nk > 0;
  if (pairs && (q.q_doc != nullptr) != (q.k_doc != nullptr)) return fail(XPIPE_EINVAL, "q_doc without k_doc, or k_doc without q_doc");
  if (q.bias && q.bias_range < 1) return fail(XPIPE_EINVAL, "bias_range must be >= 1");
  if (q.bias && q.bias_range > 1 << 20) return fail(XPIPE_EUNSUPPORTED, "bias_range beyond 2^20");
  for (const void* p : {(const void*)q.q_len, (const void*)q.k_len, (const void*)q.prefix, (const void*)q.q_doc, (const void*)q.k_doc,
                        (const void*)q.bias})
    if (!at_multiple(p, 4)) return fail(XPIPE_EINVAL, "lengths, prefix, documents or bias not aligned to their element");
  const int es = esize(q.dtype);
  XP_TRY(check_heads("q", q.q, q.batch, q.nq, q.heads, q.head_dim, es, false));
  XP_TRY(check_heads("k", q.k, q.batch, q.nk, q.kv_heads, q.head_dim, es, false));
  XP_TRY(check_heads("v", q.v, q.batch, q.nk, q.kv_heads, q.head_dim, es, false));
  a->batch = q.batch;
  a->nq = q.nq;
  a->nk = q.nk;
  a->heads = q.heads;
  a->kv_heads = q.kv_heads;
  a->dim = q.head_dim;
  a->causal = q.causal != 0;
  a->range = q.bias ? q.bias_range : 0;
  a->scale = (float)q.scale;
  a->cap = (float)q.cap;
  a->q = matrix(q.q);
  a->k = matrix(q.k);
  a->v = matrix(q.v);
  a->q_len = q.q_len;
  a->k_len = q.k_len;
  a->prefix = q.prefix;
  a->q_doc = pairs ? q.q_doc : nullptr;
  a->k_doc = pairs ? q.k_doc : nullptr;
  a->bias = q.bias;
  return XPIPE_OK;
}

// whether an output is one of the inputs' buffers, or another output's
bool is_input(const xpipe_attention_inputs& q, const void* p) {
  for (const void* i : {q.q.p, q.k.p, q.v.p, (const void*)q.q_len, (const void*)q.k_len, (const void*)q.prefix, (const void*)q.q_doc,
                        (const void*)q.k_doc, (const void*)q.bias})
    if (p && p == i) return true;
  return false;
}
bool all_differ(std::initializer_list<const void*> v) {
  for (auto i = v.begin(); i != v.end(); ++i)
    for (auto j = v.begin(); j != i; ++j)
      if (*i && *i == *j) return false;
  return true;
}

xpipe_status fwd_args(const xpipe_attention_fwd_args* q, AttnArgs* a) {
  if (!q) return fail(XPIPE_EINVAL, "null arguments");
  XP_TRY(check_inputs(q->in, a));
  XP_TRY(check_heads("o", q->o, a->batch, a->nq, a->heads, a->dim, esize(q->in.dtype), true));
  if (!at_multiple(q->stats, 4)) return fail(XPIPE_EINVAL, "stats not aligned to its element");
  if (!all_differ({q->o.p, q->stats}) || is_input(q->in, q->o.p) || is_input(q->in, q->stats))
    return fail(XPIPE_EINVAL, "an output is an input's or another output's buffer");
  a->o = matrix(q->o);
  a->stats = q->stats;
  return XPIPE_OK;
}

xpipe_status bwd_args(const xpipe_attention_bwd_args* q, AttnArgs* a) {
  if (!q) return fail(XPIPE_EINVAL, "null arguments");
  XP_TRY(check_inputs(q->in, a));
  const int es = esize(q->in.dtype);
  if (q->grad_bias && !q->in.bias) return fail(XPIPE_EINVAL, "grad_bias without bias");
  XP_TRY(check_heads("dout", q->dout, a->batch, a->nq, a->heads, a->dim, es, false));
  XP_TRY(check_heads("o", q->o, a->batch, a->nq, a->heads, a->dim, es, false));
  XP_TRY(check_heads("dq", q->dq, a->batch, a->nq, a->heads, a->dim, es, true));
  XP_TRY(check_heads("dk", q->dk, a->batch, a->nk, a->kv_heads, a->dim, es, true));
  XP_TRY(check_heads("dv", q->dv, a->batch, a->nk, a->kv_heads, a->dim, es, true));
  if (!q->stats && (int64_t)a->batch * a->nq > 0) return fail(XPIPE_EINVAL, "null stats");
  if (!at_multiple(q->stats, 4) || !at_multiple(q->grad_bias, 4)) return fail(XPIPE_EINVAL, "stats or grad_bias not aligned to its element");
  if (!all_differ({q->dq.p, q->dk.p, q->dv.p, q->grad_bias}))
    return fail(XPIPE_EINVAL, "two outputs are one buffer");
  for (const void* p : {q->dq.p, q->dk.p, q->dv.p, (const void*)q->grad_bias})
    if (p && (is_input(q->in, p) || p == q->dout.p || p == q->o.p || p == q->stats))
      return fail(XPIPE_EINVAL, "an output is an input's buffer");
  a->dout = matrix(q->dout);
  a->o = matrix(q->o);
  a->stats = const_cast<float*>(q->stats);
  a->dq = matrix(q->dq);
  a->dk = matrix(q->dk);
  a->dv = matrix(q->dv);
  a->grad_bias = q->grad_bias;
  return XPIPE_OK;
}

}  // namespace

extern "C" {

xpipe_status xpipe_attention_fwd_query(const xpipe_attention_fwd_args* args, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  AttnArgs a;
  XP_TRY(fwd_args(args, &a));
  *workspace_bytes = attn_fwd_bytes(args->in.dtype, a);
  return XPIPE_OK;
}

xpipe_status xpipe_attention_bwd_query(const xpipe_attention_bwd_args* args, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(XPIPE_EINVAL, "null output");
  AttnArgs a;
  XP_TRY(bwd_args(args, &a));
  *workspace_bytes = attn_bwd_bytes(args->in.dtype, a);
  return XPIPE_OK;
}

xpipe_status xpipe_attention_fwd(const xpipe_attention_fwd_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AttnArgs a;
  XP_TRY(fwd_args(args, &a));
  if ((int64_t)a.batch * a.nq == 0) return XPIPE_OK;
  XP_TRY(check_workspace(workspace, workspace_bytes, attn_fwd_bytes(args->in.dtype, a)));
  XP_HIP(launch_attn_fwd(args->in.dtype, a, workspace, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

xpipe_status xpipe_attention_bwd(const xpipe_attention_bwd_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AttnArgs a;
  XP_TRY(bwd_args(args, &a));
  if (a.batch == 0 || (a.nq == 0 && a.nk == 0)) return XPIPE_OK;
  XP_TRY(check_workspace(workspace, workspace_bytes, attn_bwd_bytes(args->in.dtype, a)));
  XP_HIP(launch_attn_bwd(args->in.dtype, a, workspace, (hipStream_t)hip_stream));
  return XPIPE_OK;
}

}  // extern "C"
