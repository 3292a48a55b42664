// C-ABI of the sequence-surrogate operators (declared in baco_gp.h): argument checks and
// dispatch.
#include <cmath>
#include <cstring>

#include "seq.h"

using namespace bgp;

namespace {

gp_status bad(const std::string &msg) { return seq_fail(GP_E_INVALID, msg); }

gp_status check_attention(const gp_attention *t) {
  if (!t) return bad("attention description is NULL");
  if (t->dtype != GP_BF16 && t->dtype != GP_FP16)
    return seq_fail(GP_E_UNSUPPORTED, "attention takes GP_BF16 or GP_FP16");
  if (t->kv_heads < 1 || t->heads < 1 || t->heads % t->kv_heads)
    return bad("heads must be a positive multiple of kv_heads");
  if (t->heads > 65536) return seq_fail(GP_E_UNSUPPORTED, "more than 65536 heads");
  if (t->dim < 8 || t->dim > kSeqMaxDim || t->dim % 8)
    return seq_fail(GP_E_UNSUPPORTED, "head size must be a multiple of 8 in 8..128");
  if (t->n_docs < 0 || t->q_rows < 0 || t->k_rows < 0 || t->max_q < 0 || t->max_k < 0)
    return bad("negative size");
  if (t->q_rows > (1 << 30) || t->k_rows > (1 << 30) || t->n_docs > (1 << 24) ||
      t->max_q > t->q_rows || t->max_k > t->k_rows)
    return bad("need max_q <= q_rows, max_k <= k_rows, at most 2^30 rows and 2^24 documents");
  if (t->n_docs > 0 && (!t->q_begin || !t->q_end || !t->k_begin || !t->k_end))
    return bad("document ranges missing");
  if (t->prefix && !t->causal) return bad("a prefix needs a causal mask");
  if (!(t->scale > 0.f) || !std::isfinite(t->scale)) return bad("scale must be finite and > 0");
  if (!(t->cap >= 0.f) || !std::isfinite(t->cap)) return bad("cap must be finite and >= 0");
  if (t->per_side < 0 || t->per_side > kMaxBuckets)
    return seq_fail(GP_E_UNSUPPORTED, "1..64 buckets per side");
  if (t->per_side > 0) {
    if (t->slopes) return bad("a table and slopes exclude each other");
    if (!t->bucket_start) return bad("bucket_start is NULL");
    if (t->bucket_start[0] != 0) return bad("bucket_start[0] must be 0");
    for (int i = 1; i < t->per_side; ++i)
      if (t->bucket_start[i] <= t->bucket_start[i - 1])
        return bad("bucket_start must be strictly ascending");
    if (t->bucket_start[t->per_side - 1] > kMaxReach)
      return seq_fail(GP_E_UNSUPPORTED, "the last bucket must start at 1024 or less");
  }
  return GP_OK;
}

gp_status check_heads(const gp_heads *x, const char *name, int32_t rows) {
  const std::string n(name);
  if (!x) return bad(n + " is NULL");
  if (!x->data && rows > 0) return bad(n + ".data is NULL");
  if (reinterpret_cast<uintptr_t>(x->data) % 16)
    return seq_fail(GP_E_UNSUPPORTED, n + " must be 16-byte aligned");
  if (x->row < 0 || x->head < 0 || x->row % 8 || x->head % 8)
    return seq_fail(GP_E_UNSUPPORTED, n + "'s strides must be multiples of 8 elements, >= 0");
  if (x->row > (1 << 23)) return seq_fail(GP_E_UNSUPPORTED, n + "'s row stride is above 2^23");
  return GP_OK;
}

// A tensor that is written: no two of its rows and heads may share memory.
gp_status check_output(const gp_heads *x, const char *name, int32_t rows, int32_t heads, int32_t dim) {
  const gp_status st = check_heads(x, name, rows);
  if (st != GP_OK) return st;
  bool apart = (rows < 2 || x->row >= dim) && (heads < 2 || x->head >= dim);
  // head b is apart from head 0 if no row of it is within dim of one: the nearest two multiples
  for (int64_t b = 1; apart && rows > 1 && b < heads; ++b) {
    const int64_t at = b * x->head, r = at / x->row;
    apart = (r >= rows || at - r * x->row >= dim) && (r + 1 >= rows || (r + 1) * x->row - at >= dim);
  }
  return apart ? GP_OK : bad(std::string(name) + "'s rows or heads overlap");
}

AttnArgs make_args(const gp_attention *t) {
  AttnArgs a;
  std::memset(&a, 0, sizeof a);
  a.qb = t->q_begin, a.qe = t->q_end, a.kb = t->k_begin, a.ke = t->k_end, a.prefix = t->prefix;
  a.docs = t->n_docs, a.heads = t->heads, a.kv_heads = t->kv_heads;
  a.group = t->heads / t->kv_heads;
  a.bytes = 2 * t->dim;
  a.q_rows = t->q_rows, a.k_rows = t->k_rows, a.max_q = t->max_q, a.max_k = t->max_k;
  a.causal = t->causal ? 1 : 0;
  a.scale = t->scale, a.cap = t->cap;
  a.slopes = t->slopes;
  a.buckets.per_side = t->per_side;
  a.buckets.two_sided = t->two_sided ? 1 : 0;
  for (int i = 0; i < kMaxBuckets; ++i)
    a.buckets.start[i] = i < t->per_side ? t->bucket_start[i] : INT32_MAX;
  a.fp16 = t->dtype == GP_FP16;
  return a;
}

void set_tensors(AttnArgs &a, const gp_heads *q, const gp_heads *k, const gp_heads *v,
                 const gp_heads *o, const gp_heads *rest, const void *table, float *lse) {
  a.q = static_cast<const char *>(q->data);
  a.k = static_cast<const char *>(k->data);
  a.v = static_cast<const char *>(v->data);
  a.o = static_cast<char *>(o->data);
  a.q_row = 2 * q->row, a.q_head = 2 * q->head;
  a.k_row = 2 * k->row, a.k_head = 2 * k->head;
  a.v_row = 2 * v->row, a.v_head = 2 * v->head;
  a.o_row = 2 * o->row, a.o_head = 2 * o->head;
  if (rest) {
    a.rest = static_cast<char *>(rest->data);
    a.rest_row = 2 * rest->row, a.rest_head = 2 * rest->head;
  }
  a.table = table;
  a.lse = lse;
}

gp_status check_workspace(const void *ws, size_t bytes, size_t need) {
  if (need == 0) return GP_OK;
  if (!ws) return seq_fail(GP_E_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % 256)
    return seq_fail(GP_E_WORKSPACE, "workspace must be 256-byte aligned");
  if (bytes < need)
    return seq_fail(GP_E_WORKSPACE, "workspace too small: need " + std::to_string(need) +
                                        " bytes, have " + std::to_string(bytes));
  return GP_OK;
}

// The description, and whether its grids are within a launch's limits. (Before anything else of a
// call, so that a call with nothing but a description returns the description's own status.)
gp_status check_description(const gp_attention *t, bool grad) {
  const gp_status st = check_attention(t);
  if (st != GP_OK) return st;
  const AttnArgs a = make_args(t);
  const bool ok = grad ? attend_grad_fits(a)
                       : a.docs == 0 || a.max_q == 0 ||
                             (attend_use_few(a) ? attend_few_fits(a) : attend_fits(a));
  return ok ? GP_OK : seq_fail(GP_E_UNSUPPORTED, "too many tiles: a launch has at most 2^24 - 1 blocks");
}

size_t attend_bytes(const AttnArgs &a) {
  if (a.docs == 0 || a.max_q == 0 || !attend_use_few(a)) return 0;
  return attend_few_bytes(a);
}

gp_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return GP_OK;
  return seq_fail(GP_E_HIP, std::string(what) + " failed: " + hipGetErrorString(e));
}

gp_status check_logits(int32_t dtype, const void *x, int64_t stride, int32_t rows, int32_t width,
                       float scale, const char *name) {
  if (dtype != GP_BF16 && dtype != GP_FP16 && dtype != GP_FP32)
    return bad("dtype must be GP_BF16, GP_FP16 or GP_FP32");
  if (rows < 0) return bad("rows must be >= 0");
  if (width < 1) return bad("width must be >= 1");
  if (stride < 0) return bad("row strides must be >= 0");
  if (!x && rows > 0) return bad(std::string(name) + " is NULL");
  if (reinterpret_cast<uintptr_t>(x) % (dtype == GP_FP32 ? 4 : 2))
    return bad(std::string(name) + " is not aligned to its type");
  if (!(scale > 0.f) || !std::isfinite(scale)) return bad("scale must be finite and > 0");
  return GP_OK;
}

// From lse or from norm.
gp_status logprob_grad(int32_t dtype, const void *x, int64_t stride, int32_t rows, int32_t width,
                       float scale, const int64_t *target, const float *lse, const float *norm,
                       const float *entropy, const float *g_logp, const float *g_entropy, void *dx,
                       int64_t dx_stride, void *stream) {
  gp_status st = check_logits(dtype, x, stride, rows, width, scale, "x");
  if (st == GP_OK) st = check_logits(dtype, dx, dx_stride, rows, width, scale, "dx");
  if (st != GP_OK) return st;
  if (g_logp && !target) return bad("g_logp needs target");
  if (g_entropy && !entropy) return bad("g_entropy needs entropy");
  if (rows > 1 && dx_stride < width) return bad("rows of dx overlap");
  if (rows == 0) return GP_OK;
  LogprobArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = x, a.row = stride, a.rows = rows, a.width = width, a.dtype = dtype, a.scale = scale;
  a.target = target, a.lse = const_cast<float *>(lse), a.norm = const_cast<float *>(norm);
  a.entropy = const_cast<float *>(entropy);
  a.g_logp = g_logp, a.g_entropy = g_entropy, a.dx = dx, a.dx_row = dx_stride;
  return hip_status(launch_logprob_grad(a, static_cast<hipStream_t>(stream)),
                    "log probability gradient");
}

template <class F>
gp_status guarded(F f) {
  try {
    return f();
  } catch (const std::exception &e) {
    return seq_fail(GP_E_INVALID, std::string("internal error: ") + e.what());
  } catch (...) {
    return GP_E_INVALID;
  }
}

}  // namespace

extern "C" {

size_t gp_attend_workspace_bytes(const gp_attention *t, int32_t with_grad) {
  size_t n = SIZE_MAX;
  guarded([&] {
    const gp_status st = check_description(t, with_grad);
    if (st != GP_OK) return st;
    const AttnArgs a = make_args(t);
    n = with_grad ? attend_grad_bytes(a) : attend_bytes(a);
    return GP_OK;
  });
  return n;
}

gp_status gp_attend(const gp_attention *t, const gp_heads *q, const gp_heads *k, const gp_heads *v,
                    const void *table, const gp_heads *out, const gp_heads *rest, float *lse,
                    void *workspace, size_t ws_bytes, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_description(t, false);
    if (st == GP_OK) st = check_heads(q, "q", t->q_rows);
    if (st == GP_OK) st = check_heads(k, "k", t->k_rows);
    if (st == GP_OK) st = check_heads(v, "v", t->k_rows);
    if (st == GP_OK) st = check_output(out, "out", t->q_rows, t->heads, t->dim);
    if (st == GP_OK && rest) st = check_output(rest, "rest", t->q_rows, t->heads, t->dim);
    if (st != GP_OK) return st;
    if ((t->per_side > 0) != (table != nullptr)) return bad("a table goes with per_side > 0");
    if (!lse && t->q_rows > 0) return bad("lse is NULL");
    if (t->n_docs == 0 || t->max_q == 0) return GP_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    AttnArgs a = make_args(t);
    set_tensors(a, q, k, v, out, rest, table, lse);
    st = check_workspace(workspace, ws_bytes, attend_bytes(a));
    if (st != GP_OK) return st;
    if (attend_use_few(a))
      return hip_status(launch_attend_few(a, workspace, s), "attention");
    return hip_status(launch_attend(a, s), "attention");
  });
}

gp_status gp_attend_grad(const gp_attention *t, const gp_heads *q, const gp_heads *k,
                         const gp_heads *v, const void *table, const gp_heads *out,
                         const gp_heads *rest, const float *lse, const gp_heads *dout, const gp_heads *dq,
                         const gp_heads *dk, const gp_heads *dv, void *dtable, void *workspace,
                         size_t ws_bytes, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_description(t, true);
    if (st == GP_OK) st = check_heads(q, "q", t->q_rows);
    if (st == GP_OK) st = check_heads(k, "k", t->k_rows);
    if (st == GP_OK) st = check_heads(v, "v", t->k_rows);
    if (st == GP_OK) st = check_heads(out, "out", t->q_rows);
    if (st == GP_OK) st = check_heads(rest, "rest", t->q_rows);
    if (st == GP_OK) st = check_heads(dout, "dout", t->q_rows);
    if (st == GP_OK) st = check_output(dq, "dq", t->q_rows, t->heads, t->dim);
    if (st == GP_OK) st = check_output(dk, "dk", t->k_rows, t->kv_heads, t->dim);
    if (st == GP_OK) st = check_output(dv, "dv", t->k_rows, t->kv_heads, t->dim);
    if (st != GP_OK) return st;
    if ((t->per_side > 0) != (table != nullptr)) return bad("a table goes with per_side > 0");
    if ((table != nullptr) != (dtable != nullptr)) return bad("dtable goes with a table");
    if (!lse && t->q_rows > 0) return bad("lse is NULL");
    AttnGradArgs g;
    std::memset(&g, 0, sizeof g);
    g.f = make_args(t);
    set_tensors(g.f, q, k, v, out, rest, table, const_cast<float *>(lse));
    st = check_workspace(workspace, ws_bytes, attend_grad_bytes(g.f));
    if (st != GP_OK) return st;
    g.dout = static_cast<const char *>(dout->data);
    g.dq = static_cast<char *>(dq->data);
    g.dk = static_cast<char *>(dk->data);
    g.dv = static_cast<char *>(dv->data);
    g.dtable = dtable;
    g.do_row = 2 * dout->row, g.do_head = 2 * dout->head;
    g.dq_row = 2 * dq->row, g.dq_head = 2 * dq->head;
    g.dk_row = 2 * dk->row, g.dk_head = 2 * dk->head;
    g.dv_row = 2 * dv->row, g.dv_head = 2 * dv->head;
    return hip_status(launch_attend_grad(g, workspace, static_cast<hipStream_t>(stream)),
                      "attention gradient");
  });
}

size_t gp_logprob_workspace_bytes(int32_t rows, int32_t width, int32_t top) {
  if (rows < 1 || width < 1 || top < 0 || top > kMaxTop) return 0;
  return logprob_bytes(rows, width, top);
}

gp_status gp_logprob_norm(int32_t dtype, const void *x, int64_t stride, int32_t rows, int32_t width,
                          float scale, const int64_t *target, int32_t top, float *logp,
                          float *entropy, float *lse, float *norm, float *top_logp,
                          int64_t *top_id, void *workspace, size_t ws_bytes, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_logits(dtype, x, stride, rows, width, scale, "x");
    if (st != GP_OK) return st;
    if (top < 0 || top > width) return bad("top must be in 0..width");
    if (top > kMaxTop) return seq_fail(GP_E_UNSUPPORTED, "at most 128 alternatives");
    if (top > 0 && rows > 0 && (!top_logp || !top_id)) return bad("top_logp and top_id are required");
    if (logp && !target && rows > 0) return bad("logp needs target");
    if (rows == 0) return GP_OK;
    st = check_workspace(workspace, ws_bytes, logprob_bytes(rows, width, top));
    if (st != GP_OK) return st;
    LogprobArgs a;
    std::memset(&a, 0, sizeof a);
    a.x = x, a.row = stride, a.rows = rows, a.width = width, a.top = top, a.dtype = dtype;
    a.scale = scale, a.target = target, a.logp = logp, a.entropy = entropy, a.lse = lse;
    a.norm = norm, a.top_logp = top_logp, a.top_id = top_id;
    return hip_status(launch_logprob(a, workspace, static_cast<hipStream_t>(stream)),
                      "log probabilities");
  });
}

gp_status gp_logprob(int32_t dtype, const void *x, int64_t stride, int32_t rows, int32_t width,
                     float scale, const int64_t *target, int32_t top, float *logp, float *entropy,
                     float *lse, float *top_logp, int64_t *top_id, void *workspace, size_t ws_bytes,
                     void *stream) {
  return gp_logprob_norm(dtype, x, stride, rows, width, scale, target, top, logp, entropy, lse,
                         nullptr, top_logp, top_id, workspace, ws_bytes, stream);
}

gp_status gp_logprob_grad(int32_t dtype, const void *x, int64_t stride, int32_t rows, int32_t width,
                          float scale, const int64_t *target, const float *lse,
                          const float *entropy, const float *g_logp, const float *g_entropy,
                          void *dx, int64_t dx_stride, void *stream) {
  return guarded([&]() -> gp_status {
    if (rows > 0 && !lse) return bad("lse is NULL");
    return logprob_grad(dtype, x, stride, rows, width, scale, target, lse, nullptr, entropy, g_logp,
                        g_entropy, dx, dx_stride, stream);
  });
}

gp_status gp_logprob_norm_grad(int32_t dtype, const void *x, int64_t stride, int32_t rows,
                               int32_t width, float scale, const int64_t *target, const float *norm,
                               const float *entropy, const float *g_logp, const float *g_entropy,
                               void *dx, int64_t dx_stride, void *stream) {
  return guarded([&]() -> gp_status {
    if (rows > 0 && !norm) return bad("norm is NULL");
    return logprob_grad(dtype, x, stride, rows, width, scale, target, nullptr, norm, entropy, g_logp,
                        g_entropy, dx, dx_stride, stream);
  });
}

}  // extern "C"
