// C-ABI of a sequence surrogate's layers beside attention (declared in baco_gp.h): argument checks
// and dispatch.
#include <cmath>
#include <cstring>

#include "layer.h"

using namespace bgp;

namespace {

gp_status bad(const std::string &msg) { return seq_fail(GP_E_INVALID, msg); }
gp_status unsupported(const std::string &msg) { return seq_fail(GP_E_UNSUPPORTED, msg); }

bool is_type(int32_t t) { return t == GP_BF16 || t == GP_FP16 || t == GP_FP32; }
int size_of(int32_t t) { return t == GP_FP32 ? 4 : 2; }
bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

gp_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return GP_OK;
  return seq_fail(GP_E_HIP, std::string(what) + " failed: " + hipGetErrorString(e));
}

gp_status check_workspace(const void *ws, size_t bytes, size_t need) {
  if (need == 0) return GP_OK;
  if (!ws) return seq_fail(GP_E_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, 256)) return seq_fail(GP_E_WORKSPACE, "workspace must be 256-byte aligned");
  if (bytes < need)
    return seq_fail(GP_E_WORKSPACE, "workspace too small: need " + std::to_string(need) +
                                        " bytes, have " + std::to_string(bytes));
  return GP_OK;
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

// ------------------------------------------------------------------ norms
constexpr int kMaxWidth = 1 << 24;

gp_status check_norm(const gp_norm_spec *t, int32_t rows) {
  if (!t) return bad("norm description is NULL");
  if (!is_type(t->dtype)) return bad("dtype must be GP_BF16, GP_FP16 or GP_FP32");
  if (t->weight_dtype != t->dtype && t->weight_dtype != GP_FP32)
    return unsupported("weight_dtype must be dtype or GP_FP32");
  if (t->width < 1) return bad("width must be >= 1");
  if (t->width > kMaxWidth) return unsupported("at most 2^24 entries a row");
  if (!(t->eps > 0.f) || !std::isfinite(t->eps)) return bad("eps must be finite and > 0");
  if (rows < 0) return bad("rows must be >= 0");
  return GP_OK;
}
gp_status check_rows(const void *p, int64_t stride, const gp_norm_spec *t, int32_t rows, bool written,
                     const char *name) {
  const std::string n(name);
  if (!p) return rows > 0 ? bad(n + " is NULL") : GP_OK;
  if (!aligned(p, size_of(t->dtype))) return bad(n + " is not aligned to its type");
  if (stride < 0) return bad(n + "'s stride must be >= 0");
  if (written && rows > 1 && stride < t->width) return bad("rows of " + n + " overlap");
  return GP_OK;
}
gp_status check_weight(const void *p, const gp_norm_spec *t, const char *name) {
  if (!aligned(p, size_of(t->weight_dtype))) return bad(std::string(name) + " is not aligned to its type");
  return GP_OK;
}

NormGradArgs norm_grad_args(const gp_norm_spec *t, int32_t rows, void *dweight, void *dbias) {
  NormGradArgs a;
  std::memset(&a, 0, sizeof a);
  a.rows = rows, a.width = t->width, a.dtype = t->dtype, a.weight_dtype = t->weight_dtype;
  a.centre = t->centre != 0, a.dweight = dweight, a.dbias = dbias;
  return a;
}

// ------------------------------------------------------------------ rotary positions
gp_status check_rotary(const gp_rotary *t, int32_t rows, const int32_t *positions) {
  if (!t) return bad("rotary description is NULL");
  if (!is_type(t->dtype)) return bad("dtype must be GP_BF16, GP_FP16 or GP_FP32");
  if (t->dim < 8 || t->dim > kSeqMaxDim || t->dim % 8)
    return unsupported("head size must be a multiple of 8 in 8..128");
  if (t->rotated < 2 || t->rotated > t->dim || t->rotated % 2)
    return bad("rotated must be even, in 2..dim");
  if (!t->turns || !aligned(t->turns, 8)) return bad("turns is NULL or not aligned");
  if (!std::isfinite(t->magnitude)) return bad("magnitude must be finite");
  if (rows < 0) return bad("rows must be >= 0");
  if (rows > (1 << 30)) return unsupported("at most 2^30 rows");
  if (rows > 0 && (!positions || !aligned(positions, 4))) return bad("positions is NULL or not aligned");
  return GP_OK;
}
gp_status check_heads(const gp_heads *x, int64_t rows, int32_t heads, const gp_rotary *t, bool written,
                      const char *name) {
  const std::string n(name);
  if (!x) return bad(n + " is NULL");
  if (heads < 1) return bad("heads must be >= 1");
  if (heads > 65536) return unsupported("more than 65536 heads");
  if (!x->data && rows > 0) return bad(n + ".data is NULL");
  if (!aligned(x->data, 16)) return unsupported(n + " must be 16-byte aligned");
  if (x->row < 0 || x->head < 0 || x->row % 8 || x->head % 8)
    return unsupported(n + "'s strides must be multiples of 8 elements, >= 0");
  if (x->row > (1 << 23)) return unsupported(n + "'s row stride is above 2^23");
  if (!written) return GP_OK;
  // no two rows or heads may share memory: head b is apart from head 0 if no row of it is within
  // dim of one (the nearest two multiples of the row stride)
  bool apart = (rows < 2 || x->row >= t->dim) && (heads < 2 || x->head >= t->dim);
  for (int64_t b = 1; apart && rows > 1 && b < heads; ++b) {
    const int64_t at = b * x->head, r = at / x->row;
    apart = (r >= rows || at - r * x->row >= t->dim) &&
            (r + 1 >= rows || (r + 1) * x->row - at >= t->dim);
  }
  return apart ? GP_OK : bad(n + "'s rows or heads overlap");
}
RotateArgs rotate_args(const gp_rotary *t, int32_t rows, const int32_t *positions) {
  RotateArgs a;
  std::memset(&a, 0, sizeof a);
  a.positions = positions, a.turns = t->turns, a.magnitude = t->magnitude;
  a.rows = rows, a.dim = t->dim, a.rotated = t->rotated, a.interleaved = t->interleaved != 0;
  a.dtype = t->dtype;
  return a;
}
RotateArgs::Part part_of(const gp_heads *in, const gp_heads *out, int32_t heads, int size) {
  return {static_cast<const char *>(in->data), static_cast<char *>(out->data), in->row * size,
          in->head * size, out->row * size, out->head * size, heads};
}

// ------------------------------------------------------------------ gated block
constexpr int64_t kMaxRowStride = 1 << 21;   // elements: a tile's rows stay within a buffer's 2^31

gp_status check_gated(const gp_gated_spec *t, int32_t rows, bool grad) {
  if (!t) return bad("gated block's description is NULL");
  if (t->dtype != GP_BF16 && t->dtype != GP_FP16)
    return unsupported("the gated block takes GP_BF16 or GP_FP16");
  if (t->activation != GP_SILU && t->activation != GP_GELU)
    return bad("activation must be GP_SILU or GP_GELU");
  if (t->width < 8 || t->hidden < 8 || t->width % 8 || t->hidden % 8)
    return unsupported("width and hidden must be multiples of 8");
  if (t->width > kMaxRowStride || t->hidden > kMaxRowStride)
    return unsupported("width and hidden must be 2^21 or less");
  if (rows < 0) return bad("rows must be >= 0");
  if (!gated_fits(rows, t->width, t->hidden, grad)) return unsupported("too many tiles for a launch");
  return GP_OK;
}
gp_status check_matrix(const gp_matrix *x, int64_t rows, int64_t width, bool written, const char *name) {
  const std::string n(name);
  if (!x) return bad(n + " is NULL");
  if (!x->data && rows > 0) return bad(n + ".data is NULL");
  if (!aligned(x->data, 16)) return unsupported(n + " must be 16-byte aligned");
  if (x->row < 0 || x->row % 8) return unsupported(n + "'s row stride must be a multiple of 8 elements, >= 0");
  if (x->row > kMaxRowStride) return unsupported(n + "'s row stride is above 2^21");
  if (written && rows > 1 && x->row < width) return bad("rows of " + n + " overlap");
  return GP_OK;
}
GatedArgs gated_args(const gp_gated_spec *t, int32_t rows, const gp_matrix *x, const gp_matrix *gate,
                     const gp_matrix *up) {
  GatedArgs a;
  std::memset(&a, 0, sizeof a);
  a.x = static_cast<const char *>(x->data), a.x_row = 2 * x->row;
  a.w_gate = static_cast<const char *>(gate->data), a.gate_row = 2 * gate->row;
  a.w_up = static_cast<const char *>(up->data), a.up_row = 2 * up->row;
  a.rows = rows, a.width = t->width, a.hidden = t->hidden, a.act = t->activation;
  a.fp16 = t->dtype == GP_FP16;
  return a;
}

}  // namespace

extern "C" {

gp_status gp_norm(const gp_norm_spec *t, int32_t rows, const void *x, int64_t x_stride,
                  const void *residual, int64_t residual_stride, const void *weight, const void *bias,
                  void *out, int64_t out_stride, void *sum, int64_t sum_stride, float *stats,
                  void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_norm(t, rows);
    if (st == GP_OK) st = check_rows(x, x_stride, t, rows, false, "x");
    if (st == GP_OK) st = check_rows(out, out_stride, t, rows, true, "out");
    if (st == GP_OK) st = check_weight(weight, t, "weight");
    if (st == GP_OK) st = check_weight(bias, t, "bias");
    if (st == GP_OK && residual) {
      st = check_rows(residual, residual_stride, t, rows, false, "residual");
      if (st == GP_OK) st = check_rows(sum, sum_stride, t, rows, true, "sum");
    }
    if (st != GP_OK) return st;
    if (!residual && sum) return bad("a sum needs a residual");
    if (!aligned(stats, 4)) return bad("stats is not aligned to its type");
    if (rows == 0) return GP_OK;
    if (residual && out == sum) return bad("out and sum are the same");
    NormArgs a;
    std::memset(&a, 0, sizeof a);
    a.x = {x, x_stride}, a.residual = {residual, residual_stride};
    a.out = {out, out_stride}, a.sum = {sum, sum_stride};
    a.weight = weight, a.bias = bias, a.stats = stats;
    a.rows = rows, a.width = t->width, a.dtype = t->dtype, a.weight_dtype = t->weight_dtype;
    a.centre = t->centre != 0, a.eps = t->eps;
    return hip_status(launch_norm(a, static_cast<hipStream_t>(stream)), "norm");
  });
}

size_t gp_norm_grad_workspace_bytes(const gp_norm_spec *t, int32_t rows) {
  size_t n = SIZE_MAX;
  guarded([&] {
    const gp_status st = check_norm(t, rows);
    if (st != GP_OK) return st;
    char any;
    n = norm_grad_bytes(norm_grad_args(t, rows, &any, &any));
    return GP_OK;
  });
  return n;
}

gp_status gp_norm_grad(const gp_norm_spec *t, int32_t rows, const void *h, int64_t h_stride,
                       const float *stats, const void *weight, const void *dout, int64_t dout_stride,
                       const void *dsum, int64_t dsum_stride, void *dx, int64_t dx_stride, void *dweight,
                       void *dbias, void *workspace, size_t ws_bytes, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_norm(t, rows);
    if (st == GP_OK) st = check_rows(h, h_stride, t, rows, false, "h");
    if (st == GP_OK) st = check_rows(dout, dout_stride, t, rows, false, "dout");
    if (st == GP_OK && dsum) st = check_rows(dsum, dsum_stride, t, rows, false, "dsum");
    if (st == GP_OK) st = check_rows(dx, dx_stride, t, rows, true, "dx");
    if (st == GP_OK) st = check_weight(weight, t, "weight");
    if (st == GP_OK) st = check_weight(dweight, t, "dweight");
    if (st == GP_OK) st = check_weight(dbias, t, "dbias");
    if (st != GP_OK) return st;
    if (!stats && rows > 0) return bad("stats is NULL");
    if (!aligned(stats, 4)) return bad("stats is not aligned to its type");
    NormGradArgs a = norm_grad_args(t, rows, dweight, dbias);
    st = check_workspace(workspace, ws_bytes, norm_grad_bytes(a));
    if (st != GP_OK) return st;
    a.h = {h, h_stride}, a.dout = {dout, dout_stride}, a.dsum = {dsum, dsum_stride};
    a.dx = {dx, dx_stride}, a.stats = stats, a.weight = weight;
    return hip_status(launch_norm_grad(a, workspace, static_cast<hipStream_t>(stream)), "norm gradient");
  });
}

gp_status gp_rotate(const gp_rotary *t, int32_t rows, const int32_t *positions, int32_t heads,
                    const gp_heads *x, const gp_heads *out, int32_t inverse, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_rotary(t, rows, positions);
    if (st == GP_OK) st = check_heads(x, rows, heads, t, false, "x");
    if (st == GP_OK) st = check_heads(out, rows, heads, t, true, "out");
    if (st != GP_OK) return st;
    RotateArgs a = rotate_args(t, rows, positions);
    a.inverse = inverse != 0;
    a.part[0] = part_of(x, out, heads, size_of(t->dtype));
    return hip_status(launch_rotate(a, static_cast<hipStream_t>(stream)), "rotary positions");
  });
}

gp_status gp_rotate_append(const gp_rotary *t, int32_t rows, const int32_t *positions,
                           const int64_t *slots, int32_t heads, const gp_heads *q, const gp_heads *out,
                           int32_t kv_heads, const gp_heads *k, const gp_heads *v, int64_t cache_rows,
                           const gp_heads *k_cache, const gp_heads *v_cache, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_rotary(t, rows, positions);
    if (st == GP_OK) st = check_heads(q, rows, heads, t, false, "q");
    if (st == GP_OK) st = check_heads(out, rows, heads, t, true, "out");
    if (st == GP_OK) st = check_heads(k, rows, kv_heads, t, false, "k");
    if (st == GP_OK) st = check_heads(v, rows, kv_heads, t, false, "v");
    if (st == GP_OK) st = check_heads(k_cache, cache_rows, kv_heads, t, true, "k_cache");
    if (st == GP_OK) st = check_heads(v_cache, cache_rows, kv_heads, t, true, "v_cache");
    if (st != GP_OK) return st;
    if (cache_rows < 0) return bad("cache_rows must be >= 0");
    if (rows > 0 && (!slots || !aligned(slots, 8))) return bad("slots is NULL or not aligned");
    RotateArgs a = rotate_args(t, rows, positions);
    const int size = size_of(t->dtype);
    a.slots = slots, a.slot_rows = cache_rows;
    a.part[0] = part_of(q, out, heads, size);
    a.part[1] = part_of(k, k_cache, kv_heads, size);
    a.part[2] = part_of(v, v_cache, kv_heads, size);
    return hip_status(launch_rotate(a, static_cast<hipStream_t>(stream)), "rotary positions");
  });
}

gp_status gp_gated(const gp_gated_spec *t, int32_t rows, const gp_matrix *x, const gp_matrix *w_gate,
                   const gp_matrix *w_up, const gp_matrix *out, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_gated(t, rows, false);
    if (st == GP_OK) st = check_matrix(x, rows, t->width, false, "x");
    if (st == GP_OK) st = check_matrix(w_gate, t->hidden, t->width, false, "w_gate");
    if (st == GP_OK) st = check_matrix(w_up, t->hidden, t->width, false, "w_up");
    if (st == GP_OK) st = check_matrix(out, rows, t->hidden, true, "out");
    if (st != GP_OK) return st;
    GatedArgs a = gated_args(t, rows, x, w_gate, w_up);
    a.out = static_cast<char *>(out->data), a.out_row = 2 * out->row;
    return hip_status(launch_gated(a, static_cast<hipStream_t>(stream)), "gated block");
  });
}

size_t gp_gated_grad_workspace_bytes(const gp_gated_spec *t, int32_t rows) {
  size_t n = SIZE_MAX;
  guarded([&] {
    const gp_status st = check_gated(t, rows, true);
    if (st == GP_OK) n = gated_grad_bytes(rows, t->width, t->hidden, t->dtype == GP_FP16);
    return st;
  });
  return n;
}

gp_status gp_gated_grad(const gp_gated_spec *t, int32_t rows, const gp_matrix *x,
                        const gp_matrix *w_gate, const gp_matrix *w_up, const gp_matrix *dout,
                        const gp_matrix *dx, const gp_matrix *dw_gate, const gp_matrix *dw_up,
                        void *workspace, size_t ws_bytes, void *stream) {
  return guarded([&]() -> gp_status {
    gp_status st = check_gated(t, rows, true);
    if (st == GP_OK) st = check_matrix(x, rows, t->width, false, "x");
    if (st == GP_OK) st = check_matrix(w_gate, t->hidden, t->width, false, "w_gate");
    if (st == GP_OK) st = check_matrix(w_up, t->hidden, t->width, false, "w_up");
    if (st == GP_OK) st = check_matrix(dout, rows, t->hidden, false, "dout");
    if (st == GP_OK) st = check_matrix(dx, rows, t->width, true, "dx");
    if (st == GP_OK) st = check_matrix(dw_gate, t->hidden, t->width, true, "dw_gate");
    if (st == GP_OK) st = check_matrix(dw_up, t->hidden, t->width, true, "dw_up");
    if (st != GP_OK) return st;
    st = check_workspace(workspace, ws_bytes,
                         gated_grad_bytes(rows, t->width, t->hidden, t->dtype == GP_FP16));
    if (st != GP_OK) return st;
    GatedGradArgs g;
    std::memset(&g, 0, sizeof g);
    g.f = gated_args(t, rows, x, w_gate, w_up);
    g.dout = static_cast<const char *>(dout->data), g.dout_row = 2 * dout->row;
    g.dx = static_cast<char *>(dx->data), g.dx_row = 2 * dx->row;
    g.dw_gate = static_cast<char *>(dw_gate->data), g.dgate_row = 2 * dw_gate->row;
    g.dw_up = static_cast<char *>(dw_up->data), g.dup_row = 2 * dw_up->row;
    return hip_status(launch_gated_grad(g, workspace, static_cast<hipStream_t>(stream)),
                      "gated block's gradient");
  });
}

gp_status gp_adamw(const gp_adamw_spec *t, int32_t count, const gp_adamw_tensor *tensors,
                   const void *const *grads, void *stream) {
  return guarded([&]() -> gp_status {
    if (!t) return bad("AdamW's description is NULL");
    if (!is_type(t->dtype)) return bad("dtype must be GP_BF16, GP_FP16 or GP_FP32");
    if (t->grad_dtype != t->dtype && t->grad_dtype != GP_FP32)
      return unsupported("grad_dtype must be dtype or GP_FP32");
    if (t->state_bits != 8 && t->state_bits != 32) return unsupported("states have 8 or 32 bits");
    if (!(t->beta1 >= 0. && t->beta1 < 1. && t->beta2 >= 0. && t->beta2 < 1.))
      return bad("beta1 and beta2 must be in 0..1, below 1");
    // (in fp32, as the kernels take it)
    if (!((float)t->eps > 0.f) || !std::isfinite((float)t->eps)) return bad("eps must be finite and > 0 in fp32");
    if (!std::isfinite(t->decay)) return bad("decay must be finite");
    if (!t->lr_device && !std::isfinite(t->lr)) return bad("lr must be finite");
    if (!t->step_device && t->step < 1) return bad("step must be >= 1");
    if (!aligned(t->lr_device, 4) || !aligned(t->factor, 4) || !aligned(t->step_device, 8))
      return bad("lr_device, factor or step_device is not aligned");
    if (count < 0) return bad("negative number of tensors");
    if (count > 0 && (!tensors || !grads)) return bad("tensors or grads is NULL");
    const uintptr_t size = size_of(t->dtype), gsize = size_of(t->grad_dtype);
    const uintptr_t ssize = t->state_bits == 8 ? 1 : 4;
    for (int32_t i = 0; i < count; ++i) {
      const gp_adamw_tensor &x = tensors[i];
      const std::string n = "tensor " + std::to_string(i);
      if (x.count < 0) return bad(n + ": negative count");
      if (x.count > (int64_t)1 << 40) return unsupported(n + " has more than 2^40 values");
      if (x.count == 0 || !grads[i]) continue;
      if (!x.param || !x.m || !x.v) return bad(n + ": param, m or v is NULL");
      if (x.master && t->dtype == GP_FP32) return bad(n + ": a master copy goes with 16-bit weights");
      if ((t->state_bits == 8) != (x.scales != nullptr)) return bad(n + ": scales go with 8-bit states");
      if (!aligned(x.param, size) || !aligned(grads[i], gsize) || !aligned(x.master, 4) ||
          !aligned(x.m, ssize) || !aligned(x.v, ssize) || !aligned(x.scales, 4))
        return bad(n + " is not aligned to its type");
    }
    AdamArgs a;
    std::memset(&a, 0, sizeof a);
    a.dtype = t->dtype, a.grad_dtype = t->grad_dtype;
    a.key0 = (uint32_t)t->seed, a.key1 = (uint32_t)(t->seed >> 32);
    a.step = t->step, a.step_dev = t->step_device, a.lr_dev = t->lr_device, a.factor = t->factor;
    a.beta1 = t->beta1, a.beta2 = t->beta2, a.lr = t->lr, a.eps = t->eps, a.decay = t->decay;
    uint64_t first = 0;
    for (int32_t i = 0; i < count; ++i) {
      const gp_adamw_tensor &x = tensors[i];
      if (x.count > 0 && grads[i])
        a.t[a.n++] = {x.param, x.master, x.m, x.v, grads[i], x.scales, x.count, 0, first};
      first += (uint64_t)((x.count + 255) / 256);
      if (a.n == kAdamTensors || (i == count - 1 && a.n > 0)) {
        const gp_status st = hip_status(launch_adamw(a, t->state_bits, static_cast<hipStream_t>(stream)), "AdamW");
        if (st != GP_OK) return st;
        a.n = 0;
      }
    }
    return GP_OK;
  });
}

}  // extern "C"
