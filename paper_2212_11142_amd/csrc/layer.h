// Internal declarations of a sequence surrogate's layers beside attention: norms (norm.hip),
// rotary positions (rotate.hip), the gated feed-forward block (gated.hip) and AdamW (adamw.hip);
// their C-ABI is in layer_abi.hip.
#pragma once
#include "seq.h"

namespace bgp {

// Rows of a matrix: row r at data + r * row (elements).
struct Rows {
  const void *data;
  int64_t row;
};

struct NormArgs {
  Rows x, residual;                    // residual.data may be null
  Rows out, sum;                       // written; sum with a residual
  const void *weight, *bias;           // null: 1 and 0
  float *stats;                        // [rows][2] mean, 1 / sqrt(var + eps); null: not kept
  int32_t rows, width, dtype, weight_dtype, centre;
  float eps;
};
hipError_t launch_norm(const NormArgs &a, hipStream_t s);

struct NormGradArgs {
  Rows h, dout, dsum, dx;              // dsum.data may be null; dx is written
  const void *weight;                  // null: 1
  const float *stats;
  void *dweight, *dbias;               // of weight_dtype; null: not wanted
  int32_t rows, width, dtype, weight_dtype, centre;
  // workspace
  float *part;                         // [blocks][2][width] sums of the weight's and bias's gradients
  float *sums;                         // wide rows: [rows][2] means of g and g xh
};
size_t norm_grad_bytes(const NormGradArgs &a);
hipError_t launch_norm_grad(NormGradArgs a, void *ws, hipStream_t s);

struct RotateArgs {
  // parts of a row's heads: 0 is rotated and stays in its row, 1 is rotated and 2 copied into row
  // slots[r] of its output (with slots)
  struct Part {
    const char *in;
    char *out;
    int64_t in_row, in_head, out_row, out_head;   // bytes
    int32_t heads;
  } part[3];
  const int32_t *positions;
  const int64_t *slots;
  int64_t slot_rows;
  const double *turns;                 // [rotated / 2] turns per position
  float magnitude;
  int32_t rows, dim, rotated, interleaved, inverse, dtype;
};
hipError_t launch_rotate(const RotateArgs &a, hipStream_t s);

struct GatedArgs {
  const char *x, *w_gate, *w_up;
  char *out;
  int64_t x_row, gate_row, up_row, out_row;       // bytes
  int32_t rows, width, hidden, act, fp16;
};
hipError_t launch_gated(const GatedArgs &a, hipStream_t s);

struct GatedGradArgs {
  GatedArgs f;                         // (without out)
  const char *dout;
  char *dx, *dw_gate, *dw_up;
  int64_t dout_row, dx_row, dgate_row, dup_row;   // bytes
};
// whether the products' grids are within a launch's limits
bool gated_fits(int64_t rows, int64_t width, int64_t hidden, bool grad);
size_t gated_grad_bytes(int32_t rows, int32_t width, int32_t hidden, bool fp16);
hipError_t launch_gated_grad(const GatedGradArgs &a, void *ws, hipStream_t s);

constexpr int kAdamTensors = 48;       // tensors of a launch: what its arguments hold
struct AdamTensor {
  void *param, *master, *m, *v;
  const void *grad;
  float *scales;
  int64_t count;
  int64_t begin;                       // its first wavefront's values, of those of the launch
  uint64_t first;                      // its first block of 256 values, counted through all tensors of a call
};
struct AdamStep {
  float lr_m, root, decay;             // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), lr decay
};
struct AdamArgs {
  AdamTensor t[kAdamTensors];
  int32_t n, dtype, grad_dtype;
  uint32_t key0, key1;
  int64_t step;
  const int64_t *step_dev;
  const float *lr_dev, *factor;
  double beta1, beta2, lr, eps, decay;
  AdamStep s;                          // without step_dev and lr_dev
};
hipError_t launch_adamw(const AdamArgs &a, int bits, hipStream_t s);

}  // namespace bgp
