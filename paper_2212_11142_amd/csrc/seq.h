// Internal declarations of the sequence-surrogate operators (attention over packed
// histories and log probabilities): kernels in attend.hip, attend_few.hip, attend_grad.hip
// and logprob.hip, their C-ABI in seq_abi.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>
#include <string>

#include "baco_gp.h"
#include "lds_limit.h"

namespace bgp {

constexpr int kSeqMaxDim = 128;       // head size
constexpr int kSeqCus = 256;          // compute units of an MI355X: what splits are sized for
constexpr int kMaxBuckets = 64;       // buckets of one side
constexpr int kMaxReach = 1024;       // first distance of the last bucket
constexpr int kMaxTop = 128;          // alternatives of a row
constexpr int kLdsBytes = 160 * 1024; // of a compute unit
// Blocks of 256 threads of a launch, at most: it has fewer than 2^32 threads.
constexpr int64_t kMaxBlocks = (1 << 24) - 1;

// First distance of each bucket of a side (start[0] = 0, ascending; INT32_MAX past the last).
struct BucketMap {
  int32_t per_side;
  int32_t two_sided;
  int32_t start[kMaxBuckets];
};

struct AttnArgs {
  const char *q, *k, *v;
  char *o;
  char *rest;                          // what rounding took from o (null: not kept)
  float *lse;                          // [heads][q_rows]
  // strides in bytes
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, rest_row, rest_head;
  const int32_t *qb, *qe, *kb, *ke, *prefix;
  int32_t docs, heads, kv_heads, group, bytes;  // bytes: of a head's row, 2 dim
  int32_t q_rows, k_rows, max_q, max_k;
  int32_t causal;
  float scale, cap;
  const float *slopes;                 // [heads]
  const void *table;                   // [heads][buckets]
  BucketMap buckets;
  int32_t fp16;
};

// Gradient: q, k, v, o, rest, lse as of the forward call.
struct AttnGradArgs {
  AttnArgs f;
  const char *dout;
  char *dq, *dk, *dv;
  void *dtable;                        // [heads][buckets] or null
  int64_t do_row, do_head, dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
  // workspace
  float *rows;                         // [heads][q_rows][2] log-sum, dout . out
  float *bound;                        // fp16: largest |dout|^2 and |v|^2 of every 16 rows
  float *tpart;                        // [tiles][heads][buckets] partial table gradients
  float *kv_part;                      // [shares][k_rows][kv_heads][dK, dV], with shares
  int32_t shares;                      // blocks of a key tile
};

// attend_fits and the like: whether a description's grids are within a launch's limits
bool attend_fits(const AttnArgs &a);
hipError_t launch_attend(const AttnArgs &a, hipStream_t s);
// few query rows: key ranges split over blocks; part: attend_few_bytes() of workspace
size_t attend_few_bytes(const AttnArgs &a);
bool attend_use_few(const AttnArgs &a);
bool attend_few_fits(const AttnArgs &a);
hipError_t launch_attend_few(const AttnArgs &a, void *part, hipStream_t s);

size_t attend_grad_bytes(const AttnArgs &f);
bool attend_grad_fits(const AttnArgs &f);
hipError_t launch_attend_grad(const AttnGradArgs &a, void *ws, hipStream_t s);

struct LogprobArgs {
  const void *x;
  int64_t row;                         // row stride in elements
  int32_t rows, width, top, dtype;
  float scale;
  const int64_t *target;
  float *logp, *entropy, *lse, *top_logp;
  float *norm;                         // [rows][2] the maximum m, log sum e^(scale (x - m))
  int64_t *top_id;
  const float *g_logp, *g_entropy;     // gradient
  void *dx;
  int64_t dx_row;
};
size_t logprob_bytes(int32_t rows, int32_t width, int32_t top);
hipError_t launch_logprob(const LogprobArgs &a, void *ws, hipStream_t s);
hipError_t launch_logprob_grad(const LogprobArgs &a, hipStream_t s);

// abi.hip: records the calling thread's error message
gp_status seq_fail(gp_status st, const std::string &msg);

}  // namespace bgp
