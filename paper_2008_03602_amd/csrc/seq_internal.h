// Internal declarations of the sequence- and linear-attention-block operators (ct_linear,
// ct_causal_conv, ct_scan, ct_norm, ct_mx, ct_decay_attention): the plans that the workspace functions and the launchers both take, so that a
// call is launched as its workspace was sized.
#pragma once

#include <cstdint>
#include <string>

#include "convtune.h"

namespace ct {

void set_error(const std::string& msg);  // the calling thread's ct_last_error

// Compute units that the choices of tiles and splits count on. Not the calling stream's
// share: a plan has to be the same wherever a call goes, and a share of them only takes
// more passes over the same blocks.
constexpr int kPlanCus = 256;

constexpr int elem_bytes(int dtype) { return dtype == CT_DT_BF16 ? 2 : 4; }

// The rows of one call's sequences, as the kernels see them.
struct SeqView {
  const int32_t* offsets;
  const int32_t* slots;
  int tokens, count, num_slots, len;  // len: rows of each sequence where offsets is null
};

// ---- ct_linear ----
struct LinearPlan {
  int kind;           // the kernel (k_linear.hip)
  int split;          // slices of the reduction, each with partial sums of its own
  int per_split;      // elements of a row in a slice
  int64_t ws_floats;  // split * m * n where the reduction is split
};
LinearPlan plan_linear(const ct_linear_op& op);
// Launchers return 0, -1 on a launch error (reason in hipGetLastError), or -2 when a size
// is refused (reason given to set_error).
int launch_linear(const ct_linear_op& op, const LinearPlan& p, const void* x, const void* w, const float* bias,
                  const void* res, void* y, float* ws, void* stream);

// ---- ct_causal_conv ----
int launch_causal_conv(const ct_causal_conv_op& op, const SeqView& s, const void* x, const float* w,
                       const float* bias, const void* state_in, void* state_out, void* y, void* stream);

// ---- ct_scan ----
struct ScanPlan {
  bool narrow;        // a prompt's lanes have four states, not 16
  int chunk;          // tokens per chunk (0: every sequence in one piece)
  int64_t chunks;     // chunks in all, an upper bound
  int64_t ws_floats;
  bool fold;          // the outputs of a chunk fold those before it themselves
};
ScanPlan plan_scan(const ct_scan_op& op, const ct_sequences& s);
struct ScanArrays {
  const void *u, *delta, *b, *c, *z;
  const float *dt_bias, *a, *d_skip, *state_in;
  float* state_out;
  void* y;
  float* ws;
};
int launch_scan(const ct_scan_op& op, const ScanPlan& p, const SeqView& s, const ScanArrays& v, void* stream);

// ---- ct_norm, ct_mx ----
int launch_norm(const ct_norm_op& op, const void* x, const void* res, void* sum, const float* w, const void* z, void* y,
                void* scales, void* stream);
// x to q and scales, or with `values` back.
int launch_mx(const ct_mx_op& op, void* x, void* q, void* scales, bool values, void* stream);

// ---- ct_mx_linear ----
struct MxLinearPlan {
  int kind;           // the kernel (k_mx_linear.hip)
  int split;          // slices of the reduction, each with partial sums of its own
  int per_split;      // steps of 128 elements in a slice
  int tail_m, tail_n; // last rows and columns of y that a launch of their own computes
  int64_t ws_floats;  // split * m * n where the reduction is split
};
MxLinearPlan plan_mx_linear(const ct_mx_linear_op& op);
struct MxLinearArrays {
  const void *x, *xs, *w, *ws;
  const float* bias;
  const void* res;
  void* y;
  float* scratch;
};
int launch_mx_linear(const ct_mx_linear_op& op, const MxLinearPlan& p, const MxLinearArrays& v, void* stream);

// ---- ct_decay_attention ----
struct DecayPlan {
  bool step;          // token by token
  int piece;          // tokens of a piece (0: every sequence in one)
  int64_t pieces;     // pieces in all, an upper bound
  int64_t ws_floats;
};
DecayPlan plan_decay(const ct_decay_attention_op& op, const ct_sequences& s);
struct DecayArrays {
  const void *q, *k, *v, *delta;
  const float *dt_bias, *a, *state_in;
  float* state_out;
  void* o;
  float* ws;
};
int launch_decay(const ct_decay_attention_op& op, const DecayPlan& p, const SeqView& s, const DecayArrays& v,
                 void* stream);

}  // namespace ct
