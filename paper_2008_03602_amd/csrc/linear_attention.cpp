// C entry points of the linear-attention-block operators: argument checks and plans (host only).
// The kernels are in k_norm.hip, k_mx.hip, k_mx_linear.hip and k_decay_attention.hip.
#include "seq_checks.h"

namespace ct {

namespace {

bool format_ok(int f) { return f == CT_MX_E4M3 || f == CT_MX_E2M1; }
int64_t mx_row_bytes(int cols, int format) {
  return ((int64_t)cols + 31) / 32 * (format == CT_MX_E4M3 ? 32 : 16);
}
int64_t mx_scale_bytes(int cols) { return ((int64_t)cols + 127) / 128 * 4; }

// Pitches of microscaled rows; nullptr, or what is wrong with them.
const char* mx_pitches(int cols, int format, int64_t ldq, int64_t lds) {
  if (!pitch_ok(ldq, mx_row_bytes(cols, format)) || !pitch_ok(lds, mx_scale_bytes(cols)))
    return "row pitch shorter than the row";
  if (ldq % 16 || lds % 4) return "pitch of microscaled rows is not a multiple of 16 bytes, of their scales 4";
  return nullptr;
}
const char* mx_addresses(const void* q, const void* scales) {
  if (!q || !scales) return "null array";
  if (!aligned(q, 16) || !aligned(scales, 4)) return "microscaled rows not aligned to 16 bytes, or their scales to 4";
  return nullptr;
}

int check_mx(const char* me, const ct_mx_op* op) {
  if (!op) return refuse(me, "null op");
  if (op->rows < 0 || op->cols < 0) return refuse(me, "negative size");
  if (op->rows > kMostRows || op->cols > kMostRows) return refuse(me, "too many rows or columns");
  if (!dtype_ok(op->dtype)) return refuse(me, "unknown dtype");
  if (!format_ok(op->format)) return refuse(me, "unknown format");
  if (!pitch_ok(op->ldx, op->cols)) return refuse(me, "row pitch shorter than the row");
  if (const char* why = mx_pitches(op->cols, op->format, op->ldq, op->lds)) return refuse(me, why);
  return CT_OK;
}

int run_mx(const char* me, const ct_mx_op* op, void* x, void* q, void* scales, bool values, void* stream) {
  if (const int rc = check_mx(me, op)) return rc;
  if (!op->rows || !op->cols) return CT_OK;
  if (!x) return refuse(me, "null array");
  if (!aligned(x, elem_bytes(op->dtype))) return refuse(me, "array not aligned to its element");
  if (const char* why = mx_addresses(q, scales)) return refuse(me, why);
  if (const int rc = require_init()) return rc;
  return launched(me, launch_mx(*op, x, q, scales, values, stream));
}

int check_mx_linear(const ct_mx_linear_op* op) {
  const char* me = "ct_mx_linear";
  if (!op) return refuse(me, "null op");
  if (op->m < 0 || op->n < 0 || op->k < 0) return refuse(me, "negative size");
  if (op->m > kMostRows || op->n > kMostRows || op->k > kMostRows) return refuse(me, "too many rows or columns");
  if (!format_ok(op->x_format) || !format_ok(op->w_format)) return refuse(me, "unknown format");
  if (!dtype_ok(op->out_dtype)) return refuse(me, "unknown dtype");
  if (op->act < CT_ACT_NONE || op->act > CT_ACT_GELU) return refuse(me, "unknown activation");
  if (op->res < CT_RES_NONE || op->res > CT_RES_ADD_ACT) return refuse(me, "unknown residual mode");
  if (const char* why = mx_pitches(op->k, op->x_format, op->ldx, op->ldxs)) return refuse(me, why);
  if (const char* why = mx_pitches(op->k, op->w_format, op->ldw, op->ldws)) return refuse(me, why);
  if (!pitch_ok(op->ldy, op->n) || (op->res && !pitch_ok(op->ldr, op->n)))
    return refuse(me, "row pitch shorter than the row");
  if (op->ldx > kMaxPitchBytes || op->ldw > kMaxPitchBytes || op->ldxs > kMaxPitchBytes || op->ldws > kMaxPitchBytes)
    return refuse(me, "rows of x or w more than 4 MiB apart");
  return CT_OK;
}

int check_norm(const ct_norm_op* op) {
  const char* me = "ct_norm";
  if (!op) return refuse(me, "null op");
  if (op->rows < 0 || op->cols < 0) return refuse(me, "negative size");
  if (op->rows > kMostRows || op->cols > kMostRows) return refuse(me, "too many rows or columns");
  if (op->groups < 1 || op->cols % op->groups) return refuse(me, "groups do not divide the columns");
  if (!dtype_ok(op->dtype)) return refuse(me, "unknown dtype");
  if (!dtype_ok(op->out) && !format_ok(op->out)) return refuse(me, "unknown output type");
  if (!(op->eps >= 0.f)) return refuse(me, "eps is negative or NaN");
  if (!pitch_ok(op->ldx, op->cols)) return refuse(me, "row pitch shorter than the row");
  if (format_ok(op->out)) {
    if (op->groups > 1 && op->cols / op->groups % 32) return refuse(me, "parts of microscaled rows are not whole blocks");
    if (const char* why = mx_pitches(op->cols, op->out, op->ldy, op->lds)) return refuse(me, why);
  } else if (!pitch_ok(op->ldy, op->cols)) {
    return refuse(me, "row pitch shorter than the row");
  }
  return CT_OK;
}

int check_decay(const ct_decay_attention_op* op) {
  const char* me = "ct_decay_attention";
  if (!op) return refuse(me, "null op");
  if (op->heads < 0) return refuse(me, "negative size");
  if (op->groups < 1 || op->heads % op->groups) return refuse(me, "groups do not divide the heads");
  if (op->key_dim < 1 || op->key_dim > 256 || op->value_dim < 1 || op->value_dim > 256)
    return refuse(me, "key or value dimension outside 1..256");
  if (!dtype_ok(op->dtype) || !dtype_ok(op->delta_dtype)) return refuse(me, "unknown dtype");
  if ((op->softplus != 0 && op->softplus != 1) || (op->step_input != 0 && op->step_input != 1) || op->reserved)
    return refuse(me, "unknown flag");
  const int64_t gk = (int64_t)op->groups * op->key_dim, hv = (int64_t)op->heads * op->value_dim;
  if (!pitch_ok(op->ldq, gk) || !pitch_ok(op->ldk, gk) || !pitch_ok(op->ldv, hv) || !pitch_ok(op->ldo, hv))
    return refuse(me, "row pitch shorter than the row");
  const int64_t e = elem_bytes(op->dtype);
  if (op->ldq * e > kMaxPitchBytes || op->ldk * e > kMaxPitchBytes || op->ldv * e > kMaxPitchBytes ||
      op->ldo * e > kMaxPitchBytes)
    return refuse(me, "rows of q, k, v or o more than 4 MiB apart");
  return CT_OK;
}

}  // namespace
}  // namespace ct

using namespace ct;

extern "C" {

int ct_mx_quantise_run(const ct_mx_op* op, const void* x, void* q, void* scales, void* stream) {
  return guarded([&] { return run_mx("ct_mx_quantise_run", op, const_cast<void*>(x), q, scales, false, stream); });
}

int ct_mx_values_run(const ct_mx_op* op, const void* q, const void* scales, void* x, void* stream) {
  return guarded([&] {
    return run_mx("ct_mx_values_run", op, x, const_cast<void*>(q), const_cast<void*>(scales), true, stream);
  });
}

int ct_mx_linear_workspace(const ct_mx_linear_op* op, int64_t* bytes) {
  return guarded([&]() -> int {
    if (const int rc = check_mx_linear(op)) return rc;
    if (!bytes) return refuse("ct_mx_linear_workspace", "null bytes");
    *bytes = op->m && op->n ? plan_mx_linear(*op).ws_floats * (int64_t)sizeof(float) : 0;
    return CT_OK;
  });
}

int ct_mx_linear_run(const ct_mx_linear_op* op, const void* x, const void* x_scales, const void* w,
                     const void* w_scales, const float* bias, const void* res, void* y, void* ws, int64_t ws_bytes,
                     void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_mx_linear_run";
    if (const int rc = check_mx_linear(op)) return rc;
    if (!op->m || !op->n) return CT_OK;
    if (!y || (op->res && !res)) return refuse(me, "null array");
    if (op->k) {
      if (const char* why = mx_addresses(x, x_scales)) return refuse(me, why);
      if (const char* why = mx_addresses(w, w_scales)) return refuse(me, why);
    }
    const int o = elem_bytes(op->out_dtype);
    if (!aligned(bias, 4) || !aligned(y, o) || (op->res && !aligned(res, o)))
      return refuse(me, "array not aligned to its element");
    const MxLinearPlan p = plan_mx_linear(*op);
    if (const int rc = check_workspace(me, ws, ws_bytes, p.ws_floats)) return rc;
    if (const int rc = require_init()) return rc;
    const MxLinearArrays v = {x, x_scales, w, w_scales, bias, res, y, (float*)ws};
    return launched(me, launch_mx_linear(*op, p, v, stream));
  });
}

int ct_norm_run(const ct_norm_op* op, const void* x, const void* res, void* sum, const float* w, const void* z,
                void* y, void* scales, void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_norm_run";
    if (const int rc = check_norm(op)) return rc;
    if ((res && !pitch_ok(op->ldres, op->cols)) || (sum && !pitch_ok(op->ldsum, op->cols)) ||
        (z && !pitch_ok(op->ldz, op->cols)))
      return refuse(me, "row pitch shorter than the row");
    if (!op->rows || !op->cols) return CT_OK;
    if (!x || !y) return refuse(me, "null array");
    const int e = elem_bytes(op->dtype);
    for (const void* p : {x, res, (const void*)sum, z})
      if (!aligned(p, e)) return refuse(me, "array not aligned to its element");
    if (!aligned(w, 4) || (dtype_ok(op->out) && !aligned(y, elem_bytes(op->out))))
      return refuse(me, "array not aligned to its element");
    if (format_ok(op->out))
      if (const char* why = mx_addresses(y, scales)) return refuse(me, why);
    if (const int rc = require_init()) return rc;
    return launched(me, launch_norm(*op, x, res, sum, w, z, y, scales, stream));
  });
}

int ct_decay_attention_workspace(const ct_decay_attention_op* op, const ct_sequences* seqs, int64_t* bytes) {
  return guarded([&]() -> int {
    if (const int rc = check_decay(op)) return rc;
    if (const int rc = check_sequences("ct_decay_attention_workspace", seqs, false)) return rc;
    if (!bytes) return refuse("ct_decay_attention_workspace", "null bytes");
    *bytes = op->heads && seqs->count ? plan_decay(*op, *seqs).ws_floats * (int64_t)sizeof(float) : 0;
    return CT_OK;
  });
}

int ct_decay_attention_run(const ct_decay_attention_op* op, const ct_sequences* seqs, const void* q, const void* k,
                           const void* v, const void* delta, const float* dt_bias, const float* a,
                           const float* state_in, float* state_out, void* o, void* ws, int64_t ws_bytes,
                           void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_decay_attention_run";
    if (const int rc = check_decay(op)) return rc;
    if (delta && !pitch_ok(op->lddelta, op->heads)) return refuse(me, "row pitch shorter than the row");
    if (const int rc = check_sequences(me, seqs, state_in || state_out)) return rc;
    if (dt_bias && !delta && seqs->tokens) return refuse(me, "dt_bias without delta");
    if (!op->heads || !seqs->count) return CT_OK;
    if (!a || (seqs->tokens && (!q || !k || !v || !o))) return refuse(me, "null array");
    const int e = elem_bytes(op->dtype);
    for (const void* p : {q, k, v, (const void*)o})
      if (!aligned(p, e)) return refuse(me, "array not aligned to its element");
    if (!aligned(delta, elem_bytes(op->delta_dtype))) return refuse(me, "array not aligned to its element");
    for (const float* p : {dt_bias, a, state_in, (const float*)state_out})
      if (!aligned(p, 4)) return refuse(me, "array not aligned to its element");
    const DecayPlan p = plan_decay(*op, *seqs);
    if (const int rc = check_workspace(me, ws, ws_bytes, p.ws_floats)) return rc;
    if (const int rc = require_init()) return rc;
    const DecayArrays arrays = {q, k, v, delta, dt_bias, a, state_in, state_out, o, (float*)ws};
    return launched(me, launch_decay(*op, p, view_of(*seqs), arrays, stream));
  });
}

}  // extern "C"
