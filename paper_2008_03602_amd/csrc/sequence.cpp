// C entry points of the sequence-block operators: argument checks and plans (host only).
// The kernels are in k_linear.hip, k_causal_conv.hip and k_scan.hip.
#include <algorithm>
#include <exception>

#include "seq_internal.h"

namespace ct {

int require_init();                       // runtime.hip: CT_OK, or CT_E_NOINIT with its message
int launch_failed(const char* what);      // runtime.hip: CT_E_HIP with the HIP error's message

namespace {

int refuse(const char* who, const char* why) {
  set_error(std::string(who) + ": " + why);
  return CT_E_ARG;
}

bool dtype_ok(int d) { return d == CT_DT_F32 || d == CT_DT_BF16; }
bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
// A row pitch: at least the row, and few enough elements that a whole array's offsets fit 64 bits.
bool pitch_ok(int64_t ld, int64_t cols) { return ld >= cols && ld <= ((int64_t)1 << 31); }

// Rows of an operand lie at most this far apart, so that a tile's offsets fit 32 bits.
constexpr int64_t kMaxPitchBytes = 4 << 20;

// A row number plus a tile of rows is still an int.
constexpr int32_t kMostRows = 0x7FFFFFFF - 4096;

int check_linear(const ct_linear_op* op) {
  const char* me = "ct_linear";
  if (!op) return refuse(me, "null op");
  if (op->m < 0 || op->n < 0 || op->k < 0) return refuse(me, "negative size");
  if (op->m > kMostRows || op->n > kMostRows) return refuse(me, "too many rows");
  if (!dtype_ok(op->dtype) || !dtype_ok(op->out_dtype)) return refuse(me, "unknown dtype");
  if (op->act < CT_ACT_NONE || op->act > CT_ACT_GELU) return refuse(me, "unknown activation");
  if (op->res < CT_RES_NONE || op->res > CT_RES_ADD_ACT) return refuse(me, "unknown residual mode");
  if (op->reserved) return refuse(me, "reserved field is not 0");
  if (!pitch_ok(op->ldx, op->k) || !pitch_ok(op->ldw, op->k) || !pitch_ok(op->ldy, op->n) ||
      (op->res && !pitch_ok(op->ldr, op->n)))
    return refuse(me, "row pitch shorter than the row");
  const int64_t e = elem_bytes(op->dtype);
  if (op->ldx * e > kMaxPitchBytes || op->ldw * e > kMaxPitchBytes)
    return refuse(me, "rows of x or w more than 4 MiB apart");
  return CT_OK;
}

int check_sequences(const char* me, const ct_sequences* s, bool states) {
  if (!s) return refuse(me, "null sequences");
  if (s->tokens < 0 || s->count < 0 || s->num_slots < 0 || s->max_len < 0) return refuse(me, "negative count");
  if (s->tokens > kMostRows || s->count > kMostRows) return refuse(me, "too many rows");
  if (!aligned(s->offsets, 4) || !aligned(s->slots, 4)) return refuse(me, "misaligned offsets or slots");
  if (!s->offsets && (s->count ? s->tokens % s->count != 0 : s->tokens != 0))
    return refuse(me, "without offsets the tokens are a multiple of the sequences");
  if (states && !s->slots && s->count > s->num_slots) return refuse(me, "more sequences than state slots");
  return CT_OK;
}

SeqView view_of(const ct_sequences& s) {
  return {s.offsets, s.slots, s.tokens, s.count, s.num_slots, !s.offsets && s.count ? s.tokens / s.count : 0};
}

int check_conv(const ct_causal_conv_op* op) {
  const char* me = "ct_causal_conv";
  if (!op) return refuse(me, "null op");
  if (op->channels < 0) return refuse(me, "negative size");
  if (op->width < 2 || op->width > 8) return refuse(me, "width outside 2..8");
  if (!dtype_ok(op->dtype)) return refuse(me, "unknown dtype");
  if (op->act != CT_ACT_NONE && op->act != CT_ACT_SILU) return refuse(me, "activation is neither none nor SiLU");
  if (!pitch_ok(op->ldx, op->channels) || !pitch_ok(op->ldy, op->channels))
    return refuse(me, "row pitch shorter than the row");
  return CT_OK;
}

int check_scan(const ct_scan_op* op) {
  const char* me = "ct_scan";
  if (!op) return refuse(me, "null op");
  if (op->channels < 0) return refuse(me, "negative size");
  if (op->states < 1 || op->states > 256) return refuse(me, "states outside 1..256");
  if (op->groups < 1 || op->channels % op->groups) return refuse(me, "groups do not divide the channels");
  if (!dtype_ok(op->dtype)) return refuse(me, "unknown dtype");
  if ((op->softplus != 0 && op->softplus != 1) || op->reserved) return refuse(me, "unknown flag");
  const int64_t gn = (int64_t)op->groups * op->states;
  if (!pitch_ok(op->ldu, op->channels) || !pitch_ok(op->lddelta, op->channels) || !pitch_ok(op->ldb, gn) ||
      !pitch_ok(op->ldc, gn) || !pitch_ok(op->ldy, op->channels))
    return refuse(me, "row pitch shorter than the row");
  const int64_t e = elem_bytes(op->dtype);
  if (op->ldu * e > kMaxPitchBytes || op->lddelta * e > kMaxPitchBytes || op->ldy * e > kMaxPitchBytes)
    return refuse(me, "rows of u, delta or y more than 4 MiB apart");
  return CT_OK;
}

int check_workspace(const char* me, const void* ws, int64_t have, int64_t floats) {
  if (!floats) return CT_OK;
  if (!ws || have < floats * (int64_t)sizeof(float)) return refuse(me, "workspace is too small");
  if (!aligned(ws, 16)) return refuse(me, "workspace is not 16-byte aligned");
  return CT_OK;
}

int launched(const char* me, int rc) { return rc == 0 ? CT_OK : rc == -2 ? CT_E_ARG : launch_failed(me); }

// Nothing thrown (an allocation of an error's text, say) leaves an entry point.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::exception&) {
    return CT_E_OOM;
  }
}

}  // namespace
}  // namespace ct

using namespace ct;

extern "C" {

int ct_linear_workspace(const ct_linear_op* op, int64_t* bytes) {
  return guarded([&]() -> int {
    if (const int rc = check_linear(op)) return rc;
    if (!bytes) return refuse("ct_linear_workspace", "null bytes");
    *bytes = op->m && op->n ? plan_linear(*op).ws_floats * (int64_t)sizeof(float) : 0;
    return CT_OK;
  });
}

int ct_linear_run(const ct_linear_op* op, const void* x, const void* w, const float* bias, const void* res,
                  void* y, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_linear_run";
    if (const int rc = check_linear(op)) return rc;
    if (!op->m || !op->n) return CT_OK;
    if ((op->k && (!x || !w)) || !y || (op->res && !res)) return refuse(me, "null array");
    const int e = elem_bytes(op->dtype), o = elem_bytes(op->out_dtype);
    if (!aligned(x, e) || !aligned(w, e) || !aligned(bias, 4) || !aligned(y, o) || (op->res && !aligned(res, o)))
      return refuse(me, "array not aligned to its element");
    const LinearPlan p = plan_linear(*op);
    if (const int rc = check_workspace(me, ws, ws_bytes, p.ws_floats)) return rc;
    if (const int rc = require_init()) return rc;
    return launched(me, launch_linear(*op, p, x, w, bias, res, y, (float*)ws, stream));
  });
}

int ct_causal_conv_run(const ct_causal_conv_op* op, const ct_sequences* seqs, const void* x, const float* w,
                       const float* bias, const void* state_in, void* state_out, void* y, void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_causal_conv_run";
    if (const int rc = check_conv(op)) return rc;
    if (const int rc = check_sequences(me, seqs, state_in || state_out)) return rc;
    if (!op->channels || !seqs->count) return CT_OK;
    if (!w || (seqs->tokens && (!x || !y))) return refuse(me, "null array");
    const int e = elem_bytes(op->dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(state_in, e) || !aligned(state_out, e) || !aligned(w, 4) ||
        !aligned(bias, 4))
      return refuse(me, "array not aligned to its element");
    if (const int rc = require_init()) return rc;
    return launched(me, launch_causal_conv(*op, view_of(*seqs), x, w, bias, state_in, state_out, y, stream));
  });
}

int ct_scan_workspace(const ct_scan_op* op, const ct_sequences* seqs, int64_t* bytes) {
  return guarded([&]() -> int {
    if (const int rc = check_scan(op)) return rc;
    if (const int rc = check_sequences("ct_scan_workspace", seqs, false)) return rc;
    if (!bytes) return refuse("ct_scan_workspace", "null bytes");
    *bytes = op->channels && seqs->count ? plan_scan(*op, *seqs).ws_floats * (int64_t)sizeof(float) : 0;
    return CT_OK;
  });
}

int ct_scan_run(const ct_scan_op* op, const ct_sequences* seqs, const void* u, const void* delta,
                const float* dt_bias, const float* a, const void* b, const void* c, const float* d_skip,
                const void* z, const float* state_in, float* state_out, void* y, void* ws, int64_t ws_bytes,
                void* stream) {
  return guarded([&]() -> int {
    const char* me = "ct_scan_run";
    if (const int rc = check_scan(op)) return rc;
    if (z && !pitch_ok(op->ldz, op->channels)) return refuse(me, "row pitch shorter than the row");
    if (z && op->ldz * elem_bytes(op->dtype) > kMaxPitchBytes) return refuse(me, "rows of z more than 4 MiB apart");
    if (const int rc = check_sequences(me, seqs, state_in || state_out)) return rc;
    if (!op->channels || !seqs->count) return CT_OK;
    if (!a || (seqs->tokens && (!u || !delta || !b || !c || !y))) return refuse(me, "null array");
    const int e = elem_bytes(op->dtype);
    for (const void* p : {u, delta, b, c, z, (const void*)y})
      if (!aligned(p, e)) return refuse(me, "array not aligned to its element");
    for (const float* p : {dt_bias, a, d_skip, state_in, (const float*)state_out})
      if (!aligned(p, 4)) return refuse(me, "array not aligned to its element");
    const ScanPlan p = plan_scan(*op, *seqs);
    if (const int rc = check_workspace(me, ws, ws_bytes, p.ws_floats)) return rc;
    if (const int rc = require_init()) return rc;
    const ScanArrays v = {u, delta, b, c, z, dt_bias, a, d_skip, state_in, state_out, y, (float*)ws};
    return launched(me, launch_scan(*op, p, view_of(*seqs), v, stream));
  });
}

}  // extern "C"
