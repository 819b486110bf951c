// Argument checks that the entry points of the sequence and block operators share (host only).
#pragma once

#include <exception>

#include "seq_internal.h"

namespace ct {

int require_init();                       // runtime.hip: CT_OK, or CT_E_NOINIT with its message
int launch_failed(const char* what);      // runtime.hip: CT_E_HIP with the HIP error's message

inline int refuse(const char* who, const char* why) {
  set_error(std::string(who) + ": " + why);
  return CT_E_ARG;
}

inline bool dtype_ok(int d) { return d == CT_DT_F32 || d == CT_DT_BF16; }
inline bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
// A row pitch: at least the row, and few enough elements that a whole array's offsets fit 64 bits.
inline bool pitch_ok(int64_t ld, int64_t cols) { return ld >= cols && ld <= ((int64_t)1 << 31); }

// Rows of an operand lie at most this far apart, so that a tile's offsets fit 32 bits.
constexpr int64_t kMaxPitchBytes = 4 << 20;

// A row number plus a tile of rows is still an int.
constexpr int32_t kMostRows = 0x7FFFFFFF - 4096;

inline int check_sequences(const char* me, const ct_sequences* s, bool states) {
  if (!s) return refuse(me, "null sequences");
  if (s->tokens < 0 || s->count < 0 || s->num_slots < 0 || s->max_len < 0) return refuse(me, "negative count");
  if (s->tokens > kMostRows || s->count > kMostRows) return refuse(me, "too many rows");
  if (!aligned(s->offsets, 4) || !aligned(s->slots, 4)) return refuse(me, "misaligned offsets or slots");
  if (!s->offsets && (s->count ? s->tokens % s->count != 0 : s->tokens != 0))
    return refuse(me, "without offsets the tokens are a multiple of the sequences");
  if (states && !s->slots && s->count > s->num_slots) return refuse(me, "more sequences than state slots");
  return CT_OK;
}

inline SeqView view_of(const ct_sequences& s) {
  return {s.offsets, s.slots, s.tokens, s.count, s.num_slots, !s.offsets && s.count ? s.tokens / s.count : 0};
}

inline int check_workspace(const char* me, const void* ws, int64_t have, int64_t floats) {
  if (!floats) return CT_OK;
  if (!ws || have < floats * (int64_t)sizeof(float)) return refuse(me, "workspace is too small");
  if (!aligned(ws, 16)) return refuse(me, "workspace is not 16-byte aligned");
  return CT_OK;
}

inline int launched(const char* me, int rc) { return rc == 0 ? CT_OK : rc == -2 ? CT_E_ARG : launch_failed(me); }

// Nothing thrown (an allocation of an error's text, say) leaves an entry point.
template <class F>
inline int guarded(F f) {
  try {
    return f();
  } catch (const std::exception&) {
    return CT_E_OOM;
  }
}

}  // namespace ct
