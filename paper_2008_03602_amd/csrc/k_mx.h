// Microscaled rows: blocks of 32 elements of 8 or 4 bits with a power of two as their scale.
// Four neighbouring lanes hold a block, eight values each.
#pragma once
#include "k_seq.h"

namespace ct {

constexpr int kMxBlock = 32;
constexpr int mx_blocks(int cols) { return cols / kMxBlock + (cols % kMxBlock != 0); }
// Scale bytes of a row: whole groups of four.
constexpr int mx_scales(int cols) { return (mx_blocks(cols) + 3) / 4 * 4; }

// ---- eight elements of a row ----
struct Oct {
  float v[8];
};
// Eight elements as they lie in memory, at any element's address: asked for early, looked at late.
template <typename T>
struct RawOct {
  u32x4 q[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(T) == 2) {
      q[0] = *(const u32x4_any*)p;
    } else {
      q[0] = __builtin_bit_cast(u32x4, *(const f32x4_any*)p);
      q[1] = __builtin_bit_cast(u32x4, *(const f32x4_any*)(p + 4));
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2) {
      const unsigned w = q[0][i / 2];
      return unpack<T>(w, i & 1);
    } else {
      const unsigned w = q[i / 4][i % 4];
      return __builtin_bit_cast(float, w);
    }
  }
  // The first `left` elements (1..7), 0 for the others.
  __device__ __forceinline__ void load_some(const T* p, int left) {
#pragma unroll
    for (int i = 0; i < 8 * (int)sizeof(T) / 16; ++i) q[i] = u32x4{};
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (i >= left) break;
      const float f = (float)p[i];
      if constexpr (sizeof(T) == 2) q[0][i / 2] |= (__builtin_bit_cast(unsigned, f) >> 16) << (16 * (i & 1));
      else q[i / 4][i % 4] = __builtin_bit_cast(unsigned, f);
    }
  }
};
template <typename T>
__device__ __forceinline__ void load_oct(RawOct<T>& r, const T* p, int left) {
  if (left >= 8) r.load(p);
  else r.load_some(p, left);
}
// The first `left` of eight outputs.
template <typename O>
__device__ __forceinline__ void store_oct(O* p, const float* v, int left) {
  if (left >= 8) {
    if constexpr (sizeof(O) == 2) {
      *(u32x4_any*)p = (u32x4){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
      *(f32x4_any*)p = (f32x4){v[0], v[1], v[2], v[3]};
      *(f32x4_any*)(p + 4) = (f32x4){v[4], v[5], v[6], v[7]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < left) p[i] = (O)v[i];
}

// ---- a block of four lanes ----
template <int CTRL>
__device__ __forceinline__ unsigned quad_perm(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
// The block's largest magnitude from each lane's eight values, as its bits, in whose order infinities
// and NaN come last and the exponent is on top.
__device__ __forceinline__ unsigned mx_largest(const float* v) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
  m = max(m, quad_perm<0xB1>(m));  // lanes 1 0 3 2
  return max(m, quad_perm<0x4E>(m));  // lanes 2 3 0 1
}
// The scale byte of a block by its largest magnitude: the exponent's bits are floor(log2 m) + 127 of a
// normal m, 0 of the others, whose scale is the least one anyway.
template <int FORMAT>
__device__ __forceinline__ unsigned mx_scale(unsigned largest) {
  const int e = (int)(largest >> 23);
  return e == 255 ? 255u : (unsigned)max(e - (FORMAT == CT_MX_E4M3 ? 8 : 2), 0);
}
// 1 / 2^(s - 127), a normal number for every s that mx_scale gives (246 at most); of s = 255
// nothing that is read.
__device__ __forceinline__ float mx_inverse(unsigned s) { return __builtin_bit_cast(float, (254u - min(s, 253u)) << 23); }
// 2^(s - 127); 2^-127 is not a normal number, and 255 is NaN.
__device__ __forceinline__ float mx_scale_value(unsigned s) {
  return __builtin_bit_cast(float, s == 255 ? 0x7FC00000u : s == 0 ? 0x00400000u : s << 23);
}
// Eight elements of a lane: two words of e4m3, or one of e2m1. Values over the scale (times `inv`, of
// mx_inverse), which is exact; the conversion rounds to nearest even. It saturates e2m1, and e4m3 past
// 464 would be NaN, so those are held at 448 before it.
template <int FORMAT>
__device__ __forceinline__ u32x2 mx_elements(const float* v, float inv) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = v[i] * inv;
  if constexpr (FORMAT == CT_MX_E4M3) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    unsigned w[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __builtin_amdgcn_fmed3f(t[i], -448.f, 448.f);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i16x2 p = {0, 0};
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, t[4 * h], t[4 * h + 1], 1.f, false);
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, t[4 * h + 2], t[4 * h + 3], 1.f, true);
      w[h] = __builtin_bit_cast(unsigned, p);
    }
    return (u32x2){w[0], w[1]};
  } else {
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[0], t[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[2], t[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[4], t[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[6], t[7], 1.f, 3);
    return (u32x2){w, 0};
  }
}
// A lane's elements from column `col` on (a multiple of 8) of a row of `cols`, and their block's scale,
// to the row.
template <int FORMAT>
__device__ __forceinline__ void mx_write(u32x2 w, unsigned scale, char* q, unsigned char* scales, unsigned col, int cols) {
  if constexpr (FORMAT == CT_MX_E4M3) *(u32x2*)(q + col) = w;
  else *(unsigned*)(q + col / 2) = w.x;
  if (col % kMxBlock == 0) {
    const unsigned block = col / kMxBlock, blocks = (unsigned)mx_blocks(cols);
    scales[block] = (unsigned char)scale;
    if (block == blocks - 1)
      for (int b = (int)blocks; b < mx_scales(cols); ++b) scales[b] = 0;
  }
}

}  // namespace ct
