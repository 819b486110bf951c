// Product of microscaled rows with its epilogue: y = act(x w^T + bias) + r, or act(x w^T + bias + r),
// x and w of e4m3 or e2m1 elements in blocks of 32 with a power of two as their scale.
//
// The matrix instruction takes 128 elements of a row, a lane's 32 of them and the scale of one
// block: of e2m1 lane group g holds elements 32 g to 32 g + 31, of e4m3 16 g to 16 g + 15 and the
// same 64 further on, and either way its scale is the one of block g. Fragments and scales are
// read from LDS as they lie in memory. The weights are the first operand: a lane's four
// consecutive accumulators are then four consecutive outputs of one row of y.
//
// Sums. Of each eight consecutive products the instruction drops what lies below 2^-13 of the
// largest (measured: 2^-13 of it survives beside it and 2^-14 does not, across eights all 23 bits
// do), 1.5e-5 of the result for two operands of normal values in e4m3, which an output of bf16
// (2^-9) does not show. For fp32 outputs the elements are turned into bf16, which holds each with
// its scale exactly while both are of normal size, and multiplied by the 16-bit instruction: products
// exact, sums in fp32. A wave that meets a block whose scale would leave bf16 (bytes below 10 or above 246
// of e4m3, 2 and 252 of e2m1, in a block that is not all 0) sums its part of the tile again, of elements
// without their scales, and scales each block's sum: the other operand's scale may bring it back. Rows
// without such a block keep the sums that they had.
//
// Measured, 8-bit x by 4-bit w: 8192 x 4096 by 8192 with SiLU 236-275 us by the card (2.0-2.3 PFLOP/s). Its
// matrix cores are busy 52 % of its clocks, at 1.9 GHz: 65 % of a step's, and 23 thousand clocks of each
// tile's 124 are its first copies and its epilogue, when none is (with 2048 elements 142-165 us). 24 x 8192
// by 4096 9.5 us, 1.9 TB/s, bound by the latency of a wave's eight steps; 1021 x 515 by 1277 of 4 bits to
// fp32 11 us.
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "k_linear.h"
#include "k_mx.h"
#include "mx_linear_plan.h"

namespace ct {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MxLinearArgs : OutArgs {
  const char *x, *w;
  const unsigned char *xs, *wsc;
  int blocks;     // of a row
  int per_split;  // steps of 128 elements in a slice of the reduction
  int64_t ldx, ldxs, ldw, ldws;
};

constexpr int mx_step_bytes(int format) { return format == CT_MX_E4M3 ? 128 : 64; }  // of 128 elements

// A lane's 32 elements of a row.
template <int FORMAT>
struct MxFrag {
  u32x4 lo, hi;  // e2m1: hi is not used
};
// Eight elements, of one word (e2m1) or two, with their scale in bf16.
template <int FORMAT>
__device__ __forceinline__ bf16x8 mx_eight(unsigned w0, unsigned w1, unsigned scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float s = __builtin_bit_cast(float, scale << 23);  // the conversion takes the exponent's bits as they are
  bf16x2 p[4];
  if constexpr (FORMAT == CT_MX_E4M3) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 3);
  }
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = p[i].x;
    r[2 * i + 1] = p[i].y;
  }
  return r;
}
// Eight of a lane's 32 elements, number c of them, with their scale.
template <int FORMAT>
__device__ __forceinline__ bf16x8 mx_bf16(const MxFrag<FORMAT>& f, int c, unsigned scale) {
  if constexpr (FORMAT == CT_MX_E4M3) {
    const u32x4 q = c < 2 ? f.lo : f.hi;
    return mx_eight<FORMAT>(q[c % 2 * 2], q[c % 2 * 2 + 1], scale);
  } else {
    return mx_eight<FORMAT>(f.lo[c], 0, scale);
  }
}
// Eight elements as they lie at byte `off` of rows.
template <int FORMAT>
__device__ __forceinline__ u32x2 mx_raw(__amdgpu_buffer_rsrc_t rows, unsigned off) {
  if constexpr (FORMAT == CT_MX_E4M3)
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, (int)off, 0, 0));
  else
    return (u32x2){(unsigned)__builtin_amdgcn_raw_buffer_load_b32(rows, (int)off, 0, 0), 0};
}
__device__ __forceinline__ unsigned mx_word(__amdgpu_buffer_rsrc_t rows, unsigned off) {
  return (unsigned)__builtin_amdgcn_raw_buffer_load_b32(rows, (int)off, 0, 0);
}
template <int FORMAT>
__device__ __forceinline__ i32x8 mx_operand(const MxFrag<FORMAT>& f) {
  if constexpr (FORMAT == CT_MX_E4M3)
    return __builtin_bit_cast(i32x8, __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7));
  else
    return __builtin_bit_cast(i32x8, __builtin_shufflevector(f.lo, f.lo, 0, 1, 2, 3, -1, -1, -1, -1));
}
// Whether bf16 does not hold every element of a block with this scale as a normal number; 255 is NaN.
template <int FORMAT>
__device__ __forceinline__ bool mx_far(int scale) {
  constexpr int LOW = FORMAT == CT_MX_E4M3 ? 10 : 2, HIGH = FORMAT == CT_MX_E4M3 ? 246 : 252;
  return (unsigned)(scale - LOW) > (unsigned)(HIGH - LOW);
}
// Whether that matters for elements of a block: not where all of them are 0.
template <int FORMAT>
__device__ __forceinline__ bool mx_counts(u32x2 bits, int scale) {
  return mx_far<FORMAT>(scale) && (scale == 255 || ((bits.x | bits.y) & (FORMAT == CT_MX_E4M3 ? 0x7F7F7F7Fu : 0x77777777u)) != 0);
}
template <int FORMAT>
__device__ __forceinline__ bool mx_counts(const MxFrag<FORMAT>& f, int scale) {
  u32x2 bits = {f.lo.x | f.lo.y, f.lo.z | f.lo.w};
  if constexpr (FORMAT == CT_MX_E4M3) bits |= (u32x2){f.hi.x | f.hi.y, f.hi.z | f.hi.w};
  return mx_counts<FORMAT>(bits, scale);
}
constexpr int mx_code(int format) { return format == CT_MX_E4M3 ? 0 : 4; }  // of the instruction

// The rows of an operand, or of its scales, from row r0 on (at most `most` of `rows`).
struct MxRows {
  const void* base;
  unsigned bytes;
};
__device__ __forceinline__ MxRows mx_rows(const void* p, int64_t ld, int r0, int rows, int most, int row_bytes) {
  const int have = min(rows - r0, most);
  return {(const char*)p + r0 * ld, have > 0 && row_bytes > 0 ? (unsigned)((have - 1) * ld + row_bytes) : 0};
}

// Operands go through LDS also where no two waves share them: a copy of 16 bytes a lane takes whole
// 64-byte pieces of rows, lane by lane, while a lane's own fragment of 16 rows straight from memory is
// 16 lines to the cache at each load (24 x 8192 by 4096: 18.7 us so, 9.5 through LDS).
//
// A block computes BM x BN outputs with WK teams of WM x WN waves, each team every WK-th step of
// 128 elements. Steps go through STAGES buffers in LDS, copied straight into it, the later ones in
// flight while one is multiplied; the 16-byte groups of a row are permuted by its number, so that
// the 16 rows of a fragment lie in distinct banks. Every address is in bounds: rows are a buffer
// that ends with the last of the tile's, and rows, groups and scales past the end have an offset
// past it, and read 0.
// Waves of a SIMD that the registers leave room for: three blocks of 128 x 128 fit LDS.
constexpr int mx_waves(bool exact, int tile) { return exact && tile == 128 * 128 ? 3 : 1; }

template <int FW, int FX, bool EXACT, int BM, int BN, int WM, int WN, int WK, int STAGES>
__global__ void __launch_bounds__(64 * WM * WN * WK, mx_waves(EXACT, BM * BN)) mx_linear_kernel(MxLinearArgs a) {
  constexpr int WAVES = WM * WN, RBW = mx_step_bytes(FW), RBX = mx_step_bytes(FX);
  constexpr int RPCW = 1024 / RBW, RPCX = 1024 / RBX;  // rows of one copy
  constexpr int NCW = BN / RPCW / WAVES, NCX = BM / RPCX / WAVES;  // copies of a wave
  constexpr int SW = BN / WAVES, SX = BM / WAVES;  // rows whose scales a wave copies
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int AT_X = BN * RBW, AT_SW = AT_X + BM * RBX, AT_SX = AT_SW + BN * 4, TEAM = AT_SX + BM * 4;
  constexpr int STAGE = WK * TEAM;
  static_assert(BN % (RPCW * WAVES) == 0 && BM % (RPCX * WAVES) == 0 && SW <= 64 && SX <= 64, "every wave copies as many rows");
  extern __shared__ __align__(16) char lds[];

  const TileAt tile = tile_of_block(a, (int)blockIdx.x);
  const int m0 = tile.mi * BM, n0 = tile.ni * BN, sp = (int)blockIdx.y;
  const int lane = (int)threadIdx.x & 63, team = wave_id() / WAVES, wave = wave_id() % WAVES;
  const int steps = (a.blocks + 3) / 4, begin = sp * a.per_split, end = min(steps, begin + a.per_split);
  const int rounds = (end - begin + WK - 1) / WK;  // steps of a team

  const int row_w = a.blocks * (RBW / 4), row_x = a.blocks * (RBX / 4), row_s = steps * 4;  // bytes
  const MxRows vw = mx_rows(a.w, a.ldw, n0, a.n, BN, row_w), vx = mx_rows(a.x, a.ldx, m0, a.m, BM, row_x);
  const MxRows vsw = mx_rows(a.wsc, a.ldws, n0, a.n, BN, row_s), vsx = mx_rows(a.xs, a.ldxs, m0, a.m, BM, row_s);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(vw.base, vw.bytes), rx = make_rsrc(vx.base, vx.bytes);
  const __amdgpu_buffer_rsrc_t rsw = make_rsrc(vsw.base, vsw.bytes), rsx = make_rsrc(vsx.base, vsx.bytes);

  // The row of copy i that a lane copies 16 bytes of in each step, and which: whole rows to a copy,
  // lane by lane in LDS, so that the permutation of a row's groups is one of the addresses that its
  // lanes read (the same for every copy, but for a single wave's of 8-bit rows).
  const auto row_of = [&](int rb, int i) { return (i * WAVES + wave) * (1024 / rb) + lane / (rb / 16); };
  const auto first = [&](int rb, int i) {
    const bool same = WAVES * (1024 / rb) % (rb / 8) == 0;
    return ((lane % (rb / 16)) ^ ((row_of(rb, same ? 0 : i) >> 1) & (rb / 16 - 1))) * 16;
  };
  unsigned off_w[NCW], off_x[NCX];
#pragma unroll
  for (int i = 0; i < NCW; ++i) {
    const int r = row_of(RBW, i);
    off_w[i] = n0 + r < a.n ? (unsigned)(r * (int)a.ldw + first(RBW, i)) : kOobGroup;
  }
#pragma unroll
  for (int i = 0; i < NCX; ++i) {
    const int r = row_of(RBX, i);
    off_x[i] = m0 + r < a.m ? (unsigned)(r * (int)a.ldx + first(RBX, i)) : kOobGroup;
  }
  // Rows past the last have its scales: their elements are 0, and no scale is there that the operands do not have.
  const unsigned off_sw = (unsigned)(min(wave * SW + lane, a.n - 1 - n0) * (int)a.ldws);
  const unsigned off_sx = (unsigned)(min(wave * SX + lane, a.m - 1 - m0) * (int)a.ldxs);

  auto fetch = [&](int c, int stage) __attribute__((always_inline)) {
    const int step = begin + c * WK + team;
    char* dst = lds + stage * STAGE + team * TEAM;
    auto go = [&](auto tail) __attribute__((always_inline)) {
      const bool none = tail.value && step >= end;
      const auto at = [&](int rb, unsigned bytes) {
        const unsigned k = (unsigned)step * (unsigned)rb;
        return tail.value ? uniform_part(k, bytes) : (int)k;
      };
      const int kw = at(RBW, vw.bytes), kx = at(RBX, vx.bytes), ksw = at(4, vsw.bytes), ksx = at(4, vsx.bytes);
#pragma unroll
      for (int i = 0; i < NCW; ++i) {
        const bool out = none || (tail.value && step * RBW + first(RBW, i) >= row_w);
        copy_lds<16>(rw, dst + (i * WAVES + wave) * 1024, out ? kOobGroup : off_w[i], kw);
      }
#pragma unroll
      for (int i = 0; i < NCX; ++i) {
        const bool out = none || (tail.value && step * RBX + first(RBX, i) >= row_x);
        copy_lds<16>(rx, dst + AT_X + (i * WAVES + wave) * 1024, out ? kOobGroup : off_x[i], kx);
      }
      // some lane of every wave copies, so that the copies on their way are as many in each
      if (lane < SW) copy_lds<4>(rsw, dst + AT_SW + wave * SW * 4, none ? kOobGroup : off_sw, ksw);
      if (lane < SX) copy_lds<4>(rsx, dst + AT_SX + wave * SX * 4, none ? kOobGroup : off_sx, ksx);
    };
    if (step * 4 + 4 <= a.blocks && step < end) go(std::false_type{});
    else go(std::true_type{});
  };

  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const int lrow = lane & 15, kg = lane >> 4;
  // Where a lane's 32 elements of row lrow lie: e2m1 one group, e4m3 two.
  const auto place = [&](int rb, int half) {
    const int g = rb == 64 ? kg : EXACT ? 2 * kg + half : kg + 4 * half;
    return lrow * rb + ((g ^ (lrow >> 1)) & (rb / 16 - 1)) * 16;
  };
  const int pw0 = place(RBW, 0), pw1 = place(RBW, 1), px0 = place(RBX, 0), px1 = place(RBX, 1);
  f32x4 acc[TN][TM] = {};
  bool again = false;  // exact sums: bf16 does not hold all elements of the wave's rows
  auto multiply = [&](int c, int stage) __attribute__((always_inline)) {
    const char* base = lds + stage * STAGE + team * TEAM;
    const char *sw = base + wn * RBW, *sx = base + AT_X + wm * RBX;
    const unsigned char *cw = (const unsigned char*)base + AT_SW + (wn + lrow) * 4 + kg,
                        *cx = (const unsigned char*)base + AT_SX + (wm + lrow) * 4 + kg;
    // scales behind a row's last block, or the slice's, are not read as such: their elements are 0
    const bool real = (begin + c * WK + team) * 4 + kg < min(a.blocks, end * 4);
    const auto read_w = [&](int i) __attribute__((always_inline)) {
      MxFrag<FW> f;
      f.lo = *(const u32x4*)(sw + i * 16 * RBW + pw0);
      if constexpr (FW == CT_MX_E4M3) f.hi = *(const u32x4*)(sw + i * 16 * RBW + pw1);
      return f;
    };
    const auto read_x = [&](int j) __attribute__((always_inline)) {
      MxFrag<FX> f;
      f.lo = *(const u32x4*)(sx + j * 16 * RBX + px0);
      if constexpr (FX == CT_MX_E4M3) f.hi = *(const u32x4*)(sx + j * 16 * RBX + px1);
      return f;
    };
    MxFrag<FW> fw[TN];
    MxFrag<FX> fx[TM];
    int ew[TN], ex[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      fw[i] = read_w(i);
      ew[i] = cw[i * 64];
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      fx[j] = read_x(j);
      ex[j] = cx[j * 64];
    }
    if (!real) {
#pragma unroll
      for (int i = 0; i < TN; ++i) ew[i] = 127;
#pragma unroll
      for (int j = 0; j < TM; ++j) ex[j] = 127;
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int c4 = 0; c4 < 4; ++c4) {
        bf16x8 bw[TN];
#pragma unroll
        for (int i = 0; i < TN; ++i) bw[i] = mx_bf16<FW>(fw[i], c4, (unsigned)ew[i]);
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          const bf16x8 bx = mx_bf16<FX>(fx[j], c4, (unsigned)ex[j]);
#pragma unroll
          for (int i = 0; i < TN; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[i], bx, acc[i][j], 0, 0, 0);
        }
      }
      int low_w = ew[0], high_w = ew[0], low_x = ex[0], high_x = ex[0];
#pragma unroll
      for (int i = 1; i < TN; ++i) {
        low_w = min(low_w, ew[i]);
        high_w = max(high_w, ew[i]);
      }
#pragma unroll
      for (int j = 1; j < TM; ++j) {
        low_x = min(low_x, ex[j]);
        high_x = max(high_x, ex[j]);
      }
      if (__ballot(mx_far<FW>(low_w) || mx_far<FW>(high_w) || mx_far<FX>(low_x) || mx_far<FX>(high_x))) {
        asm volatile("" ::: "memory");  // the elements are read again, or they would stay in registers until here
        bool counts = false;
#pragma unroll
        for (int i = 0; i < TN; ++i) counts |= mx_counts<FW>(read_w(i), ew[i]);
#pragma unroll
        for (int j = 0; j < TM; ++j) counts |= mx_counts<FX>(read_x(j), ex[j]);
        again |= __ballot(counts) != 0;
      }
    } else {
      constexpr int CW = mx_code(FW), CX = mx_code(FX);
#pragma unroll
      for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int i = 0; i < TN; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand<FW>(fw[i]), mx_operand<FX>(fx[j]), acc[i][j],
                                                                       CW, CX, 0, ew[i], 0, ex[j]);
    }
  };

  // Steps past the end read 0, so that STAGES - 1 of them are in flight at every wait. The
  // barrier also says that every wave has read the stage that is filled next; a team of one wave has
  // copied and read its stages itself, and does not wait for the others.
  static_assert((NCW + NCX + 2) * (STAGES - 2) <= 63, "the counter of loads on their way has six bits");
  if (rounds > 0) {
#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c) fetch(c, c);
    int stage = 0;
    for (int c = 0; c < rounds; ++c) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NCW + NCX + 2) * (STAGES - 2)) : "memory");
      if constexpr (WAVES > 1) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      fetch(c + STAGES - 1, stage ? stage - 1 : STAGES - 1);
      multiply(c, stage);
      stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
  }
  if constexpr (EXACT) {
    if (again) {
      // The wave's sums once more, a tile at a time and a block, 32 elements, with each instruction: the tiles
      // that are done wait where the sums of every wave are, and nothing else needs registers that others do not.
      // Outputs of rows without such a block keep theirs: their bits are no matter of other rows.
      const auto at = [&](int row, int64_t ld, int block, int bytes) { return (unsigned)(row * (int)ld + block * bytes * 4 + kg * bytes); };
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          const int of_w = wn + i * 16 + lrow, of_x = wm + j * 16 + lrow, to = wn + i * 16 + kg * 4;
          const bool has_w = n0 + of_w < a.n, has_x = m0 + of_x < a.m;
          f32x4 total = {};
          int bad_w = 0, bad_x = 0;  // of the rows whose elements the lane reads
#pragma unroll 1
          for (int step = begin + team; step < end; step += WK) {
            u32x2 w[4], x[4];
            unsigned e_w[4], e_x, own_w;  // of four blocks each: bytes behind the last block are not read as scales
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const bool real = step * 4 + b < a.blocks;
              w[b] = mx_raw<FW>(rw, has_w && real ? at(of_w, a.ldw, step * 4 + b, RBW / 16) : kOobGroup);
              x[b] = mx_raw<FX>(rx, has_x && real ? at(of_x, a.ldx, step * 4 + b, RBX / 16) : kOobGroup);
            }
            own_w = mx_word(rsw, has_w ? (unsigned)(of_w * (int)a.ldws + step * 4) : kOobGroup);
            e_x = mx_word(rsx, has_x ? (unsigned)(of_x * (int)a.ldxs + step * 4) : kOobGroup);
#pragma unroll
            for (int e = 0; e < 4; ++e) e_w[e] = mx_word(rsw, n0 + to + e < a.n ? (unsigned)((to + e) * (int)a.ldws + step * 4) : kOobGroup);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              if (step * 4 + b >= a.blocks) break;
              const f32x4 none = {};
              const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx_eight<FW>(w[b].x, w[b].y, 127), mx_eight<FX>(x[b].x, x[b].y, 127), none, 0, 0, 0);
              const int sx = e_x >> 8 * b & 255;
              bad_w |= mx_counts<FW>(w[b], own_w >> 8 * b & 255);
              bad_x |= mx_counts<FX>(x[b], sx);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int sw = e_w[e] >> 8 * b & 255;
                total[e] += sw == 255 || sx == 255 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(sum[e], sw + sx - 254);
              }
            }
          }
          const auto whole = [](int bad) {  // of the row, from its four lanes
            bad |= __shfl_xor(bad, 16);
            return bad | __shfl_xor(bad, 32);
          };
          bad_w = whole(bad_w);
          bad_x = whole(bad_x);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = __shfl(bad_w, kg * 4 + e) | bad_x ? total[e] : acc[i][j][e];
        }
    }
  }
  // The compiler counts the waits behind this instruction's results by the passes of 4-bit
  // operands on some paths, four too few of e4m3.
  asm volatile("s_nop 15" ::: "memory");
  write_tile<BM, BN, WM, WN, WK, STAGES * STAGE>(a, lds, acc, m0, n0, sp);
}

// ------------------------------------------------------------------ plans and launches
MxLinearPlan plan_mx_linear(const ct_mx_linear_op& op) { return mx_linear_plan(op); }

template <int FW, int FX, bool EXACT, int KIND>
static int mxl_launch(MxLinearArgs a, hipStream_t st) {
  constexpr MxShape t = kMxTiles[KIND];
  constexpr int stage = t.wk * (t.bn * (mx_step_bytes(FW) + 4) + t.bm * (mx_step_bytes(FX) + 4));
  if (!set_tiles(a, t.bm, t.bn, 64 * t.wm * t.wn * t.wk)) return refuse_size("ct_mx_linear_run");
  return launch(mx_linear_kernel<FW, FX, EXACT, t.bm, t.bn, t.wm, t.wn, t.wk, t.stages>,
                dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.split), 64 * t.wm * t.wn * t.wk, t.stages * stage, st, a);
}
template <int FW, int FX, bool EXACT>
static int mxl_pick(const MxLinearArgs& a, int kind, hipStream_t st) {
  switch (kind) {
    case MXL_32X16: return mxl_launch<FW, FX, EXACT, MXL_32X16>(a, st);
    case MXL_32: return mxl_launch<FW, FX, EXACT, MXL_32>(a, st);
    case MXL_64: return mxl_launch<FW, FX, EXACT, MXL_64>(a, st);
    case MXL_128X64: return mxl_launch<FW, FX, EXACT, MXL_128X64>(a, st);
    case MXL_128: return mxl_launch<FW, FX, EXACT, MXL_128>(a, st);
    default:
      if constexpr (!EXACT) return mxl_launch<FW, FX, EXACT, MXL_256>(a, st);
      set_error("ct_mx_linear_run: no 256 x 256 tiles of exact sums");  // mx_linear_plan takes none
      return -2;
  }
}
template <int FW, int FX>
static int mxl_sums(const MxLinearArgs& a, int kind, hipStream_t st) {
  return a.out_bf16 ? mxl_pick<FW, FX, false>(a, kind, st) : mxl_pick<FW, FX, true>(a, kind, st);
}

int launch_mx_linear(const ct_mx_linear_op& op, const MxLinearPlan& p, const MxLinearArrays& v, void* stream) {
  if (p.tail_m || p.tail_n) {
    const int64_t o = elem_bytes(op.out_dtype);
    const auto part = [&](int m0, int m, int n0, int n, bool whole) {
      ct_mx_linear_op sub = op;
      sub.m = m;
      sub.n = n;
      MxLinearPlan q = p;
      q.tail_m = q.tail_n = 0;
      if (!whole) q.kind = plan_mx_linear(sub).kind;
      const int64_t at = m0 * op.ldy + n0, rat = m0 * op.ldr + n0;
      const MxLinearArrays a = {(const char*)v.x + m0 * op.ldx, (const char*)v.xs + m0 * op.ldxs,
                                (const char*)v.w + n0 * op.ldw, (const char*)v.ws + n0 * op.ldws,
                                v.bias ? v.bias + n0 : nullptr, op.res ? (const char*)v.res + rat * o : nullptr,
                                (char*)v.y + at * o, nullptr};
      return launch_mx_linear(sub, q, a, stream);
    };
    const int m = op.m - p.tail_m, n = op.n - p.tail_n;
    int rc = part(0, m, 0, n, true);
    if (!rc && p.tail_n) rc = part(0, op.m, n, p.tail_n, false);
    if (!rc && p.tail_m) rc = part(m, p.tail_m, 0, n, false);
    return rc;
  }
  MxLinearArgs a = {};
  a.x = (const char*)v.x; a.xs = (const unsigned char*)v.xs;
  a.w = (const char*)v.w; a.wsc = (const unsigned char*)v.ws;
  a.bias = v.bias; a.res = v.res; a.y = v.y; a.ws = v.scratch;
  a.m = op.m; a.n = op.n; a.blocks = mx_blocks(op.k);
  a.ldx = op.ldx; a.ldxs = op.ldxs; a.ldw = op.ldw; a.ldws = op.ldws; a.ldr = op.ldr; a.ldy = op.ldy;
  a.act = op.act; a.res_mode = op.res; a.out_bf16 = op.out_dtype == CT_DT_BF16;
  a.split = p.split; a.per_split = p.per_split;
  a.stream = (int64_t)op.m * op.n * elem_bytes(op.out_dtype) >= kStreamBytes;
  hipStream_t st = (hipStream_t)stream;
  const bool w8 = op.w_format == CT_MX_E4M3, x8 = op.x_format == CT_MX_E4M3;
  const int rc = w8 ? x8 ? mxl_sums<CT_MX_E4M3, CT_MX_E4M3>(a, p.kind, st) : mxl_sums<CT_MX_E4M3, CT_MX_E2M1>(a, p.kind, st)
                    : x8 ? mxl_sums<CT_MX_E2M1, CT_MX_E4M3>(a, p.kind, st) : mxl_sums<CT_MX_E2M1, CT_MX_E2M1>(a, p.kind, st);
  return rc || p.split == 1 ? rc : launch_join(a, st);
}

}  // namespace ct
