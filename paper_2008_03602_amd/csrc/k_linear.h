// What the products share: which tile a block computes, and the epilogue of its sums.
#pragma once
#include "k_seq.h"

namespace ct {

// One wave instruction: lane i copies BYTES bytes at byte offset off + k of r to lds + BYTES i.
template <int BYTES>
__device__ __forceinline__ void copy_lds(__amdgpu_buffer_rsrc_t r, char* lds, unsigned off, int k) {
  if constexpr (BYTES == 4) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 4, (int)off, k, 0, 0);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 16, (int)off, k, 0, 0);
}

// The outputs of a product and what goes into them beside the sums.
struct OutArgs {
  const void* res;
  const float* bias;
  void* y;
  float* ws;
  int m, n;
  int64_t ldr, ldy;
  int act, res_mode, out_bf16;
  int stream;  // y goes past the caches
  int tiles_m, tiles_n;
  int split;  // slices of the reduction
  FastDiv dgroup, dlast;
};

// Tile (mi, ni) of block b.
struct TileAt {
  int mi, ni;
};
__device__ __forceinline__ TileAt tile_of_block(const OutArgs& a, int b) {
  // Each XCD takes one band of tiles, in columns four tiles wide: the tiles at work on it
  // share a few panels of x and four of w in its L2.
  const int idx = xcd_band_tile(b, a.tiles_m * a.tiles_n);
  const int grp = fdiv(idx, a.dgroup), in = idx - grp * a.dgroup.d;
  int mi, ni;
  if (grp * 4 + 4 <= a.tiles_n) {
    mi = in >> 2;
    ni = grp * 4 + (in & 3);
  } else {
    mi = fdiv(in, a.dlast);
    ni = grp * 4 + in - mi * a.dlast.d;
  }
  return {mi, ni};
}
// The tile counts of a launch; false where a block's number would not fit.
inline bool set_tiles(OutArgs& a, int bm, int bn, int threads) {
  a.tiles_m = (a.m + bm - 1) / bm;
  a.tiles_n = (a.n + bn - 1) / bn;
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
  if (!fits_launch(tiles, threads) || 4 * (int64_t)a.tiles_m > 0x7FFFFFFF) return false;
  a.dgroup = make_fastdiv(4 * (int64_t)a.tiles_m);
  a.dlast = make_fastdiv(a.tiles_n % 4 ? a.tiles_n % 4 : 4);
  return true;
}

// ------------------------------------------------------------------ epilogue
// Four columns of the bias, and of a row of the residual, from column j on: 0 where there
// are none.
__device__ __forceinline__ Quad load_bias(const OutArgs& a, int j) {
  Quad q = {};
  if (!a.bias || j >= a.n) return q;
  if (j + 4 <= a.n) return load_quad4(a.bias + j);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < a.n) q.v[e] = a.bias[j + e];
  return q;
}
__device__ __forceinline__ Quad load_res(const OutArgs& a, int i, int j) {
  Quad q = {};
  if (!a.res_mode || i >= a.m || j >= a.n) return q;
  const int64_t at = i * a.ldr + j;
  if (j + 4 <= a.n)
    return a.out_bf16 ? load_quad4((const bf16_t*)a.res + at) : load_quad4((const float*)a.res + at);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < a.n) q.v[e] = a.out_bf16 ? (float)((const bf16_t*)a.res)[at + e] : ((const float*)a.res)[at + e];
  return q;
}
// N quads of outputs from their sums, one choice of the activation for all of them.
template <int N>
__device__ __forceinline__ void finish(const OutArgs& a, float (&v)[N][4], const Quad& bias, const Quad (&res)[N]) {
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q][e] = f(v[q][e], q, e);
  };
  each([&](float x, int, int e) { return x + bias.v[e]; });
  if (a.res_mode == CT_RES_ADD_ACT) each([&](float x, int q, int e) { return x + res[q].v[e]; });
  switch (a.act) {
    case CT_ACT_RELU: each([](float x, int, int) { return activate(x, CT_ACT_RELU); }); break;
    case CT_ACT_RELU6: each([](float x, int, int) { return activate(x, CT_ACT_RELU6); }); break;
    case CT_ACT_SILU: each([](float x, int, int) { return activate(x, CT_ACT_SILU); }); break;
    case CT_ACT_GELU: each([](float x, int, int) { return activate(x, CT_ACT_GELU); }); break;
  }
  if (a.res_mode == CT_RES_ADD) each([&](float x, int q, int e) { return x + res[q].v[e]; });
}
// Outputs (i, j .. j+3), those of them that exist.
__device__ __forceinline__ void store4(const OutArgs& a, int i, int j, f32x4 acc, const Quad& bias, const Quad& r) {
  float v[1][4] = {{acc.x, acc.y, acc.z, acc.w}};
  const Quad res[1] = {r};
  finish(a, v, bias, res);
  const int64_t at = i * a.ldy + j;
  if (j + 4 <= a.n) {
    if (a.out_bf16) store_quad4((bf16_t*)a.y + at, v[0], false);
    else store_quad4((float*)a.y + at, v[0], false);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (j + e >= a.n) break;
    if (a.out_bf16) ((bf16_t*)a.y)[at + e] = (bf16_t)v[0][e];
    else ((float*)a.y)[at + e] = v[0][e];
  }
}
// Partial sums of slice sp: rows of n rounded up to four.
__device__ __forceinline__ void store_part(const OutArgs& a, int sp, int i, int j, f32x4 acc) {
  const int64_t n4 = (a.n + 3) / 4 * 4;
  *(f32x4*)(a.ws + ((int64_t)sp * a.m + i) * n4 + j) = acc;
}
// A block's sums, f32x4 acc[TN][TM] of every wave (tile rows of w by tile rows of x, the weights as the
// matrix instruction's first operand), to y, or to the workspace where the reduction is split. BYTES of
// LDS, which the block no longer needs; copies to it may still be on their way.
template <int BM, int BN, int WM, int WN, int WK, int BYTES, int TN, int TM>
__device__ __forceinline__ void write_tile(const OutArgs& a, char* lds, f32x4 (&acc)[TN][TM], int m0, int n0, int sp) {
  constexpr int WAVES = WM * WN;
  static_assert(TM == BM / WM / 16 && TN == BN / WN / 16, "");
  const int lane = (int)threadIdx.x & 63, team = wave_id() / WAVES, wave = wave_id() % WAVES;
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN), lrow = lane & 15, kg = lane >> 4;
  // The sums go through the wave's share of LDS, as many rows of its tile at a time as it
  // holds, so that each access to y and r takes whole rows of the tile.
  constexpr int RM = BM / WM, RN = BN / WN, SLOTS = RN / 4;  // 16-byte slots of a row
  constexpr int FIT = BYTES / WK / WAVES / (RN * 4), POW = FIT >= 64 ? 64 : FIT >= 32 ? 32 : 16, H = POW < RM ? POW : RM;
  constexpr int STEP = 64 / SLOTS;  // rows of one access
  static_assert(RM % H == 0 && FIT >= 16, "");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // slices past the end, too
  __syncthreads();
  if constexpr (WK > 1) {  // the teams' sums, added in their order by the first
    constexpr int SUMS = BM * BN * 4;
    static_assert(WK * SUMS <= BYTES && H == RM, "");
    if (team > 0) {
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
          *(f32x4*)(lds + team * SUMS + ((wave * TN + i) * TM + j) * 1024 + lane * 16) = acc[i][j];
    }
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int t = 1; t < WK; ++t)
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
          acc[i][j] += *(const f32x4*)(lds + t * SUMS + ((wave * TN + i) * TM + j) * 1024 + lane * 16);
  }
  char* mine = lds + wave * (H * RN * 4);
  auto slot = [](int r, int s) { return (s ^ ((SLOTS >= 16 ? r : r >> 1) & (SLOTS - 1))) * 16; };
  const int sl = lane % SLOTS, col = n0 + wn + sl * 4, r0 = lane / SLOTS;
  const bool whole = m0 + BM <= a.m && n0 + BN <= a.n;  // no output of the tile is missing
  const Quad bias = a.split > 1 ? Quad{} : load_bias(a, col);
  constexpr int ROWS_EACH = H / STEP, Q = ROWS_EACH % 4 ? ROWS_EACH : 4;  // rows of a lane, and at a time
  auto take = [&](int r) { return *(const f32x4*)(mine + r * RN * 4 + slot(r, sl)); };
  auto finish_rows = [&](int h, auto zero) __attribute__((always_inline)) {
    using O = decltype(zero);
    const int64_t row = m0 + wm + h + r0;
    O* y = (O*)a.y + row * a.ldy + col;
    const O* rp = (const O*)a.res + row * a.ldr + col;
#pragma unroll 1
    for (int r = r0; r < H; r += Q * STEP) {
      Quad res[Q] = {};
      if (a.res_mode) {
#pragma unroll
        for (int q = 0; q < Q; ++q) res[q] = load_quad4(rp + q * STEP * a.ldr);
        rp += Q * STEP * a.ldr;
      }
      float v[Q][4];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const f32x4 s = take(r + q * STEP);
        v[q][0] = s.x; v[q][1] = s.y; v[q][2] = s.z; v[q][3] = s.w;
      }
      finish(a, v, bias, res);
#pragma unroll
      for (int q = 0; q < Q; ++q) store_quad4(y + q * STEP * a.ldy, v[q], a.stream);
      y += Q * STEP * a.ldy;
    }
  };
#pragma unroll
  for (int h = 0; h < RM; h += H) {
#pragma unroll
    for (int j = 0; j < H / 16; ++j)
#pragma unroll
      for (int i = 0; i < TN; ++i)
        *(f32x4*)(mine + (j * 16 + lrow) * RN * 4 + slot(j * 16 + lrow, i * 4 + kg)) = acc[i][h / 16 + j];
    if (a.split > 1) {
      for (int r = r0; r < H; r += STEP)
        if (m0 + wm + h + r < a.m && col < a.n) store_part(a, sp, m0 + wm + h + r, col, take(r));
    } else if (whole) {
      if (a.out_bf16) finish_rows(h, bf16_t());
      else finish_rows(h, 0.f);
    } else {
#pragma unroll 1
      for (int r = r0; r < H; r += STEP) {
        const int row = m0 + wm + h + r;
        if (row < a.m && col < a.n) store4(a, row, col, take(r), bias, load_res(a, row, col));
      }
    }
  }
}

// Adds the slices of a split reduction and finishes the outputs (k_linear.hip).
int launch_join(const OutArgs& a, hipStream_t st);

}  // namespace ct
