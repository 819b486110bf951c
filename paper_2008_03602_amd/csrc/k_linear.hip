// Matrix product with its epilogue: y = act(x w^T + bias) + r, or act(x w^T + bias + r).
//
// x (m x k) and w (n x k) are both contiguous along the reduction, so a fragment of either
// is 16 bytes of a row. The weights are the matrix instruction's first operand: a lane's
// four consecutive accumulators are then four consecutive outputs of one row of y.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "k_seq.h"

namespace ct {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const void *x, *w, *res;
  const float* bias;
  void* y;
  float* ws;
  int m, n, k;
  int64_t ldx, ldw, ldr, ldy;
  int act, res_mode, out_bf16;
  int vec_out;          // rows of y and r take accesses of four elements
  int tiles_m, tiles_n;
  int split, per_split; // slices of the reduction, 128-byte chunks in each
  FastDiv dgroup, dlast;
};

// acc += A B for one 16-byte group per lane: row lane % 16 of each operand, group lane / 16
// of four. Of fp32 each of the four words is a step of its own; which values of k meet in a
// step does not matter as long as both operands agree.
template <typename T>
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc,
                                                   0, 0, 0);
  } else {
    const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float va = fa[e], vb = fb[e];
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(va, vb, acc, 0, 0, 0);
    }
    return acc;
  }
}

// ------------------------------------------------------------------ epilogue
__device__ __forceinline__ float finish(const LinearArgs& a, float v, float bias, float r) {
  v += bias;
  if (a.res_mode == CT_RES_ADD_ACT) v += r;
  v = activate(v, a.act);
  if (a.res_mode == CT_RES_ADD) v += r;
  return v;
}
// Outputs (i, j .. j+3), those of them that exist.
__device__ __forceinline__ void store4(const LinearArgs& a, int i, int j, f32x4 acc) {
  float v[4] = {acc[0], acc[1], acc[2], acc[3]};
  const int64_t at = i * a.ldy + j, rt = i * a.ldr + j;
  if (a.vec_out && j + 4 <= a.n) {
    f32x4 b = {}, r = {};
    if (a.bias) b = *(const f32x4*)(a.bias + j);
    if (a.res_mode) {
      if (a.out_bf16) {
        const u32x2 q = *(const u32x2*)((const bf16_t*)a.res + rt);
        const unsigned q0 = q.x, q1 = q.y;
        r = (f32x4){unpack<bf16_t>(q0, 0), unpack<bf16_t>(q0, 1), unpack<bf16_t>(q1, 0), unpack<bf16_t>(q1, 1)};
      } else {
        r = *(const f32x4*)((const float*)a.res + rt);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float be = b[e], re = r[e];
      v[e] = finish(a, v[e], be, re);
    }
    if (a.out_bf16) *(u32x2*)((bf16_t*)a.y + at) = (u32x2){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else *(f32x4*)((float*)a.y + at) = (f32x4){v[0], v[1], v[2], v[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (j + e >= a.n) break;
    float r = 0.f;
    if (a.res_mode)
      r = a.out_bf16 ? (float)((const bf16_t*)a.res)[rt + e] : ((const float*)a.res)[rt + e];
    const float out = finish(a, v[e], a.bias ? a.bias[j + e] : 0.f, r);
    if (a.out_bf16) ((bf16_t*)a.y)[at + e] = (bf16_t)out;
    else ((float*)a.y)[at + e] = out;
  }
}
// Partial sums of slice sp: rows of n rounded up to four.
__device__ __forceinline__ void store_part(const LinearArgs& a, int sp, int i, int j, f32x4 acc) {
  const int64_t n4 = (a.n + 3) / 4 * 4;
  *(f32x4*)(a.ws + ((int64_t)sp * a.m + i) * n4 + j) = acc;
}
// Adds the slices in their order and finishes the outputs.
__global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs a) {
  const int n4 = (a.n + 3) / 4;
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= (int64_t)a.m * n4) return;
  const int i = (int)(q / n4), j = (int)(q - (int64_t)i * n4) * 4;
  const float* p = a.ws + q * 4;
  f32x4 v = *(const f32x4*)p;
  for (int s = 1; s < a.split; ++s) v += *(const f32x4*)(p + (int64_t)s * a.m * n4 * 4);
  store4(a, i, j, v);
}

// ------------------------------------------------------------------ 16-byte groups of rows
// Byte offset past every operand tile: reads as 0.
constexpr unsigned kOobGroup = 0xFFFFFFF0u;

__device__ __forceinline__ u32x4 load_quad(__amdgpu_buffer_rsrc_t r, unsigned off) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
}
// A group at any element's address, of which the first `left` elements exist: whole words
// around it, shifted where it starts in the middle of one, the rest masked to 0.
template <typename T>
__device__ __forceinline__ u32x4 load_quad_any(__amdgpu_buffer_rsrc_t r, unsigned off, int left) {
  if constexpr (sizeof(T) == 4) {
    const u32x4 q = load_quad(r, off);
    const unsigned a = q.x, b = q.y, c = q.z, d = q.w;
    return (u32x4){left > 0 ? a : 0, left > 1 ? b : 0, left > 2 ? c : 0, left > 3 ? d : 0};
  } else {
    const unsigned at = off & ~3u;
    const u32x4 q = load_quad(r, at);
    const unsigned e = __builtin_amdgcn_raw_buffer_load_b32(r, (int)(at + 16), 0, 0);
    unsigned v[5] = {q.x, q.y, q.z, q.w, e};
    const unsigned sh = (off & 2u) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __builtin_amdgcn_alignbit(v[i + 1], v[i], sh);
      v[i] = left > 2 * i + 1 ? v[i] : left > 2 * i ? v[i] & 0xFFFFu : 0;
    }
    return (u32x4){v[0], v[1], v[2], v[3]};
  }
}
// The rows of an operand from row r0 on (at most `most` of `rows`): base on a word, bytes up
// to the end of the last row in whole words. odd: 2 where the first row starts in the middle
// of a word.
struct RowsView {
  const void* base;
  unsigned bytes, odd;
};
template <typename T>
__device__ __forceinline__ RowsView rows_view(const void* p, int64_t ld, int r0, int rows, int most, int k) {
  const uintptr_t at = (uintptr_t)p + (uintptr_t)(r0 * ld * (int64_t)sizeof(T));
  const int have = min(rows - r0, most);
  const unsigned odd = (unsigned)(at & 3);
  const int64_t bytes = have > 0 && k > 0 ? (((have - 1) * ld + k) * (int64_t)sizeof(T) + odd + 3) / 4 * 4 : 0;
  return {(const void*)(at - odd), (unsigned)bytes, odd};
}

// ------------------------------------------------------------------ tiles
// A block computes BM x BN outputs with WM x WN waves. Operand slices of 128 bytes of each
// row go through two LDS stages; the 16-byte groups of a row are permuted by its number, so
// that the 16 rows of a fragment lie in distinct banks.
template <typename T, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ void __launch_bounds__(64 * WM * WN) linear_tile_kernel(LinearArgs a) {
  constexpr int WAVES = WM * WN, ROWS = BM + BN, G = 16 / (int)sizeof(T), KC = 8 * G;
  constexpr int NC = ROWS / 8 / WAVES, NW = BN / 8 / WAVES;  // copies of a wave, those of w first
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16, STAGE = ROWS * 128;
  extern __shared__ __align__(16) char lds[];

  // Each XCD takes one band of tiles, in columns four tiles wide: the tiles at work on it
  // share a few panels of x and four of w in its L2.
  const int idx = xcd_band_tile((int)blockIdx.x, a.tiles_m * a.tiles_n);
  const int grp = fdiv(idx, a.dgroup), in = idx - grp * a.dgroup.d;
  int mi, ni;
  if (grp * 4 + 4 <= a.tiles_n) {
    mi = in >> 2;
    ni = grp * 4 + (in & 3);
  } else {
    mi = fdiv(in, a.dlast);
    ni = grp * 4 + in - mi * a.dlast.d;
  }
  const int m0 = mi * BM, n0 = ni * BN, sp = (int)blockIdx.y;
  const int lane = (int)threadIdx.x & 63, wave = wave_id();
  const int c0 = sp * a.per_split, chunks = min((a.k + KC - 1) / KC - c0, a.per_split);

  const RowsView vw = rows_view<T>(a.w, a.ldw, n0, a.n, BN, a.k), vx = rows_view<T>(a.x, a.ldx, m0, a.m, BM, a.k);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(vw.base, vw.bytes), rx = make_rsrc(vx.base, vx.bytes);
  unsigned off[NC];  // of this lane's group in each copy: eight rows of eight groups
  int grp_k[NC];     // its first element in the slice
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int r = ((i < NW ? i : i - NW) * WAVES + wave) * 8 + (lane >> 3);
    const int g = (lane & 7) ^ ((r >> 1) & 7);
    grp_k[i] = g * G;
    const bool ok = i < NW ? n0 + r < a.n : m0 + r < a.m;
    const unsigned ld = (unsigned)((i < NW ? a.ldw : a.ldx) * (int)sizeof(T));
    off[i] = ok ? (unsigned)r * ld + 16u * g + (i < NW ? vw.odd : vx.odd) : kOobGroup;
  }

  u32x4 held[DIRECT ? 1 : NC];
  auto fetch = [&](int c, int stage) __attribute__((always_inline)) {
    const int k0 = (c0 + c) * KC;
    const bool tail = k0 + KC > a.k;
    char* dst = lds + stage * STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int left = a.k - k0 - grp_k[i];
      if constexpr (DIRECT) {
        const unsigned o = tail && left <= 0 ? kOobGroup : off[i];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(i < NW ? rw : rx, (lds_void_t*)(dst + i * WAVES * 1024), 16, (int)o,
                                                 k0 * (int)sizeof(T), 0, 0);
      } else {
        const unsigned o = off[i] == kOobGroup || left <= 0 ? kOobGroup : off[i] + (unsigned)(k0 * (int)sizeof(T));
        held[i] = load_quad_any<T>(i < NW ? rw : rx, o, left);
      }
    }
  };
  auto put = [&](int stage) __attribute__((always_inline)) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < NC; ++i) *(u32x4*)(lds + stage * STAGE + (i * WAVES + wave) * 1024 + lane * 16) = held[i];
    }
  };

  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const int lrow = lane & 15, kg = lane >> 4;
  const int at0 = lrow * 128 + ((kg ^ (lrow >> 1)) * 16), at1 = at0 ^ 64;  // the slice's halves
  f32x4 acc[TN][TM] = {};
  auto multiply = [&](int stage) __attribute__((always_inline)) {
    const char* sw = lds + stage * STAGE + wn * 128;
    const char* sx = lds + stage * STAGE + (BN + wm) * 128;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = s ? at1 : at0;
      u32x4 fw[TN], fx[TM];
#pragma unroll
      for (int i = 0; i < TN; ++i) fw[i] = *(const u32x4*)(sw + at + i * 2048);
#pragma unroll
      for (int j = 0; j < TM; ++j) fx[j] = *(const u32x4*)(sx + at + j * 2048);
#pragma unroll
      for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int i = 0; i < TN; ++i) acc[i][j] = mma16<T>(fw[i], fx[j], acc[i][j]);
    }
  };

  if (chunks > 0) {
    fetch(0, 0);
    put(0);
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
      if (c + 1 < chunks) fetch(c + 1, (c + 1) & 1);
      multiply(c & 1);
      if (c + 1 < chunks) put((c + 1) & 1);
      __syncthreads();
    }
  }

  // The sums go through the wave's share of LDS, as many rows of its tile at a time as it
  // holds, so that each access to y and r takes whole rows of the tile.
  constexpr int RM = BM / WM, RN = BN / WN, SLOTS = RN / 4;  // 16-byte slots of a row
  constexpr int FIT = 2 * STAGE / WAVES / (RN * 4), H = FIT < RM ? FIT : RM;
  char* mine = lds + wave * (H * RN * 4);
  auto slot = [](int r, int s) { return (s ^ ((SLOTS == 16 ? r : r >> 1) & (SLOTS - 1))) * 16; };
#pragma unroll
  for (int h = 0; h < RM; h += H) {
#pragma unroll
    for (int j = 0; j < H / 16; ++j)
#pragma unroll
      for (int i = 0; i < TN; ++i)
        *(f32x4*)(mine + (j * 16 + lrow) * RN * 4 + slot(j * 16 + lrow, i * 4 + kg)) = acc[i][h / 16 + j];
    for (int q = lane; q < H * SLOTS; q += 64) {
      const int r = q / SLOTS, s = q % SLOTS, row = m0 + wm + h + r, col = n0 + wn + s * 4;
      if (row >= a.m || col >= a.n) continue;
      const f32x4 v = *(const f32x4*)(mine + r * RN * 4 + slot(r, s));
      if (a.split > 1) store_part(a, sp, row, col, v);
      else store4(a, row, col, v);
    }
  }
}

// ------------------------------------------------------------------ few rows
// Up to 16 MT rows of x: a block of WAVES waves computes 16 columns. The waves share the
// reduction out in steps of 64 bytes of a row, D steps in flight each, and add their sums
// through LDS in the order of the waves.
template <typename T, int MT, int WAVES, int D, bool DIRECT>
__global__ void __launch_bounds__(64 * WAVES) linear_rows_kernel(LinearArgs a) {
  constexpr int G = 16 / (int)sizeof(T), KS = 4 * G;
  __shared__ f32x4 part[WAVES][MT][64];
  const int n0 = (int)blockIdx.x * 16, sp = (int)blockIdx.y;
  const int lane = (int)threadIdx.x & 63, wave = wave_id();
  const int lrow = lane & 15, kg = lane >> 4;
  const RowsView vw = rows_view<T>(a.w, a.ldw, n0, a.n, 16, a.k), vx = rows_view<T>(a.x, a.ldx, 0, a.m, 16 * MT, a.k);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(vw.base, vw.bytes), rx = make_rsrc(vx.base, vx.bytes);
  const unsigned ow = n0 + lrow < a.n ? (unsigned)lrow * (unsigned)(a.ldw * (int)sizeof(T)) + vw.odd : kOobGroup;
  unsigned ox[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j)
    ox[j] = 16 * j + lrow < a.m ? (unsigned)(16 * j + lrow) * (unsigned)(a.ldx * (int)sizeof(T)) + vx.odd : kOobGroup;

  const int s0 = sp * a.per_split * 2, s1 = min((a.k + KS - 1) / KS, s0 + a.per_split * 2);
  auto load = [&](__amdgpu_buffer_rsrc_t r, unsigned o, int k) __attribute__((always_inline)) {
    const unsigned at = o == kOobGroup || k >= a.k ? kOobGroup : o + (unsigned)(k * (int)sizeof(T));
    if constexpr (DIRECT) return load_quad(r, at);
    else return load_quad_any<T>(r, at, a.k - k);
  };
  u32x4 fw[D], fx[D][MT];
  f32x4 acc[MT] = {};
  auto fetch = [&](int u, int s) __attribute__((always_inline)) {
    const int k = s < s1 ? s * KS + kg * G : a.k;
    fw[u] = load(rw, ow, k);
#pragma unroll
    for (int j = 0; j < MT; ++j) fx[u][j] = load(rx, ox[j], k);
  };
#pragma unroll
  for (int u = 0; u < D; ++u) fetch(u, s0 + wave + u * WAVES);
  for (int s = s0 + wave; s < s1; s += D * WAVES) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[j] = mma16<T>(fw[u], fx[u][j], acc[j]);
      fetch(u, s + (u + D) * WAVES);
    }
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) part[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave < MT) {
    f32x4 v = part[0][wave][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += part[i][wave][lane];
    const int row = wave * 16 + lrow, col = n0 + 4 * kg;
    if (row < a.m && col < a.n) {
      if (a.split > 1) store_part(a, sp, row, col, v);
      else store4(a, row, col, v);
    }
  }
}

// ------------------------------------------------------------------ plans and launches
enum { LIN_ROWS, LIN_64, LIN_128, LIN_256 };

static int64_t tiles_of(const ct_linear_op& op, int t) {
  return (int64_t)((op.m + t - 1) / t) * ((op.n + t - 1) / t);
}

LinearPlan plan_linear(const ct_linear_op& op) {
  LinearPlan p = {};
  const int chunks = (int)(((int64_t)op.k * elem_bytes(op.dtype) + 127) / 128);
  int64_t blocks;
  if (op.m <= 64) {
    p.kind = LIN_ROWS;
    blocks = (op.n + 15) / 16;
  } else {
    p.kind = tiles_of(op, 256) >= kPlanCus * 3 / 4 ? LIN_256 : tiles_of(op, 128) >= kPlanCus ? LIN_128 : LIN_64;
    blocks = tiles_of(op, p.kind == LIN_256 ? 256 : p.kind == LIN_128 ? 128 : 64);
  }
  // Too few blocks for the compute units: slices of the reduction, of 8 chunks at least
  int split = blocks < kPlanCus ? (int)(kPlanCus / blocks) : 1;
  if (split > chunks / 8) split = chunks / 8;
  if (split > 16) split = 16;
  if (split < 1) split = 1;
  p.per_split = chunks ? (chunks + split - 1) / split : 1;
  p.split = chunks ? (chunks + p.per_split - 1) / p.per_split : 1;
  p.ws_floats = p.split > 1 ? (int64_t)p.split * op.m * ((op.n + 3) / 4 * 4) : 0;
  return p;
}

template <typename T, int BM, int BN, int WM, int WN, bool DIRECT>
static int launch_tile(LinearArgs a, hipStream_t st) {
  a.tiles_m = (a.m + BM - 1) / BM;
  a.tiles_n = (a.n + BN - 1) / BN;
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
  if (tiles > 0x7FFFFFFF || 4 * (int64_t)a.tiles_m > 0x7FFFFFFF) return refuse_size("ct_linear_run");
  a.dgroup = make_fastdiv(4 * (int64_t)a.tiles_m);
  a.dlast = make_fastdiv(a.tiles_n % 4 ? a.tiles_n % 4 : 4);
  hipLaunchKernelGGL((linear_tile_kernel<T, BM, BN, WM, WN, DIRECT>), dim3((unsigned)tiles, (unsigned)a.split),
                     dim3(64 * WM * WN), 2 * (BM + BN) * 128, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}
template <typename T, int MT, bool DIRECT>
static int launch_rows(const LinearArgs& a, hipStream_t st) {
  constexpr int WAVES = 16, D = MT <= 2 ? 4 : 2;
  hipLaunchKernelGGL((linear_rows_kernel<T, MT, WAVES, D, DIRECT>), dim3((unsigned)((a.n + 15) / 16), (unsigned)a.split),
                     dim3(64 * WAVES), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}
template <typename T, bool DIRECT>
static int linear_pick(const LinearArgs& a, int kind, hipStream_t st) {
  switch (kind) {
    case LIN_256:
      if constexpr (DIRECT) return launch_tile<T, 256, 256, 2, 4, DIRECT>(a, st);
    case LIN_128: return launch_tile<T, 128, 128, 2, 2, DIRECT>(a, st);
    case LIN_64: return launch_tile<T, 64, 64, 2, 2, DIRECT>(a, st);
  }
  if (a.m <= 16) return launch_rows<T, 1, DIRECT>(a, st);
  if (a.m <= 32) return launch_rows<T, 2, DIRECT>(a, st);
  return launch_rows<T, 4, DIRECT>(a, st);
}

int launch_linear(const ct_linear_op& op, const LinearPlan& p, const void* x, const void* w, const float* bias,
                  const void* res, void* y, float* ws, void* stream) {
  LinearArgs a = {};
  a.x = x; a.w = w; a.res = res; a.bias = bias; a.y = y; a.ws = ws;
  a.m = op.m; a.n = op.n; a.k = op.k;
  a.ldx = op.ldx; a.ldw = op.ldw; a.ldr = op.ldr; a.ldy = op.ldy;
  a.act = op.act; a.res_mode = op.res; a.out_bf16 = op.out_dtype == CT_DT_BF16;
  a.split = p.split; a.per_split = p.per_split;
  const int e = elem_bytes(op.dtype), four = 4 * elem_bytes(op.out_dtype);
  a.vec_out = (uintptr_t)y % four == 0 && op.ldy % 4 == 0 && (uintptr_t)bias % 16 == 0 &&
              (!op.res || ((uintptr_t)res % four == 0 && op.ldr % 4 == 0));
  const bool direct = ((uintptr_t)x | (uintptr_t)w) % 16 == 0 && op.ldx * e % 16 == 0 && op.ldw * e % 16 == 0 &&
                      op.k * (int64_t)e % 16 == 0;
  hipStream_t st = (hipStream_t)stream;
  int rc;
  if (op.dtype == CT_DT_BF16)
    rc = direct ? linear_pick<bf16_t, true>(a, p.kind, st) : linear_pick<bf16_t, false>(a, p.kind, st);
  else
    rc = direct ? linear_pick<float, true>(a, p.kind, st) : linear_pick<float, false>(a, p.kind, st);
  if (rc || p.split == 1) return rc;
  const int64_t quads = (int64_t)op.m * ((op.n + 3) / 4);
  hipLaunchKernelGGL(linear_join_kernel, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace ct
