// Matrix product with its epilogue: y = act(x w^T + bias) + r, or act(x w^T + bias + r).
//
// x (m x k) and w (n x k) are both contiguous along the reduction, so a fragment of either
// is 16 bytes of a row. The weights are the matrix instruction's first operand: a lane's
// four consecutive accumulators are then four consecutive outputs of one row of y. Products
// of bf16 are exact in fp32 and sums are in fp32; only an output is rounded.
//
// What bounds it, and what was chosen for it:
//   * Large products: the matrix cores. 256 x 256 tiles, eight waves of 64 x 128, two slices
//     of 64 KB in LDS, copied straight into it. 8192 x 4096 by 8192 with bias and GELU, bf16:
//     430-465 us, 1.18-1.28 PFLOP/s (a library's bare product: 453 us). Measured and left:
//     waves of 128 x 64 (5 % slower), the 32 x 32 instruction (5 %), slices of 64 bytes with
//     three to five stages (8-12 %), the next slice asked for after the products (16 %), and,
//     with no effect, two groups of waves in turn, priorities, columns of eight tiles.
//   * Few rows: the weights' bytes. 32 x 32 tiles and four teams of waves over the slices, so
//     that 128 tiles keep 8 MB on their way: 24 x 8192 by 4096, bf16, 14.6 us, 4.7 TB/s.
//     Fragments read straight into registers, 16 rows of 64 bytes a load, took 24.5 us.
//   * In between: rounds of the device and, below 64 x 64, a wait and a barrier (0.19 us)
//     every slice, which the teams share out (64 x 4096 by 4096: 12.3 to 9.5 us).
//   * Short reductions: the epilogue. It takes whole rows of the tile through LDS, chooses
//     the activation once for 16 values, and checks nothing where the whole tile exists
//     (12544 x 32 by 192, fp32 out: 9.5 to 5.5 us).
// Rows off 16 bytes are copied a word a lane, which is bound by the copies (471 x 3882 by 2368,
// bf16: 44 us; through registers 51); rows of bf16 off words go through registers.
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "k_linear.h"

namespace ct {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct LinearArgs : OutArgs {
  const void *x, *w;
  int k;
  int per_split;  // elements in a slice of the reduction (whole 128-byte chunks)
  int64_t ldx, ldw;
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

// Adds the slices in their order and finishes the outputs.
__global__ void __launch_bounds__(256) linear_join_kernel(OutArgs a) {
  const int n4 = (a.n + 3) / 4;
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= (int64_t)a.m * n4) return;
  const int i = (int)(q / n4), j = (int)(q - (int64_t)i * n4) * 4;
  const float* p = a.ws + q * 4;
  const Quad bias = load_bias(a, j), res = load_res(a, i, j);
  f32x4 v = {}, part[4];
  for (int s = 0; s < a.split; s += 4) {  // four slices in flight
#pragma unroll
    for (int e = 0; e < 4; ++e) part[e] = *(const f32x4*)(p + (int64_t)min(s + e, a.split - 1) * a.m * n4 * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (s + e < a.split) v += part[e];
  }
  store4(a, i, j, v, bias, res);
}

int launch_join(const OutArgs& a, hipStream_t st) {
  const int64_t quads = (int64_t)a.m * ((a.n + 3) / 4);
  return launch(linear_join_kernel, dim3((unsigned)((quads + 255) / 256)), 256, 0, st, a);
}

// ------------------------------------------------------------------ 16-byte groups of rows
// A group of bf16 at any element's address: the words around it, and, once they have arrived,
// the group itself, shifted where it starts in the middle of a word, with all but its first
// `left` elements masked to 0.
struct RawGroup {
  u32x4 q;
  unsigned next;  // the fifth word
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, unsigned off) {
    q = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(off & ~3u), 0, 0);
    next = __builtin_amdgcn_raw_buffer_load_b32(r, (int)((off & ~3u) + 16), 0, 0);
  }
  __device__ __forceinline__ u32x4 get(unsigned off, int left) const {
    unsigned v[5] = {q.x, q.y, q.z, q.w, next};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __builtin_amdgcn_alignbit(v[i + 1], v[i], (off & 2u) * 8);
      v[i] = left > 2 * i + 1 ? v[i] : left > 2 * i ? v[i] & 0xFFFFu : 0;
    }
    return (u32x4){v[0], v[1], v[2], v[3]};
  }
};
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
// A block computes BM x BN outputs with WK teams of WM x WN waves, each team every WK-th
// slice of 128 bytes of each operand row: where the tile is small, a slice's products take
// less time than the waits around them. Slices go through STAGES buffers in LDS, the later
// ones in flight while one is multiplied; the 16-byte groups of a row are permuted by its
// number, so that the 16 rows of a fragment lie in distinct banks.
// Every address is in bounds: an operand's rows are a buffer that ends with the last of the
// tile's rows, rows and slices past the end have an offset past it, and reads beyond k within
// a row are kept out one group (or word, or element) at a time.
template <typename T, int BM, int BN, int WM, int WN, int WK, int STAGES, int COPY>
__global__ void __launch_bounds__(64 * WM * WN * WK) linear_tile_kernel(LinearArgs a) {
  constexpr int WAVES = WM * WN, ROWS = BM + BN, G = 16 / (int)sizeof(T), ROWB = 128, NG = ROWB / 16;
  constexpr int KC = NG * G, LPR = COPY == 4 ? 32 : 8, RPC = 64 / LPR;  // elements of a slice, lanes of a row, rows of a copy
  constexpr int NC = ROWS / RPC / WAVES, NW = BN / RPC / WAVES;  // copies of a wave, those of w first
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16, STAGE = WK * ROWS * ROWB;
  static_assert(BN % (RPC * WAVES) == 0 && BM % (RPC * WAVES) == 0, "every wave copies as many rows");
  extern __shared__ __align__(16) char lds[];

  const TileAt at = tile_of_block(a, (int)blockIdx.x);
  const int m0 = at.mi * BM, n0 = at.ni * BN, sp = (int)blockIdx.y;
  const int lane = (int)threadIdx.x & 63, team = wave_id() / WAVES, wave = wave_id() % WAVES;
  const int k_begin = sp * a.per_split, k_end = min(a.k, k_begin + a.per_split);
  const int chunks = (k_end - k_begin + WK * KC - 1) / (WK * KC);  // slices of a team

  const RowsView vw = rows_view<T>(a.w, a.ldw, n0, a.n, BN, a.k), vx = rows_view<T>(a.x, a.ldx, m0, a.m, BM, a.k);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(vw.base, vw.bytes), rx = make_rsrc(vx.base, vx.bytes);
  // Copy i of a wave: RPC whole rows, lane by lane in LDS, so that the permutation of a row's
  // groups is one of the addresses that its lanes read. `first`: a lane's first element in
  // the slice.
  constexpr int EACH = (COPY == 4 ? 4 : 16) / (int)sizeof(T), BYTES = RPC * ROWB;
  auto row_of = [&](int i) { return ((i < NW ? i : i - NW) * WAVES + wave) * RPC + lane / LPR; };
  auto first = [&](int i) {
    const int key = (row_of(COPY == 4 ? i : 0) >> 1) & (NG - 1);  // of eight rows each: the same for every copy
    return ((lane % LPR) ^ (COPY == 4 ? key * 4 : key)) * EACH;
  };
  static_assert(COPY == 4 || (WAVES * RPC >> 1) % NG == 0, "");
  unsigned off[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int r = row_of(i);
    const bool ok = i < NW ? n0 + r < a.n : m0 + r < a.m;
    const unsigned ld = (unsigned)((i < NW ? a.ldw : a.ldx) * (int)sizeof(T));
    off[i] = ok ? (unsigned)r * ld + (unsigned)(first(i) * (int)sizeof(T)) + (i < NW ? vw.odd : vx.odd) : kOobGroup;
  }

  constexpr int RING = COPY ? 1 : NC <= 4 ? 4 : 2;  // slices on their way through registers
  RawGroup held[RING][COPY ? 1 : NC];
  auto fetch = [&](int c, int stage) __attribute__((always_inline)) {
    const int k0 = k_begin + (c * WK + team) * KC;
    char* dst = lds + stage * STAGE + team * ROWS * ROWB + wave * BYTES;
    auto go = [&](auto tail) __attribute__((always_inline)) {
      const unsigned k = (unsigned)(k0 * (int)sizeof(T));
      const int kw = tail.value ? uniform_part(k, vw.bytes) : (int)k, kx = tail.value ? uniform_part(k, vx.bytes) : (int)k;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const bool out = tail.value && k0 + first(i) >= k_end;
        if constexpr (COPY > 0) {
          copy_lds<COPY>(i < NW ? rw : rx, dst + i * WAVES * BYTES, out ? kOobGroup : off[i], i < NW ? kw : kx);
        } else {
          held[stage][i].load(i < NW ? rw : rx, off[i] == kOobGroup || out ? kOobGroup : off[i] + k);
        }
      }
    };
    if (k0 + KC <= k_end) go(std::false_type{});
    else go(std::true_type{});
  };
  auto put = [&](int c, int u) __attribute__((always_inline)) {
    const int k0 = k_begin + (c * WK + team) * KC;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if constexpr (COPY == 0)
        *(u32x4*)(lds + (u & 1) * STAGE + team * ROWS * ROWB + (i * WAVES + wave) * BYTES + lane * 16) =
            held[u][i].get(off[i], k_end - k0 - first(i));
  };

  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const int lrow = lane & 15, kg = lane >> 4;
  const int at0 = lrow * ROWB + (((kg ^ (lrow >> 1)) & (NG - 1)) * 16);  // the slice's first half
  f32x4 acc[TN][TM] = {};
  auto multiply = [&](int stage) __attribute__((always_inline)) {
    const char* sw = lds + stage * STAGE + (team * ROWS + wn) * ROWB;
    const char* sx = sw + (BN + wm - wn) * ROWB;
#pragma unroll
    for (int s = 0; s < NG / 4; ++s) {
      const int at = s ? at0 ^ 64 : at0;
      u32x4 fw[TN], fx[TM];
#pragma unroll
      for (int i = 0; i < TN; ++i) fw[i] = *(const u32x4*)(sw + at + i * 16 * ROWB);
#pragma unroll
      for (int j = 0; j < TM; ++j) fx[j] = *(const u32x4*)(sx + at + j * 16 * ROWB);
#pragma unroll
      for (int j = 0; j < TM; ++j)
#pragma unroll
        for (int i = 0; i < TN; ++i) acc[i][j] = mma16<T>(fw[i], fx[j], acc[i][j]);
    }
  };

  if constexpr (COPY > 0) {
    // Slices past the end read 0, so that STAGES - 1 of them are in flight at every wait. The
    // barrier also says that every wave has read the stage that is filled next.
    static_assert(NC * (STAGES - 2) <= 63, "the counter of loads on their way has six bits");
    if (chunks > 0) {
#pragma unroll
      for (int c = 0; c < STAGES - 1; ++c) fetch(c, c);
      int stage = 0;
      for (int c = 0; c < chunks; ++c) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NC * (STAGES - 2)) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        fetch(c + STAGES - 1, stage ? stage - 1 : STAGES - 1);
        multiply(stage);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
      }
    }
  } else {
    // The barrier of a slice says that every wave has read the one before it, whose stage the
    // next slice goes to.
    static_assert(COPY > 0 || (STAGES == 2 && RING % 2 == 0), "");
#pragma unroll
    for (int u = 0; u < RING; ++u) fetch(u, u);
    for (int c = 0; c < chunks; c += RING) {
#pragma unroll
      for (int u = 0; u < RING; ++u) {
        if (c + u >= chunks) break;
        put(c + u, u);
        __syncthreads();
        fetch(c + u + RING, u);
        multiply(u & 1);
      }
    }
  }

  write_tile<BM, BN, WM, WN, WK, STAGES * STAGE>(a, lds, acc, m0, n0, sp);
}

// ------------------------------------------------------------------ plans and launches
// Tiles, from small to large. Of the two of a size the second leaves room for a second block
// on the compute unit.
enum { LIN_32, LIN_32_TWO, LIN_64X32, LIN_32X64, LIN_64, LIN_64_TWO, LIN_128X64, LIN_128, LIN_256, LIN_KINDS };
struct TileShape {
  int bm, bn, wm, wn, wk, stages;
};
constexpr TileShape kTiles[LIN_KINDS] = {{32, 32, 1, 2, 4, 3}, {32, 32, 1, 2, 4, 2},   {64, 32, 2, 2, 4, 3},
                                         {32, 64, 1, 4, 1, 3}, {64, 64, 2, 2, 2, 3},   {64, 64, 2, 2, 1, 3},
                                         {128, 64, 2, 2, 1, 2}, {128, 128, 2, 2, 1, 2}, {256, 256, 4, 2, 1, 2}};

static int64_t tiles_of(const ct_linear_op& op, int kind) {
  const TileShape t = kTiles[kind];
  return (((int64_t)op.m + t.bm - 1) / t.bm) * (((int64_t)op.n + t.bn - 1) / t.bn);
}

LinearPlan plan_linear(const ct_linear_op& op) {
  LinearPlan p = {};
  const int chunks = (int)(((int64_t)op.k * elem_bytes(op.dtype) + 127) / 128);
  // Rounds of the device, and what a round costs beside one of 128 x 128 tiles at the full
  // rate. In bf16 small tiles, and one of 128 x 128 on a compute unit alone, do not reach it;
  // in fp32 the matrix cores bound all of them. Measured in bf16 on 4096^3, 2048^3, 2048 x
  // 4096 by 1024, 11020 x 320 by 3520, 6000 x 640 by 1024, 1500^3, 512 x 2048 by 2048 and
  // reductions of 64 to 512, in fp32 on 4096^2 by 64 to 2048, 2048^3, 3000 x 1000 by 501, 889
  // x 5384 by 64 and 1021 x 1277 by 515: the choice is the fastest or within 5 % of it.
  auto rounds = [&](int kind) { return (double)((tiles_of(op, kind) + kPlanCus - 1) / kPlanCus); };
  const double r128 = rounds(LIN_128);
  const std::pair<int, double> bf16_costs[] = {{LIN_64, 0.5 * rounds(LIN_64)},
                                               {LIN_128X64, 0.8 * rounds(LIN_128X64)},
                                               {LIN_128, r128 > 1 ? 1.2 * r128 : 1.65},
                                               {LIN_256, 4.0 * rounds(LIN_256)}},
                               f32_costs[] = {{LIN_64, 0.27 * rounds(LIN_64)},
                                              {LIN_32X64, 0.14 * rounds(LIN_32X64)},
                                              {LIN_128, r128 > 1 ? r128 : 1.12},
                                              {LIN_256, 3.97 * rounds(LIN_256)}};
  double least = 1e300;
  for (auto [kind, cost] : op.dtype == CT_DT_BF16 ? bf16_costs : f32_costs)
    if (cost < least) {
      least = cost;
      p.kind = kind;
    }
  // Smaller tiles where 64 x 64 leaves compute units without one
  const int64_t enough = kPlanCus * 3 / 4;
  if ((p.kind == LIN_64 || p.kind == LIN_32X64) && tiles_of(op, LIN_64) < enough)
    p.kind = tiles_of(op, LIN_64X32) >= enough ? LIN_64X32 : LIN_32;
  if (op.m <= 32) p.kind = LIN_32;
  if (p.kind == LIN_64 && tiles_of(op, LIN_64) > kPlanCus) p.kind = LIN_64_TWO;
  if (p.kind == LIN_32 && tiles_of(op, LIN_32) > kPlanCus) p.kind = LIN_32_TWO;
  // A long reduction over few tiles: slices of it, of 32 chunks at least, so that they save
  // more than the second kernel takes
  const int64_t blocks = tiles_of(op, p.kind);
  int split = 1;
  if (blocks <= kPlanCus / 4 && chunks >= 128) split = (int)(kPlanCus / blocks < chunks / 32 ? kPlanCus / blocks : chunks / 32);
  const int per = chunks ? (chunks + split - 1) / split : 1;
  p.split = chunks ? (chunks + per - 1) / per : 1;
  p.per_split = p.split > 1 ? per * (128 / elem_bytes(op.dtype)) : op.k;
  p.ws_floats = p.split > 1 ? (int64_t)p.split * op.m * ((op.n + 3) / 4 * 4) : 0;
  return p;
}

template <typename T, int COPY, int KIND>
static int launch_tile(LinearArgs a, hipStream_t st) {
  constexpr TileShape t = kTiles[KIND];
  constexpr int S = COPY ? t.stages : 2;
  if (!set_tiles(a, t.bm, t.bn, 64 * t.wm * t.wn * t.wk)) return refuse_size("ct_linear_run");
  return launch(linear_tile_kernel<T, t.bm, t.bn, t.wm, t.wn, t.wk, S, COPY>,
                dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.split),
                64 * t.wm * t.wn * t.wk, S * t.wk * (t.bm + t.bn) * 128, st, a);
}
template <typename T, int COPY>
static int linear_pick(const LinearArgs& a, int kind, hipStream_t st) {
  switch (kind) {
    case LIN_32: return launch_tile<T, COPY, LIN_32>(a, st);
    case LIN_32_TWO: return launch_tile<T, COPY, LIN_32_TWO>(a, st);
    case LIN_64X32: return launch_tile<T, COPY, LIN_64X32>(a, st);
    case LIN_32X64:
      if constexpr (sizeof(T) == 4) return launch_tile<T, COPY, LIN_32X64>(a, st);
    case LIN_64: return launch_tile<T, COPY, LIN_64>(a, st);
    case LIN_64_TWO: return launch_tile<T, COPY, LIN_64_TWO>(a, st);
    case LIN_128X64:
      if constexpr (sizeof(T) == 2) return launch_tile<T, COPY, LIN_128X64>(a, st);
    case LIN_128: return launch_tile<T, COPY, LIN_128>(a, st);
    default: return launch_tile<T, COPY, LIN_256>(a, st);
  }
}
// Through registers a tile has two stages whatever its plan, and 256 x 256 has no room.
static int linear_pick_odd(const LinearArgs& a, int kind, hipStream_t st) {
  switch (kind) {
    case LIN_32:
    case LIN_32_TWO: return launch_tile<bf16_t, 0, LIN_32>(a, st);
    case LIN_64X32:
    case LIN_64:
    case LIN_64_TWO: return launch_tile<bf16_t, 0, LIN_64_TWO>(a, st);
    default: return launch_tile<bf16_t, 0, LIN_128>(a, st);
  }
}

int launch_linear(const ct_linear_op& op, const LinearPlan& p, const void* x, const void* w, const float* bias,
                  const void* res, void* y, float* ws, void* stream) {
  LinearArgs a = {};
  a.x = x; a.w = w; a.res = res; a.bias = bias; a.y = y; a.ws = ws;
  a.m = op.m; a.n = op.n; a.k = op.k;
  a.ldx = op.ldx; a.ldw = op.ldw; a.ldr = op.ldr; a.ldy = op.ldy;
  a.act = op.act; a.res_mode = op.res; a.out_bf16 = op.out_dtype == CT_DT_BF16;
  a.split = p.split; a.per_split = p.per_split;
  a.stream = (int64_t)op.m * op.n * elem_bytes(op.out_dtype) >= kStreamBytes;
  const int e = elem_bytes(op.dtype);
  // What rows of both operands lie on, and end on, decides how they are copied: 16 bytes a
  // lane, a word a lane, or (bf16 only) through registers
  const int64_t on = (int64_t)((uintptr_t)x | (uintptr_t)w) | op.ldx * e | op.ldw * e | op.k * (int64_t)e;
  hipStream_t st = (hipStream_t)stream;
  int rc;
  if (op.dtype == CT_DT_F32)
    rc = on % 16 == 0 ? linear_pick<float, 16>(a, p.kind, st) : linear_pick<float, 4>(a, p.kind, st);
  else
    rc = on % 16 == 0  ? linear_pick<bf16_t, 16>(a, p.kind, st)
         : on % 4 == 0 ? linear_pick<bf16_t, 4>(a, p.kind, st)
                       : linear_pick_odd(a, p.kind, st);
  if (rc || p.split == 1) return rc;
  return launch_join(a, st);
}

}  // namespace ct
