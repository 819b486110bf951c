// Root-mean-square norm of rows, or of the parts of a row:
//   h = x + res,   y = h / sqrt(mean h^2 + eps) * w * silu(z).
//
// The bytes bound it: every input is read once and kept in registers, eight elements a lane and
// step, while the squares are summed across the part's lanes, and rows of 8 or 4 bits are made
// from the same registers. 8192 rows of 32 gated bf16 parts of 128 to 8 bits take 32.5 us, 5.2 TB/s
// (a copy reaches 5.4). Parts of whole groups of eight have a kernel without the checks of single
// elements (40 us with them, a vector ALU as busy as the memory), and everything is asked for
// before the first value is looked at (36.8 us with the weights behind the gate).
#include <hip/hip_runtime.h>

#include "k_mx.h"

namespace ct {

struct NormArgs {
  const void *x, *res, *z;
  const float* w;
  void *sum, *y;
  unsigned char* scales;
  int units;  // parts in all
  int cols, part;  // columns of a row, of a part
  float eps, inv;  // 1 / part
  int64_t ldx, ldres, ldsum, ldz, ldy, lds;
  FastDiv groups;
};

enum { NORM_F32 = CT_DT_F32, NORM_BF16 = CT_DT_BF16, NORM_MX8 = CT_MX_E4M3, NORM_MX4 = CT_MX_E2M1 };

template <int CTRL>
__device__ __forceinline__ float lane_perm(float v) {
  return __builtin_bit_cast(float, quad_perm<CTRL>(__builtin_bit_cast(unsigned, v)));
}
// The sum over the TEAM lanes (a power of two up to 64), or over a block of four waves.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v) {
  // the other lane of a pair, of four, of eight (mirrored), of sixteen: both sides add the same two numbers
  v += lane_perm<0xB1>(v);
  v += lane_perm<0x4E>(v);
  v += lane_perm<0x141>(v);
  if constexpr (TEAM > 8) v += lane_perm<0x140>(v);
  if constexpr (TEAM > 16) v += __shfl_xor(v, 16);
  if constexpr (TEAM > 32) v += __shfl_xor(v, 32);
  if constexpr (TEAM > 64) {
    __shared__ float part[TEAM / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < TEAM / 64; ++i) v += part[i];
  }
  return v;
}

// A team of TEAM lanes to a part, STEPS octs a lane in registers; STEPS = 0: as many as it takes,
// read again for the outputs.
template <typename T, int OUT, int TEAM, int STEPS, bool EVEN>
__global__ void __launch_bounds__(256) norm_kernel(NormArgs a) {
  constexpr int TEAMS = 256 / TEAM, S = STEPS ? STEPS : 1;
  const int unit = (int)blockIdx.x * TEAMS + (int)threadIdx.x / TEAM;  // below 2^31: units are, in whole blocks
  const bool mine = unit < a.units;
  const int row = mine ? fdiv(unit, a.groups) : 0, first = mine ? (unit - row * a.groups.d) * a.part : 0;
  const int lane = (int)threadIdx.x % TEAM, part = mine ? a.part : 0;
  const T* x = (const T*)a.x + row * a.ldx + first;
  const T* res = (const T*)a.res + row * a.ldres + first;
  const T* z = (const T*)a.z + row * a.ldz + first;
  T* sum = (T*)a.sum + row * a.ldsum + first;
  const float* w = a.w + first;
  const auto col = [&](int s) { return (s * TEAM + lane) * 8; };

  const auto load = [](auto& q, const auto* p, int left) __attribute__((always_inline)) {
    if constexpr (EVEN) q.load(p);
    else load_oct(q, p, left);
  };
  const auto store = [](auto* p, const float* v, int left) __attribute__((always_inline)) {
    store_oct(p, v, EVEN ? 8 : left);
  };

  float h[S][8];
  RawOct<T> gate[S];
  RawOct<float> weight[S];
  const auto values = [&](const RawOct<T>& q, const RawOct<T>& r, float* v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q.at(i);
    if (a.res) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r.at(i);
    }
  };
  const auto read = [&](int c, float* v) __attribute__((always_inline)) {
    RawOct<T> q = {}, r = {};
    if (c < part) load(q, x + c, part - c);
    if (a.res && c < part) load(r, res + c, part - c);
    values(q, r, v);
  };
  float ss = 0;
  if constexpr (STEPS > 0) {
    // everything is asked for before the first value is looked at: one latency, not three
    RawOct<T> q[S], r[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      q[s] = {}; r[s] = {}; gate[s] = {}; weight[s] = {};
      if (col(s) < part) {
        if (S <= 2 && a.w) load(weight[s], w + col(s), part - col(s));
        load(q[s], x + col(s), part - col(s));
        if (a.res) load(r[s], res + col(s), part - col(s));
        if (a.z) load(gate[s], z + col(s), part - col(s));
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      values(q[s], r[s], h[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(h[s][i], h[s][i], ss);
    }
  } else {
    for (int s = 0; col(s) < part; ++s) {
      read(col(s), h[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(h[0][i], h[0][i], ss);
    }
  }
  ss = team_sum<TEAM>(ss);
  // sqrt and the division are rounded to nearest: one call a part's lanes
  const float scale = 1.f / __builtin_sqrtf(fmaf(ss, a.inv, a.eps));

  const auto write = [&](int c, const float* v, const RawOct<T>& g, RawOct<float>& wq) __attribute__((always_inline)) {
    const int left = part - c;
    if (a.sum && left > 0) store(sum + c, v, left);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v[i] * scale;
    if (a.w) {
      if ((STEPS == 0 || S > 2) && left > 0) load(wq, w + c, left);  // more steps: no registers to keep them in
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] *= wq.at(i);
    }
    if (a.z) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] *= silu_f32(g.at(i));
    }
    if constexpr (OUT == NORM_F32) {
      if (left > 0) store((float*)a.y + row * a.ldy + first + c, y, left);
    } else if constexpr (OUT == NORM_BF16) {
      if (left > 0) store((bf16_t*)a.y + row * a.ldy + first + c, y, left);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = i < (EVEN ? 8 * (left > 0) : left) ? y[i] : 0.f;  // also where 0 met an infinite scale
      // lanes behind the part have nothing to write: behind the row's last block, or of the next part
      mx_store<OUT>(y, (char*)a.y + row * a.ldy, a.scales + row * a.lds,
                    c < (part + kMxBlock - 1) / kMxBlock * kMxBlock ? first + c : kNoColumn, a.cols);
    }
  };
  if constexpr (STEPS > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) write(col(s), h[s], gate[s], weight[s]);
  } else {
    for (int s = 0; s * TEAM * 8 < part; ++s) {  // every lane, for the blocks' sake
      read(col(s), h[0]);
      gate[0] = {};
      if (a.z && col(s) < part) load(gate[0], z + col(s), part - col(s));
      weight[0] = {};
      write(col(s), h[0], gate[0], weight[0]);
    }
  }
}

template <typename T, int OUT, int TEAM, int STEPS>
static int norm_go(const NormArgs& a, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.units + 256 / TEAM - 1) / (256 / TEAM);
  if (!fits_launch(blocks, 256)) return refuse_size("ct_norm_run");
  return a.part % 8 ? launch(norm_kernel<T, OUT, TEAM, STEPS, false>, dim3((unsigned)blocks), 256, 0, st, a)
                    : launch(norm_kernel<T, OUT, TEAM, STEPS, true>, dim3((unsigned)blocks), 256, 0, st, a);
}
template <typename T, int OUT>
static int norm_pick(const NormArgs& a, hipStream_t st) {
  const int octs = a.part / 8 + (a.part % 8 != 0);
  if (octs <= 8) return norm_go<T, OUT, 8, 1>(a, st);
  if (octs <= 16) return norm_go<T, OUT, 16, 1>(a, st);
  if (octs <= 32) return norm_go<T, OUT, 32, 1>(a, st);
  if (octs <= 64) return norm_go<T, OUT, 64, 1>(a, st);
  if (octs <= 256) return norm_go<T, OUT, 256, 1>(a, st);
  if (octs <= 512) return norm_go<T, OUT, 256, 2>(a, st);
  if (octs <= 1024) return norm_go<T, OUT, 256, 4>(a, st);
  if (octs <= 2048) return norm_go<T, OUT, 256, 8>(a, st);
  return norm_go<T, OUT, 256, 0>(a, st);
}
template <typename T>
static int norm_out(const NormArgs& a, int out, hipStream_t st) {
  switch (out) {
    case NORM_F32: return norm_pick<T, NORM_F32>(a, st);
    case NORM_BF16: return norm_pick<T, NORM_BF16>(a, st);
    case NORM_MX8: return norm_pick<T, NORM_MX8>(a, st);
    default: return norm_pick<T, NORM_MX4>(a, st);
  }
}

int launch_norm(const ct_norm_op& op, const void* x, const void* res, void* sum, const float* w, const void* z, void* y,
                void* scales, void* stream) {
  const int64_t units = (int64_t)op.rows * op.groups;
  if (units > 0x7FFFFFFF - 256) return refuse_size("ct_norm_run");
  NormArgs a = {};
  a.x = x; a.res = res; a.z = z; a.w = w; a.sum = sum; a.y = y; a.scales = (unsigned char*)scales;
  a.units = (int)units;
  a.cols = op.cols; a.part = op.cols / op.groups;
  a.eps = op.eps; a.inv = 1.f / (float)a.part;
  a.ldx = op.ldx; a.ldres = op.ldres; a.ldsum = op.ldsum; a.ldz = op.ldz; a.ldy = op.ldy; a.lds = op.lds;
  a.groups = make_fastdiv(op.groups);
  return op.dtype == CT_DT_BF16 ? norm_out<bf16_t>(a, op.out, (hipStream_t)stream)
                                : norm_out<float>(a, op.out, (hipStream_t)stream);
}

}  // namespace ct
