// Root-mean-square norm of rows, or of the parts of a row:
//   h = x + res,   y = h / sqrt(mean h^2 + eps) * w * silu(z).
//
// The bytes bound it: every input is read once and kept in registers, eight elements a lane and
// step, while the squares are summed across the part's lanes, and rows of 8 or 4 bits are made
// from the same registers. 8192 rows of 32 gated bf16 parts of 128 to 8 bits take 35 us, 4.8 TB/s
// (a copy reaches 5.4), with a vector ALU as busy as the memory. Parts of whole groups of eight have a
// kernel without the checks of single elements (7 us less), and everything is asked for before the first
// value is looked at (4 us less than with the weights behind the gate).
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
  float eps;
  double inv;  // 1 / part
  int64_t ldx, ldres, ldsum, ldz, ldy, lds;
  FastDiv groups;
  double terms[12];  // ln(2)^k / k!, where outputs are of 8 or 4 bits
};

enum { NORM_F32 = CT_DT_F32, NORM_BF16 = CT_DT_BF16, NORM_MX8 = CT_MX_E4M3, NORM_MX4 = CT_MX_E2M1 };

template <int CTRL>
__device__ __forceinline__ double lane_perm(double v) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, (u32x2){quad_perm<CTRL>(w.x), quad_perm<CTRL>(w.y)});
}
// The sum over the TEAM lanes (a power of two up to 64), or over a block of four waves.
template <int TEAM>
__device__ __forceinline__ double team_sum(double v) {
  // the other lane of a pair, of four, of eight (mirrored), of sixteen: both sides add the same two numbers
  v += lane_perm<0xB1>(v);
  v += lane_perm<0x4E>(v);
  v += lane_perm<0x141>(v);
  if constexpr (TEAM > 8) v += lane_perm<0x140>(v);
  if constexpr (TEAM > 16) v += __shfl_xor(v, 16);
  if constexpr (TEAM > 32) v += __shfl_xor(v, 32);
  if constexpr (TEAM > 64) {
    __shared__ double part[TEAM / 64];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < TEAM / 64; ++i) v += part[i];
  }
  return v;
}

// 1 / sqrt(v): the instruction's about 23 bits, and a correction of third order in what they leave. 0 of an
// infinite v; NaN of 0, which 0 over it is as well.
__device__ __forceinline__ double rsqrt_f64(double v) {
  const double y = __builtin_amdgcn_rsq(v), e = fma(-v * y, y, 1.);
  return v == __builtin_inf() ? 0. : fma(y * e, fma(e, 0.375, 0.5), y);
}

// ---- outputs of 8 and 4 bits ----
// What is a unit of fp32 off moves an element beside the middle of two by a whole step, and a largest value
// beside a power of two takes another scale: of 33 million gated outputs a few dozen, which alone are
// 6e-5 of the result. So a lane's values are rounded from both ends of what their errors allow, and where
// the two disagree (one wave in 70 for e4m3) the wave computes its values again in fp64.
//
// The error of h * scale * w * silu(z) in units of 2^-24: 1 of the scale, 1 of each product, and of the
// gate 2 |z| of the exponential's argument and 7 (the exponential 2, 1 + e 1, the reciprocal 2, products 2);
// |z| counts where it is below 0, as e / (1 + e) |z| < 0.3 otherwise. 3 more for the ends themselves.
constexpr float kUnit = 5.9604645e-8f;
constexpr float kLowestGate = -80.f;  // below it the exponential is near the end of its range
__device__ __forceinline__ float norm_error(const float* z, bool gate) {
  if (!gate) return 8 * kUnit;
  float low = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) low = fminf(low, z[i]);
  return low < kLowestGate ? 1.f : fmaf(low, -2.25f * kUnit, 16 * kUnit);
}
// The nearest float towards 0, its last bit set where that is not d itself: rounded again to a few bits it
// gives what d would.
__device__ __forceinline__ float round_odd(double d) {
  const float f = (float)d;
  if (!(__builtin_fabsf(f) < __builtin_inff()) || (double)f == d) return f;
  const unsigned bits = __builtin_bit_cast(unsigned, f);
  return __builtin_bit_cast(float, (__builtin_fabs((double)f) > __builtin_fabs(d) ? bits - 1 : bits) | 1u);
}

// 1 / (1 + e^-z) in fp64: 2^t by its series around the nearest whole t, of 12 terms 2^-46 of it. The terms
// are arguments of the kernel, so that they wait in scalar registers and not in the vector ones that every
// wave would need for them.
constexpr int kExpTerms = 12;
__device__ __forceinline__ double logistic_f64(double z, const double* terms) {
  const double t = fmin(fmax(z * -1.4426950408889634, -1100.), 1100.), n = rint(t), f = t - n;
  double p = terms[kExpTerms - 1];
#pragma unroll
  for (int k = kExpTerms - 2; k >= 0; --k) p = fma(p, f, terms[k]);
  return 1. / (1. + ldexp(p, (int)n));
}

// A team of TEAM lanes to a part, STEPS octs a lane in registers; STEPS = 0: as many as it takes,
// read again for the outputs.
template <typename T, int OUT, int TEAM, int STEPS, bool EVEN>
__global__ void __launch_bounds__(256) norm_kernel(NormArgs a) {
  constexpr int TEAMS = 256 / TEAM, S = STEPS ? STEPS : 1;
  // a wave's lanes are of one team where teams are waves and more: their row's arithmetic is the scalar ALU's
  const int team = TEAM < 64 ? (int)threadIdx.x / TEAM : __builtin_amdgcn_readfirstlane((int)threadIdx.x / TEAM);
  const int unit = (int)blockIdx.x * TEAMS + team;  // below 2^31: units are, in whole blocks
  const bool mine = unit < a.units;
  int row = mine ? unit : 0, first = 0;
  if (a.groups.d > 1) {
    row = fdiv(row, a.groups);
    first = mine ? (unit - row * a.groups.d) * a.part : 0;
  }
  const int lane = (int)threadIdx.x % TEAM, part = mine ? a.part : 0;
  // Where the part starts in an array; pitches are at most 2^31: one product of 32 by 32 bits, not three
  const auto at = [&](int64_t ld) { return (int64_t)((uint64_t)(unsigned)row * (unsigned)ld); };
  const T* x = (const T*)a.x + at(a.ldx) + first;
  const auto res = [&] { return (const T*)a.res + at(a.ldres) + first; };
  const auto z_row = [&] { return (const T*)a.z + at(a.ldz) + first; };
  const float* w = a.w + first;
  const auto col = [&](int s) { return (s * TEAM + lane) * 8; };

  // Eight elements of column c on. Lanes behind an even part read its first eight (of row 0 where they have no
  // part), which values() turns to 0; of the others' they read what exists.
  const bool whole = STEPS > 0 && a.part == TEAM * STEPS * 8 && a.units - (int)blockIdx.x * TEAMS >= TEAMS;
  const auto load = [&](auto& q, const auto* p, int c) __attribute__((always_inline)) {
    if constexpr (EVEN) {
      q.load(p + (whole || c < part ? c : 0));
    } else {
      q = {};
      if (c < part) load_oct(q, p + c, part - c);
    }
  };
  const auto store = [](auto* p, const float* v, int left) __attribute__((always_inline)) {
    store_oct(p, v, EVEN ? 8 : left);
  };

  float h[S][8];
  RawOct<T> gate[S];
  RawOct<float> weight[S];
  // The empty asm statements keep a branch that the whole launch takes alike from becoming both its sides
  // and a choice of each result.
  const auto values = [&](int c, const RawOct<T>& q, const RawOct<T>& r, float* v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q.at(i);
    if (a.res) {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r.at(i);
    }
    if (EVEN && !whole) {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c < part ? v[i] : 0.f;
    }
  };
  const auto read = [&](int c, float* v) __attribute__((always_inline)) {
    RawOct<T> q, r;
    load(q, x, c);
    if (a.res) load(r, res(), c);
    values(c, q, r, v);
  };
  const auto squares = [](const float* v) __attribute__((always_inline)) {  // of four chains, not one
    double sq[4] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) sq[i % 4] = fma((double)v[i], (double)v[i], sq[i % 4]);
    return (sq[0] + sq[1]) + (sq[2] + sq[3]);
  };
  double ss = 0;
  if constexpr (STEPS > 0) {
    // everything is asked for before the first value is looked at: one latency, not three
    RawOct<T> q[S], r[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (S <= 2 && a.w) load(weight[s], w, col(s));
      load(q[s], x, col(s));
      if (a.res) load(r[s], res(), col(s));
      if (a.z) load(gate[s], z_row(), col(s));
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      values(col(s), q[s], r[s], h[s]);
      ss += squares(h[s]);
    }
  } else {
    for (int s = 0; col(s) < part; ++s) {
      read(col(s), h[0]);
      ss += squares(h[0]);
    }
  }
  ss = team_sum<TEAM>(ss);
  const double scale64 = rsqrt_f64(fma(ss, a.inv, (double)a.eps));
  const float scale = (float)scale64;
  const auto scaled = [&](const float* v, float* y) __attribute__((always_inline)) {
    if (a.eps == 0.f) {  // a part of tiny values may have a scale past fp32: it is lifted first, exactly
      asm volatile("");
      const bool tiny = scale64 > 0x1p100;
      const float lift = tiny ? 0x1p100f : 1.f, rest = tiny ? (float)(scale64 * 0x1p-100) : scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = v[i] * lift * rest;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = v[i] * scale;
    }
  };

  // Eight outputs of 8 or 4 bits with their block's scale. Lanes behind the part have nothing to write:
  // behind the row's last block, or of the next part.
  const auto put = [&](int c, u32x2 q, unsigned e) __attribute__((always_inline)) {
    if (mine && c < (a.part + kMxBlock - 1) / kMxBlock * kMxBlock)
      mx_write<OUT>(q, e, (char*)a.y + at(a.ldy), a.scales + at(a.lds), (unsigned)(first + c), a.cols);
  };
  const auto cut = [&](int c, float* y) __attribute__((always_inline)) {  // also where 0 met an infinite scale
    if (a.part % kMxBlock == 0) return;  // no lane behind the part has a block with one that is not
    asm volatile("");
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = i < (EVEN ? 8 * (part > c) : part - c) ? y[i] : 0.f;
  };
  // Eight outputs; true where they are of 8 or 4 bits and one of the wave's is too near to a border.
  const auto write = [&](int c, const float* v, const RawOct<T>& g, RawOct<float>& wq) __attribute__((always_inline)) {
    const int left = part - c;
    float y[8], z[8];
    scaled(v, y);
    if (a.w) {
      asm volatile("");
      if (STEPS == 0 || S > 2) load(wq, w, c);  // more steps: no registers to keep them in
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] *= wq.at(i);
    }
    if (a.z) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[i] = g.at(i);
        y[i] *= silu_f32(z[i]);
      }
    }
    if constexpr (OUT == NORM_F32) {
      if (left > 0) store((float*)a.y + at(a.ldy) + first + c, y, left);
      return false;
    } else if constexpr (OUT == NORM_BF16) {
      if (left > 0) store((bf16_t*)a.y + at(a.ldy) + first + c, y, left);
      return false;
    } else {
      cut(c, y);
      const float error = norm_error(z, a.z), less = 1.f - error, more = 1.f + error;
      const unsigned largest = mx_largest(y), e = mx_scale<OUT>(largest);
      // the exponents of largest * less and of largest * more, as steps of its last bit, rounded up
      const unsigned reach = (unsigned)fmaf(error, 16777216.f, 1.f), low = largest - min(reach, largest);
      const u32x2 q = mx_elements<OUT>(y, mx_inverse(e) * less), top = mx_elements<OUT>(y, mx_inverse(e) * more);
      put(c, q, e);
      return __ballot(q.x != top.x || q.y != top.y || (low ^ (largest + reach)) >> 23 || error > 0.5f) != 0;
    }
  };
  // The same in fp64 from what is in memory still, over what write() left.
  const auto again = [&](int c) __attribute__((always_inline)) {
    float v[8], y[8];
    RawOct<T> g;
    RawOct<float> wq;
    read(c, v);
    if (a.w) load(wq, w, c);
    if (a.z) load(g, z_row(), c);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double d = (double)v[i] * scale64;
      if (a.w) d *= (double)wq.at(i);
      if (a.z) d *= (double)g.at(i) * logistic_f64((double)g.at(i), a.terms);
      y[i] = round_odd(d);
      __builtin_amdgcn_sched_barrier(0);  // one at a time, for the registers' sake
    }
    cut(c, y);
    const unsigned e = mx_scale<OUT>(mx_largest(y));
    put(c, mx_elements<OUT>(y, mx_inverse(e)), e);
  };
  // after the outputs, which may need x and res again: sum may be one of them
  const auto keep = [&](int c, const float* v) __attribute__((always_inline)) {
    if (a.sum && c < part) store((T*)a.sum + at(a.ldsum) + first + c, v, part - c);
  };
  if constexpr (STEPS > 0) {
    unsigned near = 0;  // a bit a step
#pragma unroll
    for (int s = 0; s < S; ++s) near |= (unsigned)write(col(s), h[s], gate[s], weight[s]) << s;
    if constexpr (OUT == NORM_MX8 || OUT == NORM_MX4) {
#pragma unroll 1
      for (; near; near &= near - 1) again(col(__builtin_ctz(near)));
    }
#pragma unroll
    for (int s = 0; s < S; ++s) keep(col(s), h[s]);
  } else {
    for (int s = 0; s * TEAM * 8 < part; ++s) {  // every lane, for the blocks' sake
      read(col(s), h[0]);
      if (a.z) load(gate[0], z_row(), col(s));
      const bool near = write(col(s), h[0], gate[0], weight[0]);
      if constexpr (OUT == NORM_MX8 || OUT == NORM_MX4) {
        if (near) again(col(s));
      }
      keep(col(s), h[0]);
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
  a.eps = op.eps; a.inv = 1. / (double)a.part;
  a.ldx = op.ldx; a.ldres = op.ldres; a.ldsum = op.ldsum; a.ldz = op.ldz; a.ldy = op.ldy; a.lds = op.lds;
  a.groups = make_fastdiv(op.groups);
  double term = 1;
  for (int k = 0; k < kExpTerms; ++k, term *= 0.6931471805599453 / k) a.terms[k] = term;
  return op.dtype == CT_DT_BF16 ? norm_out<bf16_t>(a, op.out, (hipStream_t)stream)
                                : norm_out<float>(a, op.out, (hipStream_t)stream);
}

}  // namespace ct
