// Selective state space scan over packed sequences.
//   h_t[n] = exp(dt_t a[n]) h_{t-1}[n] + dt_t u_t b_t[n],  y_t = (c_t . h_t + d u_t) silu(z_t)
//
// A lane holds NS states of one channel in fp32 registers and walks the tokens of a
// sequence; P neighbouring lanes share a channel where it has more than NS states.
#include <hip/hip_runtime.h>

#include "k_seq.h"

namespace ct {

struct ScanArgs {
  SeqView s;
  const void *u, *delta, *b, *c, *z;
  const float *dt_bias, *a, *d_skip, *state_in;
  float* state_out;
  void* y;
  int64_t ldu, lddelta, ldb, ldc, ldz, ldy;
  int channels, states, per_group, softplus;
  FastDiv dtiles, dgroup;  // channel tiles in all, and of one group
};

template <typename T, int NS, int P>
__global__ void __launch_bounds__(256) scan_kernel(ScanArgs a) {
  constexpr int CH = 64 / P;  // channels of a wave, all of one group
  const int64_t g = (int64_t)blockIdx.x * 4 + wave_id();
  if (g >= (int64_t)a.s.count * a.dtiles.d) return;
  const int s = fdiv((int)g, a.dtiles), tile = (int)g - s * a.dtiles.d;
  const int group = fdiv(tile, a.dgroup), in_group = (tile - group * a.dgroup.d) * CH;
  const int lane = (int)(threadIdx.x & 63), part = lane % P, ch = in_group + lane / P;
  if (ch >= a.per_group) return;
  const int d = group * a.per_group + ch, n0 = part * NS;
  const SeqRange r = seq_range(a.s, s);
  const int slot = seq_slot(a.s, s);

  float h[NS], la[NS];
  const int64_t at = ((int64_t)slot * a.channels + d) * a.states + n0;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const bool in = n0 + i < a.states;
    h[i] = in && slot >= 0 && a.state_in ? a.state_in[at + i] : 0.f;
    la[i] = in ? a.a[(int64_t)d * a.states + n0 + i] * kLog2e : 0.f;
  }
  const float bias = a.dt_bias ? a.dt_bias[d] : 0.f, skip = a.d_skip ? a.d_skip[d] : 0.f;
  const int64_t gn = (int64_t)group * a.states + n0;
  for (int t = r.begin; t < r.end; ++t) {
    float dt = (float)((const T*)a.delta)[t * a.lddelta + d] + bias;
    if (a.softplus) dt = softplus_f32(dt);
    const float u = (float)((const T*)a.u)[t * a.ldu + d], du = dt * u;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const bool in = n0 + i < a.states;
      const float b = in ? (float)((const T*)a.b)[t * a.ldb + gn + i] : 0.f;
      const float c = in ? (float)((const T*)a.c)[t * a.ldc + gn + i] : 0.f;
      h[i] = fmaf(__builtin_amdgcn_exp2f(dt * la[i]), h[i], du * b);
      y = fmaf(c, h[i], y);
    }
#pragma unroll
    for (int m = 1; m < P; m *= 2) y += __shfl_xor(y, m, 64);
    y = fmaf(skip, u, y);
    if (a.z) y *= silu_f32((float)((const T*)a.z)[t * a.ldz + d]);
    if (part == 0) ((T*)a.y)[t * a.ldy + d] = from_f32<T>(y);
  }
  if (slot >= 0 && a.state_out)
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (n0 + i < a.states) a.state_out[at + i] = h[i];
}

ScanPlan plan_scan(const ct_scan_op&, const ct_sequences&) { return {0, 0, 0}; }

template <typename T, int NS, int P>
static int scan_launch(ScanArgs a, hipStream_t st) {
  constexpr int CH = 64 / P;
  const int per = (a.per_group + CH - 1) / CH;
  const int64_t tiles = (int64_t)per * (a.channels / a.per_group), waves = tiles * a.s.count;
  if (waves > 0x7FFFFFFF) return refuse_size("ct_scan_run");
  a.dgroup = make_fastdiv(per);
  a.dtiles = make_fastdiv(tiles);
  hipLaunchKernelGGL((scan_kernel<T, NS, P>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}
template <typename T>
static int scan_pick(const ScanArgs& a, hipStream_t st) {
  if (a.states <= 16) return scan_launch<T, 4, 4>(a, st);
  if (a.states <= 32) return scan_launch<T, 4, 8>(a, st);
  if (a.states <= 64) return scan_launch<T, 8, 8>(a, st);
  if (a.states <= 128) return scan_launch<T, 8, 16>(a, st);
  return scan_launch<T, 16, 16>(a, st);
}

int launch_scan(const ct_scan_op& op, const ScanPlan&, const SeqView& s, const ScanArrays& v, void* stream) {
  ScanArgs a = {};
  a.s = s;
  a.u = v.u; a.delta = v.delta; a.b = v.b; a.c = v.c; a.z = v.z;
  a.dt_bias = v.dt_bias; a.a = v.a; a.d_skip = v.d_skip; a.state_in = v.state_in;
  a.state_out = v.state_out; a.y = v.y;
  a.ldu = op.ldu; a.lddelta = op.lddelta; a.ldb = op.ldb; a.ldc = op.ldc; a.ldz = op.ldz; a.ldy = op.ldy;
  a.channels = op.channels; a.states = op.states; a.per_group = op.channels / op.groups; a.softplus = op.softplus;
  return op.dtype == CT_DT_BF16 ? scan_pick<bf16_t>(a, (hipStream_t)stream)
                                : scan_pick<float>(a, (hipStream_t)stream);
}

}  // namespace ct
