// Linear attention with a decay for each head, along packed sequences: with l_t = min(dt_t a, 0)
//   S_t = exp(l_t) S_{t-1} + k_t^T v_t (dt_t),   o_t = scale q_t S_t.
#include <hip/hip_runtime.h>

#include "k_seq.h"

namespace ct {

struct DecayArgs {
  const void *q, *k, *v, *delta;
  const float *dt_bias, *a, *state_in;
  float* state_out;
  void* o;
  SeqView seqs;
  int heads, groups, key, value;
  int delta_bf16, softplus, step_input;
  int stream;  // states go past the caches
  float scale;
  int64_t ldq, ldk, ldv, lddelta, ldo;
  FastDiv dheads, dper;  // by heads, by heads to a group
};

// Step and log2 of the decay of a head at a token. A step or rate that is NaN stays one; below
// 2^-150 the decay is 0 in fp32, and a sum of many such logarithms would lose the small ones.
struct Step {
  float dt, l;
};
__device__ __forceinline__ Step step_of(const DecayArgs& a, int row, int head, float bias, float rate) {
  float dt = 1.f;
  if (a.delta) {
    const int64_t at = row * a.lddelta + head;
    dt = (a.delta_bf16 ? (float)((const bf16_t*)a.delta)[at] : ((const float*)a.delta)[at]) + bias;
    if (a.softplus) dt = softplus_f32(dt);
  }
  float l = dt * rate;
  l = l > 0.f ? 0.f : l;
  l = l < -104.f ? -104.f : l;
  return {dt, l * kLog2e};
}

// ------------------------------------------------------------------ token by token
// A block takes a head of a sequence with its state in registers: LANES lanes of four columns
// each, and 256 / LANES rows at a time. What it reads and writes of the state bounds it: all of it
// is on its way before the first product.
template <typename T, int LANES, int R>
__global__ void __launch_bounds__(256) decay_step_kernel(DecayArgs a) {
  constexpr int RG = 256 / LANES, COLS = LANES * 4;
  const int tid = (int)threadIdx.x, lane = tid % LANES, rg = tid / LANES;
  const int s = fdiv((int)blockIdx.x, a.dheads), head = (int)blockIdx.x - s * a.heads;
  const SeqRange r = seq_range(a.seqs, s);
  const int slot = seq_slot(a.seqs, s);
  const int c0 = (int)blockIdx.y * COLS + lane * 4, left = a.value - c0;
  const int64_t base = ((int64_t)slot * a.heads + head) * a.key * a.value + c0;

  f32x4 st[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int d = rg + i * RG;
    st[i] = f32x4{};
    if (slot < 0 || !a.state_in || d >= a.key) continue;
    const float* p = a.state_in + base + (int64_t)d * a.value;
    if (left >= 4) st[i] = *(const f32x4_any*)p;
    else
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) st[i][e] = p[e];
  }
  __shared__ float qk[2][2][256];
  __shared__ f32x4 part[RG][LANES];
  const int group = fdiv(head, a.dper);
  const float bias = a.dt_bias ? a.dt_bias[head] : 0.f, rate = a.a[head];
  for (int t = r.begin; t < r.end; ++t) {
    float(*now)[256] = qk[(t - r.begin) & 1];
    if (tid < a.key) {
      now[0][tid] = (float)((const T*)a.q)[t * a.ldq + (int64_t)group * a.key + tid];
      now[1][tid] = (float)((const T*)a.k)[t * a.ldk + (int64_t)group * a.key + tid];
    }
    const Step step = step_of(a, t, head, bias, rate);
    f32x4 v = {};
    const T* vp = (const T*)a.v + t * a.ldv + (int64_t)head * a.value + c0;
    if (left >= 4) {
      const Quad q = load_quad4(vp);
      v = (f32x4){q.v[0], q.v[1], q.v[2], q.v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) v[e] = (float)vp[e];
    }
    if (a.step_input) v *= step.dt;
    const float decay = __builtin_amdgcn_exp2f(step.l);
    __syncthreads();  // q and k are there, and the sums of the token before have been read
    f32x4 acc = {};
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int d = rg + i * RG;
      if (d < a.key) {
        const float kd = now[1][d], qd = now[0][d];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float h = fmaf(kd, v[e], decay * st[i][e]);
          st[i][e] = h;
          acc[e] = fmaf(qd, h, acc[e]);
        }
      }
    }
    part[rg][lane] = acc;
    __syncthreads();
    if (tid < COLS && (int)blockIdx.y * COLS + tid < a.value) {
      float o = 0;
#pragma unroll
      for (int g = 0; g < RG; ++g) o += part[g][tid / 4][tid % 4];
      ((T*)a.o)[t * a.ldo + (int64_t)head * a.value + (int)blockIdx.y * COLS + tid] = from_f32<T>(o * a.scale);
    }
  }
  if (slot < 0 || !a.state_out) return;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int d = rg + i * RG;
    if (d >= a.key) break;
    float* p = a.state_out + base + (int64_t)d * a.value;
    if (left >= 4) store_once((f32x4_any*)p, st[i], a.stream);
    else
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) p[e] = st[i][e];
  }
}

template <typename T, int LANES>
static int decay_step_rows(const DecayArgs& a, dim3 blocks, hipStream_t st) {
  constexpr int RG = 256 / LANES;
  if (a.key <= 4 * RG) return launch(decay_step_kernel<T, LANES, 4>, blocks, 256, 0, st, a);
  if constexpr (RG * 4 < 256)
    if (a.key <= 8 * RG) return launch(decay_step_kernel<T, LANES, 8>, blocks, 256, 0, st, a);
  if constexpr (RG * 8 < 256)
    if (a.key <= 16 * RG) return launch(decay_step_kernel<T, LANES, 16>, blocks, 256, 0, st, a);
  if constexpr (RG * 16 < 256) return launch(decay_step_kernel<T, LANES, 32>, blocks, 256, 0, st, a);
  return -1;
}
template <typename T>
static int decay_step(const DecayArgs& a, hipStream_t st) {
  const int64_t blocks = (int64_t)a.seqs.count * a.heads;
  const int lanes = a.value <= 32 ? 8 : a.value <= 64 ? 16 : 32;
  const int cols = (a.value + 4 * lanes - 1) / (4 * lanes);
  if (!fits_launch(blocks * cols, 256)) return refuse_size("ct_decay_attention_run");
  const dim3 grid((unsigned)blocks, (unsigned)cols);
  return lanes == 8    ? decay_step_rows<T, 8>(a, grid, st)
         : lanes == 16 ? decay_step_rows<T, 16>(a, grid, st)
                       : decay_step_rows<T, 32>(a, grid, st);
}

DecayPlan plan_decay(const ct_decay_attention_op&, const ct_sequences&) { return {}; }

int launch_decay(const ct_decay_attention_op& op, const DecayPlan&, const SeqView& s, const DecayArrays& v, int,
                 void* stream) {
  DecayArgs a = {};
  a.q = v.q; a.k = v.k; a.v = v.v; a.delta = v.delta; a.dt_bias = v.dt_bias; a.a = v.a;
  a.state_in = v.state_in; a.state_out = v.state_out; a.o = v.o; a.seqs = s;
  a.heads = op.heads; a.groups = op.groups; a.key = op.key_dim; a.value = op.value_dim;
  a.delta_bf16 = op.delta_dtype == CT_DT_BF16; a.softplus = op.softplus; a.step_input = op.step_input;
  a.scale = op.scale;
  a.ldq = op.ldq; a.ldk = op.ldk; a.ldv = op.ldv; a.lddelta = op.lddelta; a.ldo = op.ldo;
  a.dheads = make_fastdiv(op.heads);
  a.dper = make_fastdiv(op.heads / op.groups);
  a.stream = (int64_t)s.count * op.heads * op.key_dim * op.value_dim * 4 >= kStreamStateBytes;
  return op.dtype == CT_DT_BF16 ? decay_step<bf16_t>(a, (hipStream_t)stream) : decay_step<float>(a, (hipStream_t)stream);
}

}  // namespace ct
