// Causal depthwise convolution along the tokens of packed sequences, its history in slots.
//   y[t,c] = act(bias[c] + sum_{j<W} w[c,j] x[t-W+1+j, c])
//
// A wave computes a tile of U (8; fewer for small calls) consecutive tokens of one sequence for
// 64 lanes of VEC channels. All U + W - 1 rows that it reads are in flight before the first product,
// and each output is W multiply-adds in fp32 in the order of j. The W - 1 rows before the
// tile are read again by it (from the caches: they were read by the tile before).
// Bound by memory: 8192 x 4096 tokens and channels of bf16 in and out (134 MB) 35 us, 3.9
// TB/s, and 4.9 at four times as many (a copy of 1 GiB: 5.1); the SiLU is 8 % of it, which the
// loads do not hide. Tiles of 16 tokens keep fewer waves on a SIMD (36 us); the weights read
// by every wave for itself instead of once a block through LDS made no difference there, and of
// single tokens were 0.3 us faster for 32 sequences of 2048 channels and 1.7 us (13 %) slower
// for 256 of 8192.
// The tile that starts a sequence alone reads its history, and alone writes the new one,
// after that: in place needs no more than the order of a lane's own accesses.
#include <hip/hip_runtime.h>

#include "k_seq.h"

namespace ct {

struct ConvArgs {
  SeqView s;
  const void* x;
  const float *w, *bias;
  const void* state_in;
  void *state_out, *y;
  int64_t ldx, ldy;
  int channels, act, per, tiles;
  int stream;       // y goes past the caches
  FastDiv dblocks;  // waves across the channels
};

// VEC elements at p: one 16-byte access, or a single element.
template <typename T, int VEC>
struct Pack {
  static constexpr int WORDS = VEC == 1 ? 1 : VEC * (int)sizeof(T) / 4;
  unsigned q[WORDS];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC == 1) {
      q[0] = sizeof(T) == 4 ? *(const unsigned*)p : *(const unsigned short*)p;
    } else {
      const u32x4 v = *(const u32x4*)p;
      const unsigned a = v.x, b = v.y, c = v.z, d = v.w;
      q[0] = a; q[1] = b; q[2] = c; q[3] = d;
    }
  }
  __device__ __forceinline__ void store(T* p, bool stream) const {
    if constexpr (VEC == 1) {
      if constexpr (sizeof(T) == 4) *(unsigned*)p = q[0];
      else *(unsigned short*)p = (unsigned short)q[0];
    } else {
      store_once((u32x4*)p, (u32x4){q[0], q[1], q[2], q[3]}, stream);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) q[i] = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    return sizeof(T) == 4 ? unpack<T>(q[i], 0) : unpack<T>(q[i / 2], i % 2);
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
      if constexpr (sizeof(T) == 4) q[i] = __builtin_bit_cast(unsigned, v[i]);
      else q[i] = pack_bf16(v[2 * i < VEC ? 2 * i : 0], v[2 * i + 1 < VEC ? 2 * i + 1 : 0]);
  }
};

template <typename T, int W, int VEC, int U>
__global__ void __launch_bounds__(256) causal_conv_kernel(ConvArgs a) {
  // a sequence's second tile reads no row before the sequence
  static_assert(U == 1 || U >= W - 1, "one token: of sequences that have no second tile");
  using P = Pack<T, VEC>;
  // a block has four tiles of the same 64 VEC channels, whose weights it lays out by tap
  __shared__ __align__(16) float sw[W][64 * VEC];
  const int quad = fdiv((int)blockIdx.x, a.dblocks), c0 = ((int)blockIdx.x - quad * a.dblocks.d) * 64 * VEC;
  const int own = min(64 * VEC, a.channels - c0) * W;
  for (int e = (int)threadIdx.x; e < own; e += 256) sw[e % W][e / W] = a.w[(int64_t)c0 * W + e];
  __syncthreads();
  const int id = quad * 4 + wave_id();
  if (id >= a.tiles) return;
  int t0;
  const SeqRange r = find_tile(a.s, a.per, U, id, &t0);
  const bool first = t0 == r.begin;
  if (r.s < 0 || (t0 >= r.end && !first)) return;
  const int lc = (int)(threadIdx.x & 63) * VEC, c = c0 + lc;
  if (c >= a.channels) return;

  const T* x = (const T*)a.x + c;
  P row[U + W - 1];
  if (first) {
    const int slot = seq_slot(a.s, r.s);
    const int64_t at = ((int64_t)slot * (W - 1)) * a.channels + c;
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
      if (slot >= 0 && a.state_in)
        row[i].load((const T*)a.state_in + at + (int64_t)i * a.channels);
      else
        row[i].zero();
    if (slot >= 0 && a.state_out) {
      const int len = r.end - r.begin;
      P next[W - 1];
#pragma unroll
      for (int i = 0; i < W - 1; ++i) {
        if (len + i >= W - 1)
          next[i].load(x + (int64_t)(r.end - (W - 1) + i) * a.ldx);
        else  // a sequence shorter than the history: part of the old one stays
#pragma unroll
          for (int k = 0; k < W - 1; ++k)
            if (k == len + i) next[i] = row[k];
      }
#pragma unroll
      for (int i = 0; i < W - 1; ++i) next[i].store((T*)a.state_out + at + (int64_t)i * a.channels, false);
    }
    if (r.end == r.begin) return;
  } else {
#pragma unroll
    for (int i = 0; i < W - 1; ++i) row[i].load(x + (int64_t)(t0 - (W - 1) + i) * a.ldx);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) row[W - 1 + i].load(x + (int64_t)min(t0 + i, r.end - 1) * a.ldx);

  float w[W][VEC], bias[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    bias[i] = a.bias ? a.bias[c + i] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = sw[j][lc + i];
  }
  T* y = (T*)a.y + c;
#pragma unroll
  for (int t = 0; t < U; ++t) {
    if (t0 + t >= r.end) break;
    float v[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      v[i] = bias[i];
#pragma unroll
      for (int j = 0; j < W; ++j) v[i] = fmaf(w[j][i], row[t + j].get(i), v[i]);
      if (a.act == CT_ACT_SILU) v[i] = silu_f32(v[i]);
    }
    P out;
    out.set(v);
    out.store(y + (int64_t)(t0 + t) * a.ldy, a.stream);
  }
}

template <typename T, int W, int VEC, int U>
static int conv_launch(ConvArgs a, hipStream_t st) {
  const SeqTiles n = seq_tiles(a.s, U);
  a.per = n.per;
  a.dblocks = make_fastdiv((a.channels + 64 * VEC - 1) / (64 * VEC));
  const int64_t blocks = (n.total + 3) / 4 * a.dblocks.d;
  a.tiles = (int)n.total;
  if (n.total > 0x7FFFFFF0 || !fits_launch(blocks, 256)) return refuse_size("ct_causal_conv_run");
  return launch(causal_conv_kernel<T, W, VEC, U>, dim3((unsigned)blocks), 256, 0, st, a);
}
template <typename T, int W>
static int conv_pick(const ConvArgs& a, bool wide, hipStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  if (!a.s.offsets && a.s.len <= 1) return wide ? conv_launch<T, W, V, 1>(a, st) : conv_launch<T, W, 1, 1>(a, st);
  if (!wide) return conv_launch<T, W, 1, 8>(a, st);
  // shorter tiles where those of eight tokens are fewer than one wave for every SIMD: 1020
  // tokens of 2048 channels 6.9 to 5.9 us (8192 of 4096: 34.1 and 34.3)
  const int64_t waves = (int64_t)(a.s.tokens / 8) * ((a.channels + 64 * V - 1) / (64 * V));
  if constexpr (W <= 5)
    if (waves < 4 * kPlanCus) return conv_launch<T, W, V, 4>(a, st);
  return conv_launch<T, W, V, 8>(a, st);
}
template <typename T>
static int conv_pick_width(const ConvArgs& a, int width, bool wide, hipStream_t st) {
  switch (width) {
    case 2: return conv_pick<T, 2>(a, wide, st);
    case 3: return conv_pick<T, 3>(a, wide, st);
    case 4: return conv_pick<T, 4>(a, wide, st);
    case 5: return conv_pick<T, 5>(a, wide, st);
    case 6: return conv_pick<T, 6>(a, wide, st);
    case 7: return conv_pick<T, 7>(a, wide, st);
    default: return conv_pick<T, 8>(a, wide, st);
  }
}

int launch_causal_conv(const ct_causal_conv_op& op, const SeqView& s, const void* x, const float* w,
                       const float* bias, const void* state_in, void* state_out, void* y, void* stream) {
  ConvArgs a = {};
  a.s = s;
  a.x = x; a.w = w; a.bias = bias; a.state_in = state_in; a.state_out = state_out; a.y = y;
  a.ldx = op.ldx; a.ldy = op.ldy; a.channels = op.channels; a.act = op.act;
  a.stream = (int64_t)s.tokens * op.channels * elem_bytes(op.dtype) >= kStreamBytes;
  // 16-byte accesses need every row on a 16-byte address, the history's too
  const int v = 16 / elem_bytes(op.dtype);
  const bool wide = ((uintptr_t)x | (uintptr_t)y | (uintptr_t)state_in | (uintptr_t)state_out) % 16 == 0 &&
                    op.ldx % v == 0 && op.ldy % v == 0 && op.channels % v == 0;
  hipStream_t st = (hipStream_t)stream;
  return op.dtype == CT_DT_BF16 ? conv_pick_width<bf16_t>(a, op.width, wide, st)
                                : conv_pick_width<float>(a, op.width, wide, st);
}

}  // namespace ct
