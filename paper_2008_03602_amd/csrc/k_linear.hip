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
  int m, n, k;
  int64_t ldx, ldw, ldr, ldy;
  int act, res_mode, out_bf16;
  int tiles_n;
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

// One output through the epilogue.
__device__ __forceinline__ void store_out(const LinearArgs& a, int i, int j, float v) {
  if (a.bias) v += a.bias[j];
  float r = 0.f;
  if (a.res_mode)
    r = a.out_bf16 ? (float)((const bf16_t*)a.res)[i * a.ldr + j] : ((const float*)a.res)[i * a.ldr + j];
  if (a.res_mode == CT_RES_ADD_ACT) v += r;
  v = activate(v, a.act);
  if (a.res_mode == CT_RES_ADD) v += r;
  if (a.out_bf16) ((bf16_t*)a.y)[i * a.ldy + j] = (bf16_t)v;
  else ((float*)a.y)[i * a.ldy + j] = v;
}

// A 64 x 64 tile of y by four waves of 32 x 32, the operands through LDS a 128-byte slice
// of each row at a time, element by element.
template <typename T>
__global__ void __launch_bounds__(256) linear_kernel(LinearArgs a) {
  constexpr int G = 16 / (int)sizeof(T), KC = 8 * G;
  __shared__ __align__(16) T sx[64][KC + G], sw[64][KC + G];
  const int n0 = (int)(blockIdx.x % a.tiles_n) * 64, m0 = (int)(blockIdx.x / a.tiles_n) * 64;
  const int t = threadIdx.x, lane = t & 63, wave = wave_id();
  const int wn = (wave & 1) * 32, wm = (wave >> 1) * 32, lrow = lane & 15, kg = lane >> 4;
  f32x4 acc[2][2] = {};
  for (int k0 = 0; k0 < a.k; k0 += KC) {
    __syncthreads();
    for (int e = t; e < 64 * KC; e += 256) {
      const int r = e / KC, k = e % KC;
      const bool ok = k0 + k < a.k;
      sx[r][k] = ok && m0 + r < a.m ? ((const T*)a.x)[(m0 + r) * a.ldx + k0 + k] : (T)0.f;
      sw[r][k] = ok && n0 + r < a.n ? ((const T*)a.w)[(n0 + r) * a.ldw + k0 + k] : (T)0.f;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 fw[2], fx[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fw[i] = *(const u32x4*)&sw[wn + i * 16 + lrow][(s * 4 + kg) * G];
        fx[i] = *(const u32x4*)&sx[wm + i * 16 + lrow][(s * 4 + kg) * G];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mma16<T>(fw[i], fx[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = m0 + wm + j * 16 + lrow, col = n0 + wn + i * 16 + 4 * kg + e;
        const float v = acc[i][j][e];
        if (row < a.m && col < a.n) store_out(a, row, col, v);
      }
}

LinearPlan plan_linear(const ct_linear_op&) { return {1, 0}; }

int launch_linear(const ct_linear_op& op, const LinearPlan&, const void* x, const void* w, const float* bias,
                  const void* res, void* y, float*, void* stream) {
  LinearArgs a = {};
  a.x = x; a.w = w; a.res = res; a.bias = bias; a.y = y;
  a.m = op.m; a.n = op.n; a.k = op.k;
  a.ldx = op.ldx; a.ldw = op.ldw; a.ldr = op.ldr; a.ldy = op.ldy;
  a.act = op.act; a.res_mode = op.res; a.out_bf16 = op.out_dtype == CT_DT_BF16;
  a.tiles_n = (op.n + 63) / 64;
  const int64_t blocks = (int64_t)a.tiles_n * ((op.m + 63) / 64);
  if (blocks > 0x7FFFFFFF) return refuse_size("ct_linear_run");
  auto fn = op.dtype == CT_DT_BF16 ? linear_kernel<bf16_t> : linear_kernel<float>;
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace ct
