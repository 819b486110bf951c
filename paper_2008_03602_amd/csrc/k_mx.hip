// Rows to microscaled rows, and back to the values they stand for.
//
// A pass over the values with nothing to compute but a maximum of 32, so the bytes bound it: 16
// bytes a lane of bf16 (32 of fp32), a block to four lanes, whose maximum goes through two
// permutations of neighbouring lanes. 8192 x 4096 bf16 to 4 bits 15-20 us, to 8 bits 17.6, and back
// 15.2 and 17.0: 4.2 to 5.9 TB/s.
#include <hip/hip_runtime.h>

#include "k_mx.h"

namespace ct {

struct MxArgs {
  void* x;
  char* q;
  unsigned char* scales;
  int rows, cols;
  int64_t ldx, ldq, lds;
  FastDiv per;  // octs of a row, in whole blocks
};

constexpr int kMxThreads = 256;

// Row and first column of a thread: octs are numbered along the rows. False past the last.
__device__ __forceinline__ bool mx_place(const MxArgs& a, int* row, int* col) {
  const int64_t at = (int64_t)blockIdx.x * kMxThreads + threadIdx.x;
  if (at >= (int64_t)a.rows * a.per.d) return false;
  if (at <= 0x7FFFFFFF) *row = fdiv((int)at, a.per);
  else *row = (int)(at / a.per.d);
  *col = (int)(at - (int64_t)*row * a.per.d) * 8;
  return true;
}

template <typename T, int FORMAT>
__global__ void __launch_bounds__(kMxThreads) mx_quantise_kernel(MxArgs a) {
  int row, col;
  if (!mx_place(a, &row, &col)) return;  // whole blocks
  RawOct<T> r = {};
  if (col < a.cols) load_oct<T>(r, (const T*)a.x + row * a.ldx + col, a.cols - col);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = r.at(i);
  const unsigned scale = mx_scale<FORMAT>(mx_largest(v));  // the four lanes of a block together
  mx_write<FORMAT>(mx_elements<FORMAT>(v, mx_inverse(scale)), scale, a.q + row * a.ldq, a.scales + row * a.lds,
                   (unsigned)col, a.cols);
}

template <typename T, int FORMAT>
__global__ void __launch_bounds__(kMxThreads) mx_values_kernel(MxArgs a) {
  int row, col;
  if (!mx_place(a, &row, &col) || col >= a.cols) return;
  const char* q = a.q + row * a.ldq;
  const float scale = mx_scale_value(a.scales[row * a.lds + col / kMxBlock]);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 p[4];
  if constexpr (FORMAT == CT_MX_E4M3) {
    const u32x2 w = *(const u32x2*)(q + col);
    const unsigned w0 = w.x, w1 = w.y;
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w0, 1.f, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w0, 1.f, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w1, 1.f, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w1, 1.f, true);
  } else {
    const unsigned w = *(const unsigned*)(q + col / 2);
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
  }
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = p[i].x * scale;
    v[2 * i + 1] = p[i].y * scale;
  }
  store_oct<T>((T*)a.x + row * a.ldx + col, v, a.cols - col);
}

template <int FORMAT>
static int mx_pick(const MxArgs& a, bool bf16, bool values, unsigned blocks, hipStream_t st) {
  if (values)
    return bf16 ? launch(mx_values_kernel<bf16_t, FORMAT>, dim3(blocks), kMxThreads, 0, st, a)
                : launch(mx_values_kernel<float, FORMAT>, dim3(blocks), kMxThreads, 0, st, a);
  return bf16 ? launch(mx_quantise_kernel<bf16_t, FORMAT>, dim3(blocks), kMxThreads, 0, st, a)
              : launch(mx_quantise_kernel<float, FORMAT>, dim3(blocks), kMxThreads, 0, st, a);
}

int launch_mx(const ct_mx_op& op, void* x, void* q, void* scales, bool values, void* stream) {
  MxArgs a = {x, (char*)q, (unsigned char*)scales, op.rows, op.cols, op.ldx, op.ldq, op.lds,
              make_fastdiv(4 * (int64_t)mx_blocks(op.cols))};
  const int64_t blocks = ((int64_t)op.rows * a.per.d + kMxThreads - 1) / kMxThreads;
  if (!fits_launch(blocks, kMxThreads)) return refuse_size(values ? "ct_mx_values_run" : "ct_mx_quantise_run");
  const bool bf16 = op.dtype == CT_DT_BF16;
  return op.format == CT_MX_E4M3 ? mx_pick<CT_MX_E4M3>(a, bf16, values, (unsigned)blocks, (hipStream_t)stream)
                                 : mx_pick<CT_MX_E2M1>(a, bf16, values, (unsigned)blocks, (hipStream_t)stream);
}

}  // namespace ct
