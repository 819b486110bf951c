// Device helpers of the sequence-block operators.
#pragma once
#include <hip/hip_runtime.h>

#include "k_util.h"
#include "seq_internal.h"

namespace ct {

// A bf16 in memory. Arithmetic is in fp32; a result is rounded to nearest even.
struct bf16_t {
  unsigned short bits;
  bf16_t() = default;
  __device__ __forceinline__ explicit bf16_t(float v) : bits(__builtin_bit_cast(unsigned short, (__bf16)v)) {}
  __device__ __forceinline__ explicit operator float() const {
    return __builtin_bit_cast(float, (unsigned)bits << 16);
  }
};
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Whether `blocks` blocks fit one launch: block numbers of 31 bits, threads of 32.
inline bool fits_launch(int64_t blocks, int threads) {
  return blocks <= 0x7FFFFFFF && blocks * threads <= 0xFFFFFFFFll;
}
// 0, or -1 with the reason left in hipGetLastError. An error that another call left there is
// none of this launch's.
template <typename A>
inline int launch(void (*kernel)(A), dim3 blocks, int threads, size_t lds, hipStream_t st, A a) {
  void* args[] = {&a};
  return hipLaunchKernel((const void*)kernel, blocks, dim3((unsigned)threads), args, lds, st) == hipSuccess ? 0 : -1;
}
inline int refuse_size(const char* who) {
  set_error(std::string(who) + ": too large for one launch");
  return -2;
}

// ---- 32-bit words of packed elements ----
// Element i of a 16-bit pair, or the word itself.
template <typename T>
__device__ __forceinline__ float unpack(unsigned word, int i) {
  if constexpr (sizeof(T) == 4)
    return __builtin_bit_cast(float, word);
  else  // a bf16 is the upper half of the fp32 with its value
    return __builtin_bit_cast(float, i ? word & 0xFFFF0000u : word << 16);
}
// Two fp32 rounded to nearest even into one word.
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 p;
  p.x = (__bf16)lo;
  p.y = (__bf16)hi;
  return __builtin_bit_cast(unsigned, p);
}
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  return (T)v;
}

// ---- four elements of a row ----
struct Quad {
  float v[4];
};
// Four elements of a row that all exist, in one access wherever the row lies.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
template <typename O>
__device__ __forceinline__ Quad load_quad4(const O* p) {
  if constexpr (sizeof(O) == 2) {
    const u32x2 q = *(const u32x2_any*)p;
    const unsigned q0 = q.x, q1 = q.y;
    return {unpack<O>(q0, 0), unpack<O>(q0, 1), unpack<O>(q1, 0), unpack<O>(q1, 1)};
  } else {
    const f32x4 q = *(const f32x4_any*)p;
    return {q.x, q.y, q.z, q.w};
  }
}
// The column that a lane's four states from state n on are read from, of a row that ends on a
// multiple of four: the row's first four, whose values are not used, where there is no state n.
constexpr int quad_column(int n, int states) { return n < states ? n : 0; }

// ---- outputs larger than the caches that would hold them ----
// Bytes of an output from which its stores go past the L2s instead of pushing out of them
// what is still to be read: where the next reader would not find it in the 256 MB cache
// behind them anyway (134 MB of a product 451 to 428 us). Smaller outputs that the next
// kernel reads are better left there: four products of 67 MB one after another take 843 us,
// and 860 past the caches.
constexpr int64_t kStreamBytes = 128 << 20;
// The same for states, which nothing reads before the next token: 67 MB read and written 37
// to 27 us; in place, 33 MB in 16.5 us either way.
constexpr int64_t kStreamStateBytes = 32 << 20;
template <typename P, typename V>
__device__ __forceinline__ void store_once(P* p, V v, bool stream) {
  if (stream) {
    asm volatile("");  // between two of these, or the two stores become one, without the hint
    __builtin_nontemporal_store(v, p);
    asm volatile("");
  } else {
    *p = v;
  }
}

template <typename O>
__device__ __forceinline__ void store_quad4(O* p, const float* v, bool stream) {
  if constexpr (sizeof(O) == 2) store_once((u32x2_any*)p, (u32x2){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}, stream);
  else store_once((f32x4_any*)p, (f32x4){v[0], v[1], v[2], v[3]}, stream);
}

// ---- rows that lanes take an element of each ----
// `rows` rows from `base` on, `pitch` elements apart, of `cols` elements: a lane's byte offset
// in a row and the row's uniform one need no address arithmetic on the vector ALU. The range
// check is only asked about the lane's offset, which is the one that is past every row (fewer
// than 2^31 bytes in all): the uniform one stays among the rows.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const T* base, int rows, int64_t pitch, int cols) {
  return make_rsrc(base, ((int64_t)(rows - 1) * pitch + cols) * (int64_t)sizeof(T));
}
constexpr int row_or_last(int row, int rows) { return row < rows ? row : rows - 1; }
template <typename T>
__device__ __forceinline__ float load_elem(__amdgpu_buffer_rsrc_t r, unsigned off, int row) {
  if constexpr (sizeof(T) == 4)
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, (int)off, row, 0));
  else
    return __builtin_bit_cast(float, (unsigned)__builtin_amdgcn_raw_buffer_load_b16(r, (int)off, row, 0) << 16);
}
template <typename T>
__device__ __forceinline__ void store_elem(__amdgpu_buffer_rsrc_t r, unsigned off, int row, float v) {
  if constexpr (sizeof(T) == 4)
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, (int)off, row, 0);
  else
    __builtin_amdgcn_raw_buffer_store_b16(bf16_t(v).bits, r, (int)off, row, 0);
}

// ---- 16-byte groups, or words, of an operand's rows ----
// Byte offset past every operand tile: reads as 0.
constexpr unsigned kOobGroup = 0xFFFFFFF0u;
// The uniform offset of copies k bytes into the rows of a buffer. The range check need not count
// it, and where it subtracts it from the buffer's size the difference must not pass below 0,
// which a slice past the end of a single row's would bring about: it stops at the buffer's end,
// where no lane has anything to copy.
constexpr int uniform_part(unsigned k, unsigned bytes) { return (int)(k < bytes ? k : bytes); }

// ---- scalar functions in fp32 ----
constexpr float kLog2e = 1.4426950408889634f;
// v_exp_f32: within an ulp, results below 2^-126 flushed to 0.
__device__ __forceinline__ float exp_f32(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
// v / (1 + exp(-v)) through the approximate reciprocal (an ulp). exp(-v) = inf gives -0
// for every finite v, as the limit does.
__device__ __forceinline__ float silu_f32(float v) { return v * __builtin_amdgcn_rcpf(1.f + exp_f32(-v)); }
// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|). The step sizes of a scan are the
// small values of this function, where log(1 + e) has lost e's low bits: u = 1 + e is
// rounded, and log1p(e) = log(u) + (e - (u - 1)) / u to first order in that rounding. The
// division changes the correction, half a unit of u at most, by less than a unit of the sum.
__device__ __forceinline__ float softplus_f32(float v) {
  const float e = exp_f32(-fabsf(v)), u = 1.f + e;
  const float l = __builtin_amdgcn_logf(u) * 0.6931471805599453f;
  return fmaxf(v, 0.f) + (l + (e - (u - 1.f)));  // NaN stays in l
}
// v / 2 (1 + erf(v / sqrt(2))) = v Phi(v), with the tail probability of |v| after Abramowitz
// and Stegun, 7.1.26 (off by 7.5e-8 at most): Phi(-|v|) = t (c1 + t (c2 + ...)) exp(-v^2 / 2)
// / 2 with t = 1 / (1 + p |v| / sqrt(2)). A negative v takes the tail itself, so that nothing
// cancels there. 18 full-rate and two quarter-rate instructions.
__device__ __forceinline__ float gelu_f32(float v) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(v), 0.3275911f * 0.70710678118654752f, 1.f));
  const float e = __builtin_amdgcn_exp2f(v * v * (-0.5f * kLog2e));
  float s = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  s = fmaf(t, s, 0.5f * 1.421413741f);
  s = fmaf(t, s, 0.5f * -0.284496736f);
  s = fmaf(t, s, 0.5f * 0.254829592f);
  const float tail = s * t * e;
  const float phi = v < 0.f ? tail : 1.f - tail;
  return v * phi;
}
// Comparisons that keep NaN, unlike fmax.
__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case CT_ACT_RELU: return v < 0.f ? 0.f : v;
    case CT_ACT_RELU6: return v < 0.f ? 0.f : (v > 6.f ? 6.f : v);
    case CT_ACT_SILU: return silu_f32(v);
    case CT_ACT_GELU: return gelu_f32(v);
  }
  return v;
}

// ---- sequences ----
struct SeqRange {
  int s, begin, end;  // rows begin..end-1 of sequence s
};
// The rows of sequence s, kept inside 0..tokens whatever the offsets hold.
__device__ __forceinline__ SeqRange seq_range(const SeqView& v, int s) {
  if (!v.offsets) return {s, s * v.len, s * v.len + v.len};
  const int b = min(max(v.offsets[s], 0), v.tokens), e = min(max(v.offsets[s + 1], b), v.tokens);
  return {s, b, e};
}
// State slot of sequence s, -1 for none.
__device__ __forceinline__ int seq_slot(const SeqView& v, int s) {
  const int slot = v.slots ? v.slots[s] : s;
  return slot >= 0 && slot < v.num_slots ? slot : -1;
}

// Sequences cut into tiles of `step` rows that start at a sequence's own start. Sequence s
// owns the tile numbers from begin / step + s on: at least one, so that an empty sequence
// has a tile too, and never more than begin to end can need. A few numbers at the end of a
// sequence are unused.
constexpr int tiles_in(int rows, int step) { return rows / step + (rows % step != 0); }
struct SeqTiles {
  int64_t total;
  int per;  // tiles of each sequence where the lengths are equal
};
inline SeqTiles seq_tiles(const SeqView& v, int step) {
  if (v.offsets) return {(int64_t)v.tokens / step + v.count, 0};
  const int per = v.len > step ? tiles_in(v.len, step) : 1;
  return {(int64_t)per * v.count, per};
}
// The end of a tile that starts at row t0 of a sequence: 2^31 rows may be less than a tile away.
constexpr int tile_end(int t0, int end, int step) { return end - t0 > step ? t0 + step : end; }
// The row that tile k of a sequence starts at: its end at most, -1 for a number past that (and
// perhaps far, where offsets do not ascend).
constexpr int tile_start(int begin, int end, int step, int k) {
  return k > (end - begin) / step ? -1 : begin + k * step;
}
// The sequence that tile `id` belongs to (s = -1: none) and, in *first, the row that the tile
// starts at: the sequence's end for a number that it does not use. Uniform over the wave, which looks
// 64 sequences up at a time.
__device__ __forceinline__ SeqRange find_tile(const SeqView& v, int per, int step, int id, int* first) {
  if (!v.offsets) {
    const int s = id / per;
    const SeqRange r = seq_range(v, s);
    *first = r.begin + (id - s * per) * step;
    return r;
  }
  const int lane = (int)(threadIdx.x & 63);
  int lo = 0, n = v.count;
  while (true) {
    const int stride = (n + 63) / 64, i = lane * stride;
    const bool at_or_before =
        i < n && min(max(v.offsets[lo + min(i, n - 1)], 0), v.tokens) / step + lo + i <= id;
    const uint64_t below = __ballot(!at_or_before);  // the first lane past the tile
    const int k = below ? __builtin_ctzll(below) : 64;
    if (k == 0) return {-1, 0, 0};
    lo += (k - 1) * stride;
    n = min(stride, n - (k - 1) * stride);
    if (n <= 1) break;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const SeqRange r = seq_range(v, lo);
  *first = tile_start(r.begin, r.end, step, id - (r.begin / step + lo));
  return *first < 0 ? SeqRange{-1, 0, 0} : r;
}

}  // namespace ct
