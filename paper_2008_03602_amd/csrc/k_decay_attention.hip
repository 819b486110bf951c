// Linear attention with a decay for each head, along packed sequences: with l_t = min(dt_t a, 0)
//   S_t = exp(l_t) S_{t-1} + k_t^T v_t (dt_t),   o_t = scale q_t S_t.
#include <hip/hip_runtime.h>

#include "k_seq.h"

namespace ct {

// Sequences of at most this many tokens go token by token.
constexpr int kDecayStepTokens = 4;

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
  // pieces of a sequence (0 tokens: whole sequences): their numbering, what each leaves to the next
  int piece, per;
  f32x4* ends;    // pieces x heads x frames
  float* decays;  // pieces x heads
  int frames;     // quads of a state in the order of the matrix cores' results
};

// Step and logarithm of the decay of a head at a token. A step or rate that is NaN stays one; below
// e^-104 the decay is 0 in fp32, and a sum of many such logarithms would lose the small ones.
struct Step {
  float dt, l;
};
// What `delta` holds for a token (0 without): asked for early, looked at late.
__device__ __forceinline__ float delta_of(const DecayArgs& a, int row, int head) {
  if (!a.delta) return 0.f;
  const int64_t at = row * a.lddelta + head;
  return a.delta_bf16 ? (float)((const bf16_t*)a.delta)[at] : ((const float*)a.delta)[at];
}
__device__ __forceinline__ Step step_of(const DecayArgs& a, float delta, float bias, float rate) {
  float dt = 1.f;
  if (a.delta) {
    dt = delta + bias;
    if (a.softplus) dt = softplus_f32(dt);
  }
  float l = dt * rate;
  l = l > 0.f ? 0.f : l;
  l = l < -104.f ? -104.f : l;
  return {dt, l};
}

// ------------------------------------------------------------------ token by token
// A block takes a head of a sequence with its state in registers: LANES lanes of four columns
// each, and 256 / LANES rows at a time. What it reads and writes of the state bounds it: all of it
// is on its way before the first product. 128 sequences of 16 heads of 128 x 128: 45.6 us, 5.9 TB/s;
// 8 of 64 x 64: 4.7 us, a launch and two latencies.
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
    const Step step = step_of(a, delta_of(a, t, head), bias, rate);
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
    const float decay = __builtin_amdgcn_exp2f(step.l * kLog2e);
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

// ------------------------------------------------------------------ chunks of a prompt
// With G_i the sum of l over the tokens of a chunk up to i, and S the state before it,
//   o_i = e^{G_i} q_i S + sum_{j <= i} e^{G_i - G_j} (q_i k_j) dt_j v_j,
//   S'  = e^{G_C} S + sum_j k_j^T e^{G_C - G_j} dt_j v_j.
// A block takes a head of a sequence, or of a piece of one, and up to 64 NC columns of v, chunk by
// chunk. Its four waves have 16 NC columns each: their part of the state stays in the matrix
// cores' accumulators, whose layout is also that of an operand, so the state goes through no
// memory. Operands in rows are read from LDS as they lie there, those in columns transposed.
//
// What bounds it is the latency of a chunk's dependent steps (weights, what the state gives, what it
// gets, outputs: 13600 clocks of 128 x 128 in bf16, 17000 with a second block on the compute unit),
// not products (25 us of the 139; the matrix cores are busy 30 % of the clocks) or bytes (50 us). One
// prompt of 16384 tokens, 16 heads of 128 x 128, takes 46 us for its pieces' ends, 11 to join them and 89
// for the outputs, of which a wave lives 157 thousand clocks for its eight chunks, at 1.9 GHz; 8192 tokens
// of 32 heads of 128 x 64 that share 4 pairs of q and k 26, 7 and 66. Operands are read from LDS one
// step before the products that take them, the next chunk's copies start when this one's last reader is
// through, and four chunks' steps are made at a time, a wave to each. Chunks of 32 in fp32: of 64 they
// would take more LDS than two blocks on a compute unit have.
//
// Precision. In bf16 the inputs are exact, and what is computed from them is taken apart into bf16
// terms before it meets a matrix core: the state (for o) and the weights q k e^{..} into two, 2^-17
// of each, below the output's rounding; the weighted v, which the fp32 state is summed from, into
// three, 2^-25. fp32 takes fp32 products. G is summed in fp64 and kept as two fp32, so that weak
// decays keep their digits behind strong ones.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Mat;
template <>
struct Mat<bf16_t> {
  typedef bf16x8 Frag;  // row or column lane % 16, steps 8 (lane / 16) on, of 32
  static constexpr int CHUNK = 64, KS = 32, STATE_TERMS = 2, P_TERMS = 2, V_TERMS = 3;
  static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mat<float> {
  typedef f32x4 Frag;  // row or column lane % 16, steps 4 (lane / 16) on, of 16
  static constexpr int CHUNK = 32, KS = 16, STATE_TERMS = 1, P_TERMS = 1, V_TERMS = 1;
  static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = a[e], y = b[e];
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0);
    }
    return c;
  }
};
// Eight values as TERMS fragments whose sum they are, but for what the last one drops.
template <int TERMS>
__device__ __forceinline__ void split8(float (&v)[8], bf16x8 (&f)[TERMS]) {
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
      v[2 * i] -= unpack<bf16_t>(w[i], 0);
      v[2 * i + 1] -= unpack<bf16_t>(w[i], 1);
    }
    f[t] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
  }
}

// A tile in LDS: rows of BYTES, their 16-byte groups permuted by the row's number so that eight
// rows' groups, and the halves of four rows, lie in distinct banks.
template <int BYTES>
__device__ __forceinline__ int tile_at(int row, int group) {
  const int key = ((row & 3) << 1 | (row >> 2 & 1)) & (BYTES / 16 - 1);
  return row * BYTES + (group ^ key) * 16;
}
// The permutation is an exclusive or on the group's bits of an address, so that a lane's address of
// another group is its own one with that group's bits turned over, and that of a row a multiple of 8
// further on its own one and the rows between.
// Row r0 + lane % 16 (r0 a multiple of 8), steps of number k.
template <typename T, int BYTES>
__device__ __forceinline__ typename Mat<T>::Frag read_rows(const char* tile, int r0, int k) {
  const int lane = (int)threadIdx.x & 63;
  return *(const typename Mat<T>::Frag*)(tile + r0 * BYTES + (tile_at<BYTES>(lane & 15, lane >> 4) ^ k * 64));
}
// Column of lane % 16, steps (rows) of number k. In bf16 the lane's of four runs of four columns that
// lie RUN (4 or 8) columns apart, from column c0 on (a multiple of 16, or of 32 and 4 more); in fp32
// column c0 + lane % 16.
template <typename T, int BYTES, int RUN>
__device__ __forceinline__ typename Mat<T>::Frag read_cols(const char* tile, int k, int c0) {
  const int lane = (int)threadIdx.x & 63, g = lane >> 4, l = lane & 15;
  if constexpr (sizeof(T) == 2) {
    typedef i16x4 __attribute__((address_space(3))) * lds_i16x4;
    i16x4 part[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // this lane's run for the transposed read, of row l / 4
      const int at = tile_at<BYTES>(g * 8 + h * 4 + (l >> 2), (l & 3) * RUN / 8) ^ c0 / 8 * 16;
      const char* p = tile + k * 32 * BYTES + (c0 & 4) * 2 + at + ((l & 3) * RUN & 4) * 2;
      part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(__attribute__((address_space(3))) char*)p);
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    f32x4 f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      f[e] = *(const float*)(tile + k * 16 * BYTES + (tile_at<BYTES>(g * 4 + e, l / 4) ^ c0 * 4) + (l & 3) * 4);
    return f;
  }
}

// ROWS rows of a tile of BYTES each from memory, 16 bytes a lane straight into LDS where the rows
// lie on 16 bytes (wait_copies() and a barrier before they are read), else through registers; rows
// shorter than that element by element (8192 tokens of 8 heads of 250 x 130: 425 us with all of them so,
// 238 in groups of 16 bytes at any address). Elements past `cols` and rows past `rows` read 0.
template <typename T, int BYTES, int ROWS, bool ALIGNED>
__device__ __forceinline__ void fill_tile(char* tile, const T* base, int64_t ld, int rows, int cols) {
  constexpr int GROUPS = BYTES / 16, N = ROWS * GROUPS / 256, E = 16 / (int)sizeof(T);
  static_assert(ROWS * GROUPS % 256 == 0, "");
  const __amdgpu_buffer_rsrc_t r = make_rsrc(base, rows > 0 ? ((rows - 1) * ld + cols) * (int64_t)sizeof(T) : 0);
  // Where a thread's group i is from: whose place its slot is (the permutation is its own inverse)
  const auto offset = [&](int i, int* col) {
    const int at = i * 256 + (int)threadIdx.x, row = at / GROUPS;
    *col = (tile_at<BYTES>(row, at % GROUPS) - row * BYTES) / 16 * E;
    if (row >= rows) *col = cols;
    return (unsigned)(row * (int)ld + *col) * (unsigned)sizeof(T);
  };
  if constexpr (ALIGNED) {
    char* mine = tile + wave_id() * 1024;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int col;
      const unsigned off = offset(i, &col);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)(mine + i * 4096), 16, (int)(col < cols ? off : kOobGroup), 0, 0, 0);
    }
  } else if (cols >= E) {
    // A row's last group comes from the 16 bytes that end with the row, turned down; lanes without a
    // group read the tile's first
    const int bits = (E - cols % E) % E * 8 * (int)sizeof(T);
    u32x4 w[N];
    int left[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int col;
      offset(i, &col);
      left[i] = cols - col;
      const int row = left[i] > 0 ? (i * 256 + (int)threadIdx.x) / GROUPS : 0;
      w[i] = *(const u32x4_any*)(base + row * ld + (left[i] > 0 ? min(col, cols - E) : 0));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (left[i] < E) {
        typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
        u64x2 q = __builtin_bit_cast(u64x2, w[i]);
        if (bits >= 64) q = (u64x2){q.y >> (bits - 64), 0};
        else if (bits) q = (u64x2){q.x >> bits | q.y << (64 - bits), q.y >> bits};
        w[i] = left[i] > 0 ? __builtin_bit_cast(u32x4, q) : u32x4{};
      }
      *(u32x4*)(tile + (i * 256 + (int)threadIdx.x) * 16) = w[i];
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      int col;
      const unsigned off = offset(i, &col);
      unsigned w[4] = {};
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int o = (int)(col + e < cols ? off + e * (unsigned)sizeof(T) : kOobGroup);
        if constexpr (sizeof(T) == 2) w[e / 2] |= (unsigned)__builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0) << (16 * (e & 1));
        else w[e] = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0);
      }
      *(u32x4*)(tile + (i * 256 + (int)threadIdx.x) * 16) = (u32x4){w[0], w[1], w[2], w[3]};
    }
  }
}

// What the tokens of a chunk carry: G in two parts, e^G and the steps (1 where they do not scale the
// input), both times the scale of o, and the weights of the state's sum.
template <int C>
struct Steps {
  float hi[C], lo[C], grown[C], weight[C], dt[C];
  float end;   // e^{G_C}
  double sum;  // G_C / ln 2
};

// Whether one of a lane's values is infinite or NaN.
__device__ __forceinline__ bool any_wild(bf16x8 f) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u32x4 q = __builtin_bit_cast(u32x4, f);
  u16x2 m = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned w = q[i] & 0x7FFF7FFFu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w));
  }
  return max(m.x, m.y) >= 0x7F80;
}
__device__ __forceinline__ bool any_wild(f32x4 f) {
  bool any = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) any |= !(__builtin_fabsf(f[e]) < __builtin_inff());
  return any;
}

template <typename T, int DK, int NC, bool OUT, bool ALIGNED>
__global__ void __launch_bounds__(256, DK * (int)sizeof(T) > 512 || (!ALIGNED && DK * NC == 256) ? 1 : 2) decay_tile_kernel(DecayArgs a) {
  typedef Mat<T> M;
  typedef typename M::Frag Frag;
  constexpr int C = M::CHUNK, KS = M::KS, IT = C / 16, DT = DK / 16, DKS = DK / KS, CKS = C / KS;
  constexpr int DV = 64 * NC, KB = DK * (int)sizeof(T), VB = DV * (int)sizeof(T), PB = C * (int)sizeof(T);
  // OUT: q, k, v and the weights; else k and v, twice
  constexpr int AT_K = OUT ? C * KB : 0, AT_V = AT_K + C * KB, AT_P = AT_V + C * VB, TWICE = OUT ? 0 : AT_P;
  extern __shared__ __align__(16) char lds[];
  __shared__ Steps<C> steps[8];  // four chunks ahead, a wave to each, and the four at work
  const int lane = (int)threadIdx.x & 63, wave = wave_id(), g = lane >> 4, l16 = lane & 15;
  char *tq = lds, *tp = lds + AT_P;

  const int unit = fdiv((int)blockIdx.x, a.dheads), head = (int)blockIdx.x - unit * a.heads;
  int begin, end;
  SeqRange r;
  if (a.piece) {
    r = find_tile(a.seqs, a.per, a.piece, unit, &begin);
    if (r.s < 0 || (begin >= r.end && r.end > r.begin)) return;  // a number that no piece has
    end = tile_end(begin, r.end, a.piece);
  } else {
    r = seq_range(a.seqs, unit);
    begin = r.begin;
    end = r.end;
  }
  const bool first = begin == r.begin, last = end == r.end;
  if (!OUT && last) return;  // nothing comes after it
  const int slot = seq_slot(a.seqs, r.s), group = fdiv(head, a.dper);
  const int c0 = (int)blockIdx.y * DV, cw = c0 + wave * 16 * NC;  // the block's columns, the wave's
  const int cols = min(a.value - c0, DV);
  const float bias = a.dt_bias ? a.dt_bias[head] : 0.f, rate = a.a[head];
  const T* q = (const T*)a.q + (int64_t)group * a.key;
  const T* k = (const T*)a.k + (int64_t)group * a.key;
  const T* v = (const T*)a.v + (int64_t)head * a.value + c0;

  // What delta holds for the chunk at t, a token to a lane, as it lies there: no wait until its steps are made
  const auto ask = [&](int t) __attribute__((always_inline)) {
    if (!a.delta || t >= end) return 0u;
    const int64_t at = min((int64_t)t + lane, (int64_t)end - 1) * a.lddelta + head;
    return a.delta_bf16 ? (unsigned)((const uint16_t*)a.delta)[at] : ((const unsigned*)a.delta)[at];
  };
  unsigned delta = ask(tile_end(begin, end, wave * C));  // first: loads come back in their order
  const auto fill = [&](int t, int half) __attribute__((always_inline)) {
    const int rows = min(end - t, C);
    if constexpr (OUT) fill_tile<T, KB, C, ALIGNED>(tq, q + t * a.ldq, a.ldq, rows, a.key);
    fill_tile<T, KB, C, ALIGNED>(lds + AT_K + half * TWICE, k + t * a.ldk, a.ldk, rows, a.key);
    fill_tile<T, VB, C, ALIGNED>(lds + AT_V + half * TWICE, v + t * a.ldv, a.ldv, rows, cols);
  };
  if (begin < end) fill(begin, 0);

  // The state: element e of S[t][c] is row row0 + row_of(t) + e, column cw + 16 c + l16, of a buffer
  // that ends with its last row; columns past the last have an offset past it.
  const int row0 = sizeof(T) == 2 ? g * 8 : g * 4;
  const auto row_of = [](int t) { return sizeof(T) == 2 ? t / 2 * 32 + (t & 1) * 4 : t * 16; };
  const int64_t state_at = ((int64_t)slot * a.heads + head) * a.key * a.value;
  const unsigned state_bytes = (unsigned)(a.key * a.value) * 4;
  unsigned state_off[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = cw + 16 * c + l16;
    state_off[c] = col < a.value ? (unsigned)(row0 * a.value + col) * 4 : kOobGroup;
  }
  const auto frame_of = [&](int u) {
    return a.ends + ((int64_t)u * a.heads + head) * a.frames + (((int)blockIdx.y * 4 + wave) * NC * DT) * 64 + lane;
  };
  f32x4* frames = frame_of(unit);
  f32x4 S[DT][NC];
  if (OUT && !(first && last)) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) S[t][c] = frames[(t * NC + c) * 64];
  } else {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) S[t][c] = f32x4{};
    if (first && slot >= 0 && a.state_in) {
      const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.state_in + state_at, state_bytes);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            S[t][c][e] = load_elem<float>(rs, state_off[c] == kOobGroup ? kOobGroup : state_off[c] + (unsigned)((row_of(t) + e) * a.value) * 4, 0);
    }
    // The join hands the sequence's state on to its first piece too: state_out may be state_in, and
    // the last piece's block may write it before the first one's starts.
    if (!OUT && first) {
      f32x4* keep = frame_of(unit + tiles_in(r.end - begin, a.piece) - 1);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c) keep[(t * NC + c) * 64] = S[t][c];
    }
  }

  // The steps of the chunk at t from what was asked for before
  const auto make_steps = [&](int t, unsigned delta, Steps<C>& to) __attribute__((always_inline)) {
    const bool mine = lane < C && t < end && t + lane < end;
    const Step s = step_of(a, __builtin_bit_cast(float, a.delta_bf16 ? delta << 16 : delta), bias, rate);
    double G = mine ? (double)s.l * 1.4426950408889634 : 0.;
#pragma unroll
    for (int o = 1; o < C; o <<= 1) {
      const double up = __shfl_up(G, o);
      if (lane >= o) G += up;
    }
    const double all = __shfl(G, C - 1);
    if (lane < C) {
      const float dt = a.step_input && mine ? s.dt : 1.f;
      to.hi[lane] = (float)G;
      to.lo[lane] = (float)(G - (double)(float)G);
      to.grown[lane] = __builtin_amdgcn_exp2f((float)G) * a.scale;
      to.weight[lane] = __builtin_amdgcn_exp2f((float)(all - G)) * dt;
      to.dt[lane] = dt * a.scale;
      if (lane == 0) {
        to.end = __builtin_amdgcn_exp2f((float)all);
        to.sum = all;
      }
    }
  };

  double total = 0;
  int turn = 0;
#pragma unroll 1
  for (int t = begin; t < end; turn = (turn + 1) & 7) {
    const Steps<C>& st = steps[turn];
    const int next = tile_end(t, end, C);
    if (turn % 4 == 0) make_steps(tile_end(t, end, wave * C), delta, steps[turn + wave]);
    wait_copies();
    __syncthreads();
    if (turn % 4 == 3) delta = ask(tile_end(next, end, wave * C));
    const int half = OUT ? 0 : turn & 1;
    const char *tk = lds + AT_K + half * TWICE, *tv = lds + AT_V + half * TWICE;
    if constexpr (!OUT) {
      total += st.sum;
      if (next < end) fill(next, half ^ 1);  // whose last chunk everybody has read
    }

    f32x4 O[IT][NC];
    if constexpr (OUT) {
      // Weights of tokens i = 16 wave + l16 (a wave to 16 of them), j = 16 jt + 4 g + e
      if (wave < IT) {
        f32x4 p[IT] = {};
        Frag fq = read_rows<T, KB>(tq, wave * 16, 0), fk[IT];
#pragma unroll
        for (int jt = 0; jt < IT; ++jt) fk[jt] = read_rows<T, KB>(tk, jt * 16, 0);
#pragma unroll
        for (int s = 0; s < DKS; ++s) {
          const Frag nq = read_rows<T, KB>(tq, wave * 16, s + 1 < DKS ? s + 1 : s);
#pragma unroll
          for (int jt = 0; jt < IT; ++jt) {
            const Frag now = fk[jt];
            if (s + 1 < DKS) fk[jt] = read_rows<T, KB>(tk, jt * 16, s + 1);
            if (jt <= wave) p[jt] = M::mma(now, fq, p[jt]);
          }
          fq = nq;
          __builtin_amdgcn_sched_barrier(0);
        }
        const int i = wave * 16 + l16;
        const float hi = st.hi[i], lo = st.lo[i];
#pragma unroll
        for (int jt = 0; jt < IT; ++jt) {
          if (jt > (sizeof(T) == 2 ? wave | 1 : wave)) continue;  // a step of the product with v that no token of the wave's has
          const f32x4 hj = *(const f32x4*)&st.hi[jt * 16 + g * 4], lj = *(const f32x4*)&st.lo[jt * 16 + g * 4];
          const f32x4 dj = *(const f32x4*)&st.dt[jt * 16 + g * 4];
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float w = __builtin_amdgcn_exp2f((hi - hj[e]) + (lo - lj[e])) * dj[e];
            x[e] = jt * 16 + g * 4 + e <= i ? p[jt][e] * w : 0.f;
          }
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int n = 0; n < M::P_TERMS; ++n) {
              const unsigned w0 = pack_bf16(x[0], x[1]), w1 = pack_bf16(x[2], x[3]);
              *(u32x2*)(tp + n * C * PB + tile_at<PB>(i, jt * 2 + g / 2) + (g & 1) * 8) = (u32x2){w0, w1};
              x[0] -= unpack<T>(w0, 0);
              x[1] -= unpack<T>(w0, 1);
              x[2] -= unpack<T>(w1, 0);
              x[3] -= unpack<T>(w1, 1);
            }
          } else {
            *(f32x4*)(tp + tile_at<PB>(i, jt * 4 + g)) = (f32x4){x[0], x[1], x[2], x[3]};
          }
        }
      }
      // What the state before the chunk gives: columns of the wave, all tokens
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int c = 0; c < NC; ++c) O[i][c] = f32x4{};
      Frag nq[IT];
#pragma unroll
      for (int i = 0; i < IT; ++i) nq[i] = read_rows<T, KB>(tq, i * 16, 0);
#pragma unroll
      for (int s = 0; s < DKS; ++s) {
        Frag fs[NC][M::STATE_TERMS], fq[IT];
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          fq[i] = nq[i];
          if (s + 1 < DKS) nq[i] = read_rows<T, KB>(tq, i * 16, s + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if constexpr (sizeof(T) == 2) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = S[2 * s + e / 4][c][e % 4];
            split8(x, fs[c]);
          } else {
            fs[c][0] = S[s][c];
          }
        }
#pragma unroll
        for (int n = 0; n < M::STATE_TERMS; ++n)
#pragma unroll
          for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int c = 0; c < NC; ++c) O[i][c] = M::mma(fs[c][n], fq[i], O[i][c]);
        __builtin_amdgcn_sched_barrier(0);  // one step's operands ahead
      }
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const float grown = st.grown[i * 16 + l16];
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) O[i][c][e] *= grown;
      }
    }

    // The chunk's tokens to the state; their v stays in registers
    const float decay = st.end;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[d][c][e] *= decay;
    Frag fv[CKS][NC], nk[2];
    const auto read_k = [&](int s, int d) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) nk[h] = read_cols<T, KB, 8>(tk, s, sizeof(T) == 2 ? d / 2 * 32 + h * 4 : (d + h) * 16);
    };
    read_k(0, 0);
#pragma unroll
    for (int s = 0; s < CKS; ++s)
#pragma unroll
      for (int c = 0; c < NC; ++c) fv[s][c] = read_cols<T, VB, 4>(tv, s, wave * 16 * NC + 16 * c);
#pragma unroll
    for (int s = 0; s < CKS; ++s) {
      constexpr int E = KS / 4;
      Frag fw[NC][M::V_TERMS];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (float)fv[s][c][e] * st.weight[s * KS + g * E + e];
        if constexpr (sizeof(T) == 2) split8(x, fw[c]);
        else fw[c][0] = (f32x4){x[0], x[1], x[2], x[3]};
      }
#pragma unroll
      for (int d = 0; d < DT; d += 2) {
        const Frag fk[2] = {nk[0], nk[1]};
        if (d + 2 < DT) read_k(s, d + 2);
        else if (s + 1 < CKS) read_k(s + 1, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < M::V_TERMS; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[d + h][c] = M::mma(fk[h], fw[c][n], S[d + h][c]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (OUT) {
      // What is infinite or NaN is added by itself, to the tokens from its own on: a product with the
      // weight 0 of an earlier one would be NaN
      bool odd = false;
#pragma unroll
      for (int s = 0; s < CKS; ++s)
#pragma unroll
        for (int c = 0; c < NC; ++c) odd |= any_wild(fv[s][c]);
      odd = __ballot(odd) != 0;
      if (odd) {
#pragma unroll
        for (int s = 0; s < CKS; ++s)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < KS / 4; ++e)
              if (!(__builtin_fabsf((float)fv[s][c][e]) < __builtin_inff())) fv[s][c][e] = 0;
      }
      __syncthreads();  // the weights are there, and q, k and v have been read
      if (next < end) fill(next, 0);

      // The tokens of the chunk to the outputs behind them
#pragma unroll
      for (int s = 0; s < CKS; ++s)
#pragma unroll
        for (int n = 0; n < M::P_TERMS; ++n)
#pragma unroll
          for (int i = s * KS / 16; i < IT; ++i) {
            const Frag fp = read_rows<T, PB>(tp + n * C * PB, i * 16, s);
#pragma unroll
            for (int c = 0; c < NC; ++c) O[i][c] = M::mma(fv[s][c], fp, O[i][c]);
          }
      if (odd) {
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll 1
            for (int j = 0; j <= i * 16 + l16 && t + j < end; ++j) {
              const int row = i * 16 + l16, col = (wave * NC + c) * 16 + g * 4;
              float p = 0;
#pragma unroll
              for (int n = 0; n < M::P_TERMS; ++n)
                p += (float)*(const T*)(tp + n * C * PB + tile_at<PB>(row, j * (int)sizeof(T) / 16) + j * (int)sizeof(T) % 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (col + e >= cols) break;
                const float x = (float)v[(t + j) * a.ldv + col + e];
                if (!(__builtin_fabsf(x) < __builtin_inff())) O[i][c][e] += p * x;
              }
            }
      }
      // Rows and columns past the last have an offset past the buffer
      const __amdgpu_buffer_rsrc_t ro = make_rsrc((T*)a.o + t * a.ldo + (int64_t)head * a.value,
                                                  ((min(end - t, C) - 1) * a.ldo + a.value) * (int64_t)sizeof(T));
#pragma unroll
      for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int col = cw + 16 * c + g * 4;
          const unsigned off = (unsigned)((i * 16 + l16) * (int)a.ldo + col) * (unsigned)sizeof(T);
          const bool row = t + i * 16 + l16 < end;
          if constexpr (ALIGNED) {
            const unsigned at = row && col < a.value ? off : kOobGroup;
            if constexpr (sizeof(T) == 2)
              __builtin_amdgcn_raw_buffer_store_b64((u32x2){pack_bf16(O[i][c][0], O[i][c][1]), pack_bf16(O[i][c][2], O[i][c][3])},
                                                    ro, (int)at, 0, 0);
            else
              __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, O[i][c]), ro, (int)at, 0, 0);
          } else if (row && col + 4 <= a.value) {
            store_quad4((T*)a.o + (t + i * 16 + l16) * a.ldo + (int64_t)head * a.value + col, (const float*)&O[i][c], false);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              store_elem<T>(ro, row && col + e < a.value ? off + e * (unsigned)sizeof(T) : kOobGroup, 0, O[i][c][e]);
          }
        }
    }
    t = next;
  }

  if constexpr (!OUT) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) frames[(t * NC + c) * 64] = S[t][c];
    if (threadIdx.x == 0 && blockIdx.y == 0)
      a.decays[(int64_t)unit * a.heads + head] = __builtin_amdgcn_exp2f((float)total);
  } else if (last && slot >= 0 && a.state_out) {
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.state_out + state_at, state_bytes);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          store_elem<float>(rs, state_off[c] == kOobGroup ? kOobGroup : state_off[c] + (unsigned)((row_of(t) + e) * a.value) * 4, 0, S[t][c][e]);
  }
}

// Every piece's state at its end, from zeros (a sequence's first: from its own state), to the state
// before each piece. The place of the last one, whose end nobody needs, holds the sequence's own state
// until then.
__global__ void __launch_bounds__(256) decay_join_kernel(DecayArgs a) {
  const int s = fdiv((int)blockIdx.x, a.dheads), head = (int)blockIdx.x - s * a.heads;
  const int at = (int)blockIdx.y * 256 + (int)threadIdx.x;
  const SeqRange r = seq_range(a.seqs, s);
  const int pieces = tiles_in(r.end - r.begin, a.piece);
  const int64_t unit = a.seqs.offsets ? first_tile(r.begin, a.piece, s) : (int64_t)s * a.per;
  if (at >= a.frames || pieces < 2) return;
  const int64_t step = (int64_t)a.heads * a.frames;
  f32x4* p = a.ends + (unit * a.heads + head) * a.frames + at;
  const float* decay = a.decays + unit * a.heads + head;
  constexpr int AHEAD = 8;
  f32x4 run = *p;
  *p = p[(pieces - 1) * step];
  for (int i = 1; i < pieces; i += AHEAD) {  // pieces i to i + 7: their ends all on their way, the last one's not needed
    f32x4 end[AHEAD];
    float d[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) {
      const int from = min(i + n, pieces - 2);
      end[n] = p[from * step];
      d[n] = decay[(int64_t)from * a.heads];
    }
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) {
      if (i + n >= pieces) break;
      p[(i + n) * step] = run;
      run = end[n] + run * d[n];
    }
  }
}

// Whether rows can be read and written 16 bytes at a time.
static bool decay_aligned(const DecayArgs& a, int e) {
  const int64_t on = (int64_t)((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.o) | a.ldq * e | a.ldk * e |
                     a.ldv * e | a.ldo * e | (int64_t)a.key * e | (int64_t)a.value * e;
  return on % 16 == 0;
}
struct DecayShape {
  int dk, nc, slices, frames;
};
static DecayShape decay_shape(int key, int value) {
  const int dk = key <= 64 ? 64 : key <= 128 ? 128 : 256, nc = value <= 64 || dk == 256 ? 1 : 2;
  const int slices = (value + 64 * nc - 1) / (64 * nc);
  return {dk, nc, slices, slices * 64 * nc * dk / 4};
}
template <typename T, int DK, int NC, bool OUT>
static int decay_tiles(const DecayArgs& a, dim3 blocks, hipStream_t st) {
  constexpr int C = Mat<T>::CHUNK, e = (int)sizeof(T);
  constexpr size_t lds = OUT ? C * (2 * DK * e + 64 * NC * e + Mat<T>::P_TERMS * C * e) : 2 * C * (DK * e + 64 * NC * e);
  return decay_aligned(a, e) ? launch(decay_tile_kernel<T, DK, NC, OUT, true>, blocks, 256, lds, st, a)
                             : launch(decay_tile_kernel<T, DK, NC, OUT, false>, blocks, 256, lds, st, a);
}
template <typename T, bool OUT>
static int decay_tiles(const DecayArgs& a, const DecayShape& s, dim3 blocks, hipStream_t st) {
  switch (s.dk) {
    case 64: return s.nc == 1 ? decay_tiles<T, 64, 1, OUT>(a, blocks, st) : decay_tiles<T, 64, 2, OUT>(a, blocks, st);
    case 128: return s.nc == 1 ? decay_tiles<T, 128, 1, OUT>(a, blocks, st) : decay_tiles<T, 128, 2, OUT>(a, blocks, st);
    default: return decay_tiles<T, 256, 1, OUT>(a, blocks, st);
  }
}
template <typename T>
static int decay_prompt(const DecayArgs& a, int64_t units, hipStream_t st) {
  const DecayShape s = decay_shape(a.key, a.value);
  const int64_t blocks = units * a.heads;
  if (!fits_launch(blocks, 256) || !fits_launch((int64_t)a.seqs.count * a.heads, 256)) return refuse_size("ct_decay_attention_run");
  const dim3 grid((unsigned)blocks, (unsigned)s.slices);
  if (a.piece) {
    if (const int rc = decay_tiles<T, false>(a, s, grid, st)) return rc;
    const dim3 join((unsigned)((int64_t)a.seqs.count * a.heads), (unsigned)((a.frames + 255) / 256));
    if (const int rc = launch(decay_join_kernel, join, 256, 0, st, a)) return rc;
  }
  return decay_tiles<T, true>(a, s, grid, st);
}

DecayPlan plan_decay(const ct_decay_attention_op& op, const ct_sequences& s) {
  DecayPlan p = {};
  const int longest = !s.offsets ? (s.count ? s.tokens / s.count : 0) : s.max_len ? (s.max_len < s.tokens ? s.max_len : s.tokens) : s.tokens;
  p.step = longest <= kDecayStepTokens;
  if (p.step) return p;
  const DecayShape shape = decay_shape(op.key_dim, op.value_dim);
  // Pieces run every token twice, and a chunk takes two blocks on a compute unit 1.3 times one's
  // time. So whole sequences up to 1.5 times a unit's share of the rows: 16 heads of 128 x 128, 16
  // sequences of 512 tokens 70 us, in pieces of 256 92 us; 8 of 1024 111 and 92; one of 192 22 and 21,
  // of 256 27 and 22. Then pieces that give each unit one block up to 128 tokens, and two above (one
  // sequence of 1024 tokens in pieces of 64 31 us, of 256 47; of 2048 in 64 47, in 128 42, in 256 50;
  // of 4096 in 128 61, in 256 63; of 16384 in 512 148).
  const int64_t share = ((int64_t)s.tokens * op.heads * shape.slices / kPlanCus + 63) / 64 * 64;
  const int64_t one = share < 64 ? 64 : share < 128 ? share : 128, two = (share / 2 + 63) / 64 * 64;
  if (longest > 3 * (share < 128 ? 128 : share) / 2) p.piece = (int)(one > two ? one : two);
  if (!p.piece) return p;
  const SeqView v = {s.offsets, s.slots, s.tokens, s.count, s.num_slots, !s.offsets && s.count ? s.tokens / s.count : 0};
  p.pieces = seq_tiles(v, p.piece).total;
  p.ws_floats = p.pieces * op.heads * ((int64_t)shape.frames * 4 + 1);
  return p;
}

int launch_decay(const ct_decay_attention_op& op, const DecayPlan& p, const SeqView& s, const DecayArrays& v,
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
  hipStream_t st = (hipStream_t)stream;
  if (p.step) return op.dtype == CT_DT_BF16 ? decay_step<bf16_t>(a, st) : decay_step<float>(a, st);
  const int64_t units = p.piece ? p.pieces : s.count;
  a.piece = p.piece;
  a.per = p.piece ? seq_tiles(s, p.piece).per : 0;
  a.frames = decay_shape(op.key_dim, op.value_dim).frames;
  a.ends = (f32x4*)v.ws;
  a.decays = v.ws + (p.piece ? p.pieces * op.heads * a.frames * 4 : 0);
  return op.dtype == CT_DT_BF16 ? decay_prompt<bf16_t>(a, units, st) : decay_prompt<float>(a, units, st);
}

}  // namespace ct
