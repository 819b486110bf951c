// Selective state space scan over packed sequences.
//   h_t[n] = exp(dt_t a[n]) h_{t-1}[n] + dt_t u_t b_t[n],  y_t = (c_t . h_t + d u_t) silu(z_t)
//
// A lane holds NS states of one channel in fp32 registers and walks tokens; P neighbouring
// lanes share a channel of more than NS states. Of a state and token the vector ALU has an
// exponential (measured: 8 clocks of a SIMD for 64 lanes) and four instructions of 4 clocks:
// 24 in all, 82 us for 16384 tokens of 2048 channels of 16 states, against 53 for their bytes.
// So prompts are bound by the vector ALU, and single tokens by the states' bytes.
//
// Where channels and sequences are too few for the device, sequences are cut into chunks:
//   sum:    h at each chunk's end from h = 0 at its start, and the sum of its steps;
//   carry:  h at each chunk's start, chunk after chunk, by
//           h(end) = exp(a * sum of steps) h(start) + h(end from 0);
//   out:    the outputs of each chunk from h at its start.
// That is nearly twice the exponentials, but as many chunks at once as fill the device: the
// 16384 tokens take 235 us (kernels at their fastest: sum 95, carry 23, out 133), whole sequences
// alone 4 ms. The vector ALU is busy 89 % of sum and 85 % of out, with 112 instructions a token
// in out, 80 of them the states'. b and c through scalar registers instead of LDS lost 5 % (no
// room to have the next token's on their way), five waves on a SIMD instead of four spill, and
// the products dt u b as rank-one updates on the matrix cores, 12 vector instructions a token
// fewer, lost 3-4 %.
// Of a few chunks, outputs fold the ends before them and carry is left out: sum then leaves the
// state from state_in in the place of the last chunk's end, which nothing needs.
// Either way state_in is read before any chunk's outputs write state_out, so that both may be
// one array.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "k_seq.h"

namespace ct {

struct ScanArgs {
  SeqView s;
  const void *u, *delta, *b, *c, *z;
  const float *dt_bias, *a, *d_skip, *state_in;
  float *state_out, *ws, *ws_dt;
  void* y;
  int64_t ldu, lddelta, ldb, ldc, ldz, ldy;
  int channels, states, per_group, softplus;
  int stream;         // the states go past the caches
  int vec_bc;         // rows of b and c take accesses of four values
  int per, chunk;     // chunks of a sequence where all are equal, tokens of a chunk
  int fold;           // a chunk's outputs fold the chunks before it; no carries
  FastDiv dtiles, dgroup;  // channel tiles in all, and of one group
};

template <int NS>
struct Vals {
  float v[NS];
};
// NS values from p on, 0 for those past `left`. vec: rows lie on 16-byte addresses and end on
// a multiple of four values.
template <int NS>
__device__ __forceinline__ Vals<NS> load_vals(const float* p, int left, bool vec) {
  Vals<NS> r;
  if (vec && NS % 4 == 0) {
#pragma unroll
    for (int i = 0; i < NS; i += 4) {
      f32x4 q = {};
      if (i < left) q = *(const f32x4*)(p + i);
      r.v[i] = q.x; r.v[i + 1] = q.y; r.v[i + 2] = q.z; r.v[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NS; ++i) r.v[i] = i < left ? p[i] : 0.f;
  }
  return r;
}
template <int NS>
__device__ __forceinline__ void store_vals(float* p, const float (&v)[NS], int left, bool vec, bool stream) {
  if (vec && NS % 4 == 0) {
#pragma unroll
    for (int i = 0; i < NS; i += 4)
      if (i < left) store_once((f32x4*)(p + i), (f32x4){v[i], v[i + 1], v[i + 2], v[i + 3]}, stream);
  } else {
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (i < left) p[i] = v[i];
  }
}
__device__ __forceinline__ bool rows_of_four(const void* p, int states) {
  return ((uintptr_t)p % 16 | (unsigned)states % 4) == 0;
}
// The sum over P neighbouring lanes, in all of them: pairs and quads by permutation, then the
// other quad and the other eight of a row of 16 by mirroring, whose lanes hold equal sums.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int P>
__device__ __forceinline__ float add_lanes(float v) {
  if constexpr (P > 1) v = add_dpp<0xB1>(v);   // quad_perm [1, 0, 3, 2]
  if constexpr (P > 2) v = add_dpp<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  if constexpr (P > 4) v = add_dpp<0x141>(v);  // row_half_mirror
  if constexpr (P > 8) v = add_dpp<0x140>(v);  // row_mirror
  return v;
}

// A state over a whole chunk: exp2(x) h + end, as it comes token by token. The factor is that of
// half of x, twice, so that it does not leave fp32 where its product with h would not, and kept
// finite and above 0, so that a state of 0 stays 0 and an infinite one infinite.
__device__ __forceinline__ float over_chunk(float half_x, float h, float end) {
  const float f = __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(half_x), 0x1p-126f, 0x1p127f);
  return fmaf(f * h, f, end);  // where x is NaN, so is the end
}

// ------------------------------------------------------------------ prompts
enum ScanMode { SCAN_WHOLE, SCAN_SUM, SCAN_OUT };

// Four waves walk a chunk (or a whole sequence) for 4 * 64 / P channels of one group. b and c
// of TT tokens are staged in LDS in fp32, where all channels read them; the next ones are on
// their way meanwhile.
template <typename T, int NS, int P, int MODE>
__global__ void __launch_bounds__(256) scan_kernel(ScanArgs a) {
  constexpr int CH = 64 / P, NP = NS * P, TT = NP <= 16 ? 32 : NP <= 64 ? 16 : 4;
  // Tokens whose rows are on their way while as many are walked: a wave that is nearly alone on
  // its SIMD waits for them (32 x 512 tokens of 4096 channels, whole: four 321 us, eight 287,
  // 16 280 and slower with more waves). The outputs of chunks keep a fourth wave instead.
  constexpr int U = TT > 4 && MODE != SCAN_OUT ? 8 : 4;
  constexpr int STAGED = TT * NP / 256 ? TT * NP / 256 : 1;  // values of b (and of c) that a thread stages
  __shared__ __align__(16) float sb[2][TT][NP], sc[MODE == SCAN_SUM ? 1 : 2][MODE == SCAN_SUM ? 1 : TT][NP];

  const int id = fdiv((int)blockIdx.x, a.dtiles), tile = (int)blockIdx.x - id * a.dtiles.d;
  const int group = fdiv(tile, a.dgroup), in_group = ((tile - group * a.dgroup.d) * 4 + wave_id()) * CH;
  int t0, t1;
  SeqRange r;
  if constexpr (MODE == SCAN_WHOLE) {
    r = seq_range(a.s, id);
    t0 = r.begin;
    t1 = r.end;
  } else {
    r = find_tile(a.s, a.per, a.chunk, id, &t0);
    const bool hands_on = MODE == SCAN_OUT && a.fold && r.begin == r.end && t0 == r.begin;  // an empty sequence
    if (r.s < 0 || (t0 >= r.end && !hands_on)) return;
    t1 = tile_end(t0, r.end, a.chunk);
    if (MODE == SCAN_SUM && t1 == r.end && !a.fold) return;  // nothing follows this chunk
  }
  t0 = __builtin_amdgcn_readfirstlane(t0);
  t1 = __builtin_amdgcn_readfirstlane(t1);
  const int lane = (int)threadIdx.x & 63, part = lane % P, ch = in_group + lane / P;
  const bool live = ch < a.per_group;
  const int d = group * a.per_group + (live ? ch : a.per_group - 1), n0 = part * NS;  // spare lanes repeat a channel
  const int left = a.states - n0;

  // Lanes have NP states. Those past the last one repeat states from the first on, so that no
  // product in them is NaN where the state's own is not (of an infinite step or input and a
  // state of zeros it would be), and c of a copy is small enough to add nothing that counts.
  const bool spare = a.states < NP;
  const float inv = spare ? 1.f / (float)a.states : 0.f;
  // Arrays of channels x states from uniform addresses on, which leaves the lanes one offset: at
  // most 2^31 bytes, for rows of u hold 2^21 channels at most.
  const unsigned at = ((unsigned)d * (unsigned)a.states + (unsigned)n0) * 4u;
  auto load_states = [&](const float* all, bool vec) __attribute__((always_inline)) {
    if (!spare) return load_vals<NS>((const float*)((const char*)all + at), NS, vec);
    Vals<NS> r;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      r.v[i] = *(const float*)((const char*)all + (at + (unsigned)(i - qdiv(n0 + i, inv) * a.states) * 4u));
    return r;
  };
  auto store_states = [&](float* all, const Vals<NS>& v, bool vec) __attribute__((always_inline)) {
    store_vals<NS>((float*)((char*)all + at), v.v, left, vec, false);
  };

  Vals<NS> la = load_states(a.a, rows_of_four(a.a, a.states));
#pragma unroll
  for (int i = 0; i < NS; ++i) la.v[i] *= kLog2e;
  const int slot = MODE == SCAN_SUM && !a.fold ? -1 : __builtin_amdgcn_readfirstlane(seq_slot(a.s, r.s));
  const int64_t per_chunk = (int64_t)a.channels * a.states, in_state = slot * per_chunk, in_ws = id * per_chunk;
  Vals<NS> h = {};
  const bool vec_ws = rows_of_four(a.ws, a.states);
  if (MODE == SCAN_WHOLE || (MODE == SCAN_SUM ? a.fold && t1 == r.end : t0 == t1)) {
    if (slot >= 0 && a.state_in) h = load_states(a.state_in + in_state, rows_of_four(a.state_in, a.states));
    if constexpr (MODE == SCAN_SUM) {
      if (live) store_states(a.ws + in_ws, h, vec_ws);
      return;
    }
  } else if constexpr (MODE == SCAN_OUT) {
    const int before = a.fold ? (t0 - r.begin) / a.chunk : 0;
    const int at_start = a.fold ? (r.end - t0 - 1) / a.chunk : 0;  // chunks up to the last
    h = load_states(a.ws + in_ws + at_start * per_chunk, vec_ws);
    constexpr int F = NS <= 4 ? 8 : 2;
    const float *end = a.ws + in_ws - before * per_chunk, *sum = a.ws_dt + (int64_t)(id - before) * a.channels + d;
    for (int k = 0; k < before; k += F) {
      Vals<NS> e[F];
      float dt[F];
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const int c = min(k + i, before - 1);
        // lanes of more than four states have none to spare here (plan_scan)
        if constexpr (NS <= 4) e[i] = load_states(end + c * per_chunk, vec_ws);
        else e[i] = load_vals<NS>((const float*)((const char*)(end + c * per_chunk) + at), NS, vec_ws);
        dt[i] = 0.5f * sum[(int64_t)c * a.channels];
      }
#pragma unroll
      for (int i = 0; i < F; ++i)
        if (k + i < before)
#pragma unroll
          for (int n = 0; n < NS; ++n) h.v[n] = over_chunk(dt[i] * la.v[n], h.v[n], e[i].v[n]);
    }
  }
  const float bias = a.dt_bias ? a.dt_bias[d] : 0.f, skip = a.d_skip ? a.d_skip[d] : 0.f;
  float total = 0.f;

  // staging: a thread's values are all of one state
  T kb[STAGED], kc[STAGED];
  const int nb = (int)threadIdx.x % NP, copies = spare ? qdiv(nb, inv) : 0;
  const float weight = copies ? 0x1p-28f : 1.f;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    int at_n = nb - copies * a.states;
    asm volatile("" : "+v"(at_n));  // or addresses are held from stage to stage, and waves on a SIMD are fewer
    at_n += group * a.states;
#pragma unroll
    for (int i = 0; i < STAGED; ++i) {
      const int row = (i * 256 + (int)threadIdx.x) / NP;
      const bool ok = row < TT && t + row < t1;
      const int64_t tok = ok ? t + row : t0;
      const T vb = ((const T*)a.b)[tok * a.ldb + at_n];
      kb[i] = ok ? vb : (T)0.f;
      if constexpr (MODE != SCAN_SUM) {
        const T vc = ((const T*)a.c)[tok * a.ldc + at_n];
        kc[i] = ok ? vc : (T)0.f;
      }
    }
  };
  auto put = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < STAGED; ++i) {
      const int e = i * 256 + (int)threadIdx.x;
      if (TT * NP >= 256 || e < TT * NP) {
        (&sb[s][0][0])[e] = (float)kb[i];
        if constexpr (MODE != SCAN_SUM) (&sc[s][0][0])[e] = (float)kc[i] * weight;
      }
    }
  };
  // The next U tokens of this lane's channel, from rows that start with the stage's; past the
  // last token the last row again. Lanes that store nothing have an offset past every row.
  constexpr int E = (int)sizeof(T);
  const unsigned off = (unsigned)d * (unsigned)E, off_y = part == 0 && live ? off : kOob;
  const int step_u = (int)a.ldu * E, step_d = (int)a.lddelta * E, step_z = (int)a.ldz * E, step_y = (int)a.ldy * E;
  __amdgpu_buffer_rsrc_t ru, rd, rz, ry;
  int rows = 0;
  auto aim = [&](int t) __attribute__((always_inline)) {
    rows = min(t1 - t, TT + U);
    ru = rows_rsrc((const T*)a.u + t * a.ldu, rows, a.ldu, a.channels);
    rd = rows_rsrc((const T*)a.delta + t * a.lddelta, rows, a.lddelta, a.channels);
    if constexpr (MODE != SCAN_SUM) {
      rz = rows_rsrc((const T*)a.z + t * a.ldz, a.z ? rows : 1, a.ldz, a.z ? a.channels : 0);
      ry = rows_rsrc((const T*)a.y + t * a.ldy, rows, a.ldy, a.channels);
    }
  };
  float ku[U], kd[U], kz[U];
  auto fetch_rows = [&](int q) __attribute__((always_inline)) {
    auto go = [&](auto row) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        ku[i] = load_elem<T>(ru, off, row(q + i) * step_u);
        kd[i] = load_elem<T>(rd, off, row(q + i) * step_d);
      }
      if (MODE != SCAN_SUM && a.z)
#pragma unroll
        for (int i = 0; i < U; ++i) kz[i] = load_elem<T>(rz, off, row(q + i) * step_z);
    };
    go([&](int r) __attribute__((always_inline)) { return row_or_last(r, rows); });
  };

  if (t0 < t1) {
    fetch(t0);
    aim(t0);
    fetch_rows(0);
    for (int t = t0, s = 0; t < t1; t += TT, s ^= 1) {
      put(s);
      __syncthreads();  // also: every wave is done with the stage before last
      if (t + TT < t1) fetch(t + TT);
      if (t > t0) aim(t);
      auto tokens = [&](int q, auto all) __attribute__((always_inline)) {
        float dt[U], du[U], u[U], z[U];
        auto each = [](auto f) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < U; ++i) f(i);
        };
        each([&](int i) {
          u[i] = ku[i];
          dt[i] = kd[i] + bias;
          z[i] = 1.f;
        });
        if (a.softplus) each([&](int i) { dt[i] = softplus_f32(dt[i]); });
        if (MODE != SCAN_SUM && a.z) each([&](int i) { z[i] = silu_f32(kz[i]); });
        each([&](int i) { du[i] = dt[i] * u[i]; });
        fetch_rows(q + U);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (!all.value && t + q + i >= t1) break;
          float y = 0.f;
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            h.v[n] = fmaf(__builtin_amdgcn_exp2f(dt[i] * la.v[n]), h.v[n], du[i] * sb[s][q + i][n0 + n]);
            if constexpr (MODE != SCAN_SUM) y = fmaf(sc[s][q + i][n0 + n], h.v[n], y);
          }
          if constexpr (MODE == SCAN_SUM) {
            total += dt[i];
          } else {
            y = fmaf(skip, u[i], add_lanes<P>(y)) * z[i];
            store_elem<T>(ry, off_y, (q + i) * step_y, y);
          }
        }
      };
#pragma unroll 1
      for (int q = 0; q < TT && t + q < t1; q += U) {
        if (t + q + U <= t1) tokens(q, std::true_type{});
        else tokens(q, std::false_type{});
      }
    }
  }
  if (!live) return;
  if constexpr (MODE == SCAN_SUM) {
    store_states(a.ws + in_ws, h, vec_ws);
    if (part == 0) a.ws_dt[(int64_t)id * a.channels + d] = total;
  } else if (slot >= 0 && a.state_out && t1 == r.end) {
    store_states(a.state_out + in_state, h, rows_of_four(a.state_out, a.states));
  }
}

// h at the start of every chunk, in place of h at its end from 0. A lane has one state of one
// channel; the loads of the next eight to 16 chunks are on their way while it walks (with
// eight and none ahead 256 chunks of 32768 states took 34 us, 13 % of their scan; now 22).
// An empty sequence hands its state on.
__global__ void __launch_bounds__(64) scan_carry_kernel(ScanArgs a) {
  const int64_t per_seq = (int64_t)a.channels * a.states;
  const int blocks = (int)((per_seq + 63) / 64);
  const int s = (int)(blockIdx.x / blocks);
  const int64_t e = (int64_t)(blockIdx.x % blocks) * 64 + threadIdx.x;
  if (e >= per_seq) return;
  const int d = (int)(e / a.states);
  const SeqRange r = seq_range(a.s, s);
  const int slot = seq_slot(a.s, s);
  const int n = __builtin_amdgcn_readfirstlane(tiles_in(r.end - r.begin, a.chunk));
  const int64_t id = a.s.offsets ? r.begin / a.chunk + s : (int64_t)s * a.per;
  float h = slot >= 0 && a.state_in ? a.state_in[(int64_t)slot * per_seq + e] : 0.f;
  if (n == 0) {
    if (slot >= 0 && a.state_out) a.state_out[(int64_t)slot * per_seq + e] = h;
    return;
  }
  const float half_la = a.a[e] * (0.5f * kLog2e);
  float* p = a.ws + id * per_seq + e;
  const float* dt = a.ws_dt + id * a.channels + d;
  constexpr int F = 8;
  float end[2][F], sum[2][F];
  auto fetch = [&](int u, int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < F; ++i) {
      const int k = min(c + i, n - 2);  // the last chunk's end is nobody's start
      end[u][i] = p[(int64_t)k * per_seq];
      sum[u][i] = dt[(int64_t)k * a.channels];
    }
  };
  auto walk = [&](int u, int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < F; ++i)
      if (c + i < n - 1) {
        p[(int64_t)(c + i) * per_seq] = h;
        h = over_chunk(half_la * sum[u][i], h, end[u][i]);
      }
  };
  if (n > 1) {
    fetch(0, 0);
    for (int c = 0; c < n - 1; c += 2 * F) {
      fetch(1, c + F);
      walk(0, c);
      fetch(0, c + 2 * F);
      walk(1, c + F);
    }
  }
  p[(int64_t)(n - 1) * per_seq] = h;
}

// ------------------------------------------------------------------ single tokens
// One token of each sequence: a wave updates 64 / P channels of SEQ sequences, whose loads are
// all on their way together; a, the bias and the skip weight are read once for them. Four
// states a lane make every access to the states one of 1 KB: 256 sequences of 4096 channels
// of 16 states (67 MB read, 67 MB written) 25.4 us, 5.6 TB/s; one sequence a wave 30 us, 16
// states a lane 45 (of which the stores through the caches are 10).
template <typename T, int NS, int P, int SEQ>
__global__ void __launch_bounds__(256) scan_step_kernel(ScanArgs a) {
  static_assert(NS % 4 == 0, "");
  constexpr int CH = 64 / P;
  const int64_t g = (int64_t)blockIdx.x * 4 + wave_id();
  if (g >= (int64_t)((a.s.count + SEQ - 1) / SEQ) * a.dtiles.d) return;
  const int first = fdiv((int)g, a.dtiles) * SEQ, tile = (int)g - first / SEQ * a.dtiles.d;
  const int group = fdiv(tile, a.dgroup), in_group = (tile - group * a.dgroup.d) * CH;
  const int lane = (int)(threadIdx.x & 63), part = lane % P, ch = in_group + lane / P;
  if (ch >= a.per_group) return;
  const int d = group * a.per_group + ch, n0 = part * NS, left = a.states - n0;
  const int64_t in_row = (int64_t)group * a.states;
  const bool vec = rows_of_four(a.state_in, a.states) && rows_of_four(a.state_out, a.states);

  // what does not wait for the slots goes first
  int slot[SEQ];
  Vals<NS> h[SEQ], b[SEQ], c[SEQ];
  float u[SEQ], dt[SEQ], z[SEQ];
#pragma unroll
  for (int q = 0; q < SEQ; ++q) {
    const int t = min(first + q, a.s.count - 1);
    u[q] = (float)((const T*)a.u + t * a.ldu)[d];
    dt[q] = (float)((const T*)a.delta + t * a.lddelta)[d];
    z[q] = a.z ? (float)((const T*)a.z + t * a.ldz)[d] : 0.f;
    const T *pb = (const T*)a.b + t * a.ldb + in_row, *pc = (const T*)a.c + t * a.ldc + in_row;
#pragma unroll
    for (int i = 0; i < NS; i += 4) {
      if (a.vec_bc) {
        const bool in = i < left;
        const int col = quad_column(n0 + i, a.states);
        const Quad qb = load_quad4(pb + col), qc = load_quad4(pc + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          b[q].v[i + e] = in ? qb.v[e] : 0.f;
          c[q].v[i + e] = in ? qc.v[e] : 0.f;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = i + e < left;
          b[q].v[i + e] = in ? (float)pb[n0 + i + e] : 0.f;
          c[q].v[i + e] = in ? (float)pc[n0 + i + e] : 0.f;
        }
      }
    }
  }
  Vals<NS> la = load_vals<NS>(a.a + (int64_t)d * a.states + n0, left, rows_of_four(a.a, a.states));
  const float bias = a.dt_bias ? a.dt_bias[d] : 0.f, skip = a.d_skip ? a.d_skip[d] : 0.f;
#pragma unroll
  for (int q = 0; q < SEQ; ++q) slot[q] = first + q < a.s.count ? seq_slot(a.s, first + q) : -1;
#pragma unroll
  for (int q = 0; q < SEQ; ++q) {
    h[q] = {};
    if (slot[q] >= 0 && a.state_in)
      h[q] = load_vals<NS>(a.state_in + ((int64_t)slot[q] * a.channels + d) * a.states + n0, left, vec);
  }
#pragma unroll
  for (int q = 0; q < SEQ; ++q) {
    const float v = dt[q] + bias, step = a.softplus ? softplus_f32(v) : v, du = step * u[q];
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      h[q].v[i] = fmaf(__builtin_amdgcn_exp2f(step * (la.v[i] * kLog2e)), h[q].v[i], du * b[q].v[i]);
      y = i < left ? fmaf(c[q].v[i], h[q].v[i], y) : y;  // past the last state h may be NaN
    }
    y = fmaf(skip, u[q], add_lanes<P>(y));
    if (a.z) y *= silu_f32(z[q]);
    if (first + q < a.s.count && part == 0) ((T*)a.y + (first + q) * a.ldy)[d] = from_f32<T>(y);
    if (slot[q] >= 0 && a.state_out)
      store_vals<NS>(a.state_out + ((int64_t)slot[q] * a.channels + d) * a.states + n0, h[q].v, left, vec, a.stream);
  }
}

// ------------------------------------------------------------------ plans and launches
// Lanes that share a channel of a prompt: 16 states a lane, or four where that leaves the
// device idle.
static int prompt_parts(int states, bool narrow) {
  int parts = 1;
  while (parts * (narrow ? 4 : 16) < states) parts *= 2;
  return narrow && parts < 4 ? 4 : parts;
}

ScanPlan plan_scan(const ct_scan_op& op, const ct_sequences& s) {
  ScanPlan p = {};
  if (!s.tokens) return p;
  const int most = s.offsets ? (s.max_len ? (s.max_len < s.tokens ? s.max_len : s.tokens) : s.tokens) : s.tokens / s.count;
  const double simds = 4 * kPlanCus;
  auto waves_of = [&](bool narrow) {  // of a chunk
    const int ch = 64 / prompt_parts(op.states, narrow), per_group = op.channels / op.groups;
    return (int64_t)op.groups * ((per_group + ch - 1) / ch);
  };
  // 16 states a lane (8 where a channel has no more) or four, cut or whole: what takes the
  // fewest us by fits to bf16 (1 to 128 sequences of 32 to 2048 tokens and 300 to 4096 channels
  // of 8 to 64 states; the choice is the fastest or within 5 % of it), which decide for fp32 and
  // for more states too, where nothing was fitted. A SIMD with n waves gives
  // each a token in token + wave n, its vector ALU one in full, and the longest sequence takes
  // as many; cut, all tokens are walked twice at the full rate, by three kernels. whole / cut of
  // 16 states: 32 x 512 tokens of 4096 channels 287 / 444, in fours 483 / 495; 8 x 128 of 2048:
  // 52 / 37, in fours 33 / 41; 1 x 256 of 2048: 90 / 29, in fours 53 / 21.
  struct Fit { double token, wave, full, cut, cut_token; };
  const Fit wide = op.states <= 8 ? Fit{0.2, 0.11, 0.2, 20, 0.29} : Fit{0.29, 0.13, 0.25, 26, 0.42};
  const Fit four = {0.17, 0.09, 0.09, 16, 0.19};
  double least = 1e300;
  bool cut = false;
  for (const bool narrow : {false, true}) {
    if (narrow && op.states > 64) break;
    const double per_simd = (double)s.tokens * (double)waves_of(narrow) / simds;
    const Fit& f = narrow ? four : wide;
    double whole = f.token * most + f.wave * per_simd;
    if (whole < f.full * per_simd + 0.03 * most) whole = f.full * per_simd + 0.03 * most;
    whole += 4;
    const double chunks = f.cut + f.cut_token * per_simd;
    if (whole < least) least = whole, p.narrow = narrow, cut = false;
    if (chunks < least) least = chunks, p.narrow = narrow, cut = true;
  }
  if (!cut) return p;
  // As many tokens in a chunk as leave eight blocks of four waves for every compute unit:
  // those at work together take turns evenly, and the last ones are short (a third of them:
  // 8192 ragged tokens of 4096 channels 246 to 275 us). Whole stages of 32.
  int64_t chunk = ((int64_t)s.tokens * waves_of(p.narrow) / (8 * 4 * kPlanCus) + 16) / 32 * 32;
  if (chunk < 32) chunk = 32;
  p.chunk = (int)chunk;
  // Up to eight chunks of a sequence: folding saves 2.7 us. Of 16 it takes as long as the
  // carries (1 x 512 tokens of 2048 channels 24 and 27 us, 8 x 512 81 and 76), of more longer.
  // Where lanes of eight or 16 states have some to spare, the repeated ones' ends would cost
  // the outputs a wave of four on a SIMD.
  const int lanes_states = p.narrow || op.states > 8 ? (p.narrow ? 4 : 16) * prompt_parts(op.states, p.narrow) : 8;
  p.fold = most <= 8 * chunk && (p.narrow || op.states == lanes_states);
  p.chunks = s.offsets ? s.tokens / chunk + s.count : (int64_t)s.count * ((most + chunk - 1) / chunk);
  p.ws_floats = p.chunks * op.channels * (op.states + 1);
  return p;
}

template <typename T, int NS, int P, int MODE>
static int scan_launch(ScanArgs a, int64_t pieces, hipStream_t st) {
  constexpr int CH = 4 * 64 / P;
  const int per = (a.per_group + CH - 1) / CH;
  const int64_t tiles = (int64_t)per * (a.channels / a.per_group), blocks = tiles * pieces;
  if (!fits_launch(blocks, 256)) return refuse_size("ct_scan_run");
  a.dgroup = make_fastdiv(per);
  a.dtiles = make_fastdiv(tiles);
  return launch(scan_kernel<T, NS, P, MODE>, dim3((unsigned)blocks), 256, 0, st, a);
}
template <typename T, int NS, int P>
static int scan_prompt(ScanArgs a, const ScanPlan& p, hipStream_t st) {
  if (!p.chunk) return scan_launch<T, NS, P, SCAN_WHOLE>(a, a.s.count, st);
  a.chunk = p.chunk;
  a.fold = p.fold;
  a.per = a.s.offsets ? 0 : tiles_in(a.s.len, p.chunk);
  a.ws_dt = a.ws + p.chunks * a.channels * a.states;
  int rc = scan_launch<T, NS, P, SCAN_SUM>(a, p.chunks, st);
  if (rc) return rc;
  if (!p.fold) {
    const int64_t blocks = (((int64_t)a.channels * a.states + 63) / 64) * a.s.count;
    if (!fits_launch(blocks, 64)) return refuse_size("ct_scan_run");
    if ((rc = launch(scan_carry_kernel, dim3((unsigned)blocks), 64, 0, st, a))) return rc;
  }
  return scan_launch<T, NS, P, SCAN_OUT>(a, p.chunks, st);
}
template <typename T, int NS, int P, int SEQ>
static int step_launch(ScanArgs a, hipStream_t st) {
  constexpr int CH = 64 / P;
  const int per = (a.per_group + CH - 1) / CH;
  const int64_t tiles = (int64_t)per * (a.channels / a.per_group), waves = tiles * ((a.s.count + SEQ - 1) / SEQ);
  if (waves > 0x7FFFFFF0 || !fits_launch((waves + 3) / 4, 256)) return refuse_size("ct_scan_run");
  a.dgroup = make_fastdiv(per);
  a.dtiles = make_fastdiv(tiles);
  return launch(scan_step_kernel<T, NS, P, SEQ>, dim3((unsigned)((waves + 3) / 4)), 256, 0, st, a);
}
template <typename T, int NS, int P>
static int scan_step(const ScanArgs& a, hipStream_t st) {
  // several sequences a wave once there are enough waves without
  const int64_t waves = (int64_t)a.channels * P / 64 * a.s.count;
  return waves >= 16 * 4 * kPlanCus ? step_launch<T, NS, P, 2>(a, st) : step_launch<T, NS, P, 1>(a, st);
}
template <typename T>
static int scan_pick(const ScanArgs& a, const ScanPlan& p, hipStream_t st) {
  if (!a.s.offsets && a.s.len == 1) {
    if (a.states <= 16) return scan_step<T, 4, 4>(a, st);
    if (a.states <= 32) return scan_step<T, 4, 8>(a, st);
    if (a.states <= 64) return scan_step<T, 4, 16>(a, st);
    if (a.states <= 128) return scan_step<T, 8, 16>(a, st);
    return scan_step<T, 16, 16>(a, st);
  }
  if (p.narrow) switch (prompt_parts(a.states, true)) {
      case 4: return scan_prompt<T, 4, 4>(a, p, st);
      case 8: return scan_prompt<T, 4, 8>(a, p, st);
      default: return scan_prompt<T, 4, 16>(a, p, st);
    }
  switch (prompt_parts(a.states, false)) {
    case 1: return a.states <= 8 ? scan_prompt<T, 8, 1>(a, p, st) : scan_prompt<T, 16, 1>(a, p, st);
    case 2: return scan_prompt<T, 16, 2>(a, p, st);
    case 4: return scan_prompt<T, 16, 4>(a, p, st);
    case 8: return scan_prompt<T, 16, 8>(a, p, st);
    default: return scan_prompt<T, 16, 16>(a, p, st);
  }
}

int launch_scan(const ct_scan_op& op, const ScanPlan& p, const SeqView& s, const ScanArrays& v, void* stream) {
  ScanArgs a = {};
  a.s = s;
  a.u = v.u; a.delta = v.delta; a.b = v.b; a.c = v.c; a.z = v.z;
  a.dt_bias = v.dt_bias; a.a = v.a; a.d_skip = v.d_skip; a.state_in = v.state_in;
  a.state_out = v.state_out; a.y = v.y; a.ws = v.ws;
  a.ldu = op.ldu; a.lddelta = op.lddelta; a.ldb = op.ldb; a.ldc = op.ldc; a.ldz = op.ldz; a.ldy = op.ldy;
  a.channels = op.channels; a.states = op.states; a.per_group = op.channels / op.groups; a.softplus = op.softplus;
  a.stream = (int64_t)s.count * op.channels * op.states * (int64_t)sizeof(float) >= kStreamStateBytes;
  const int four = 4 * elem_bytes(op.dtype);
  a.vec_bc = ((uintptr_t)v.b | (uintptr_t)v.c) % four == 0 && (op.ldb | op.ldc | op.states) % 4 == 0;
  return op.dtype == CT_DT_BF16 ? scan_pick<bf16_t>(a, p, (hipStream_t)stream)
                                : scan_pick<float>(a, p, (hipStream_t)stream);
}

}  // namespace ct
