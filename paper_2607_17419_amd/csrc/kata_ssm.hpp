// kata_ssm.hpp -- the selective state space scan: per head a state S [N][P] with
// a scalar decay and a step that depend on the token,
//
//   step_t = softplus(dt_t + bias),  S_t = exp(step_t A) S_{t-1} + step_t B_t x_t^T,
//   y_t = C_t^T S_t + D x_t,
//
// B and C being shared by the H / G heads of a group.  In a chunk of L tokens,
// with l_t the sum of step A over its tokens up to t, S the state before it and
// R the gradient of the state after it,
//
//   W_ts  = (C_t . B_s) exp(l_t - l_s) step_s      (s <= t, else 0)
//   y_t   = sum_s W_ts x_s + exp(l_t) C_t^T S + D x_t
//   S'    = exp(l_L) S + sum_s exp(l_L - l_s) step_s B_s x_s^T
//   R'    = exp(l_L) R + sum_t exp(l_t) C_t dy_t^T
//   M_ts  = dy_t . x_s
//   dx_s  = sum_t W_ts dy_t + exp(l_L - l_s) step_s R^T B_s + D dy_s
//   dC_t  = sum_s M_ts exp(l_t - l_s) step_s B_s + exp(l_t) S dy_t
//   dB_s  = sum_t M_ts exp(l_t - l_s) step_s C_t + exp(l_L - l_s) step_s R x_s
//
// and, for the gradient e_t of log a_t = step_t A, the sum of W_rs M_rs over
// s < t <= r and of the state terms whose path crosses token t.  All products
// are 16 x 16 tiles on the matrix cores: bf16 tensors on the bf16 ones with fp32
// accumulation, fp32 tensors on the fp32 ones.
//
// Launches.  Forward: logs of all chunks; the states that spans of chunks add, joined over
// the spans; y, a workgroup per head and span carrying the state in registers.  Backward:
// logs, span states in both directions and their join; a record of S and R per chunk; the
// gradients, a workgroup per chunk and group.  The records cost 2 x 4 bytes per state
// element and chunk each way, but let every chunk stand alone: dB and dC of a group are
// summed over its heads in registers, with no atomics.
#pragma once

#include "kata_rows.hpp"

namespace kata {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- tiles --------------------------------------------------------------------
// Operands travel as "halves": four consecutive k of one row, lane (c, g) =
// (lane % 16, lane / 16) holding row c, k = 4 g .. 4 g + 3 of a K of 16.  A tile of
// products D[m][n] comes back with lane (c, g) holding column n = c, rows
// m = 4 g .. 4 g + 3: rounded, it is again a half, of row n with k = m, so that
// states and weights pass from one product into the next without moving.
template <typename E> struct SsmHalf;
template <> struct SsmHalf<bf16_t> { typedef uint2 type; };
template <> struct SsmHalf<float> { typedef float4 type; };
template <typename E> using ssm_half = typename SsmHalf<E>::type;

__device__ __forceinline__ f32x4 mac2(uint2 a0, uint2 a1, uint2 b0, uint2 b1, f32x4 acc) {
  const bf16x8 a = __builtin_bit_cast(bf16x8, make_uint4(a0.x, a0.y, a1.x, a1.y));
  const bf16x8 b = __builtin_bit_cast(bf16x8, make_uint4(b0.x, b0.y, b1.x, b1.y));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mac2(float4 a0, float4 a1, float4 b0, float4 b1, f32x4 acc) {
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.x, b0.x, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.y, b0.y, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.z, b0.z, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0.w, b0.w, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1.x, b1.x, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1.y, b1.y, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1.z, b1.z, acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a1.w, b1.w, acc, 0, 0, 0);
}

__device__ __forceinline__ f32x4 half_f32(uint2 h) {
  return f32x4{bf16lo_f32(h.x), bf16hi_f32(h.x), bf16lo_f32(h.y), bf16hi_f32(h.y)};
}
__device__ __forceinline__ f32x4 half_f32(float4 h) { return f32x4{h.x, h.y, h.z, h.w}; }

template <typename E>
__device__ __forceinline__ ssm_half<E> to_half(f32x4 v) {
  if constexpr (sizeof(E) == 2) return make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else return make_float4(v[0], v[1], v[2], v[3]);
}

// fp32 values as operands without loss of their leading 16 bits: bf16 as a sum of
// two (within 2^-17), fp32 as they are.
template <typename E>
struct SsmSplit {
  ssm_half<E> hi, lo;
  __device__ __forceinline__ explicit SsmSplit(f32x4 v) {
    hi = to_half<E>(v);
    if constexpr (sizeof(E) == 2) lo = to_half<E>(v - half_f32(hi));
  }
};

// Tiles in LDS.  fp32: rows padded by 16 bytes.  bf16: rows unpadded, the 16-byte piece q of
// row r standing at q ^ swizzle(r): with the bits of r that decide which rows share their
// banks, reversed, the 16 rows of a row half fall on distinct banks, and so do the eight
// rows (two pieces of each) of a transposing read.
template <typename E, int COLS>
struct SsmTile {
  static constexpr bool kSwizzled = sizeof(E) == 2;
  static constexpr int stride = COLS + (kSwizzled ? 0 : 4);
  static constexpr int size(int rows) { return rows * stride; }
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (COLS >= 128) return (r & 1) * 8 + (r >> 1 & 1) * 4 + (r >> 2 & 1) * 2 + (r >> 3 & 1);
    else if constexpr (COLS == 64) return (r >> 1 & 1) * 4 + (r >> 2 & 1) * 2 + (r >> 3 & 1);
    else return (r >> 2 & 1) * 2 + (r >> 3 & 1);
  }
  static __device__ __forceinline__ int at(int r, int col) {
    if constexpr (kSwizzled) return r * stride + ((col >> 3 ^ swizzle(r)) << 3) + (col & 7);
    else return r * stride + col;
  }
  // A lane's offsets within a tile (fresh: see SsmSelf).
  struct Lane {
    int r, c;
    __device__ __forceinline__ Lane() {
      const int j = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
      r = at(j, 4 * g);
      c = kSwizzled ? at(4 * g + (j >> 2), 4 * (j & 3)) : at(4 * g, j);
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(r), "+v"(c)); }
    // Half of row r0 + lane's c, k = k0 + 4 g ...;  r0, k0 multiples of 16.
    __device__ __forceinline__ ssm_half<E> row(const E* tile, int r0, int k0) const {
      const int o = kSwizzled ? r ^ k0 : r + k0;
      return *reinterpret_cast<const ssm_half<E>*>(tile + r0 * stride + o);
    }
    // Half of column c0 + lane's c, k running over rows k0 + 4 g ...  bf16: one transposing
    // read (lane j of 16 receives in slot s element j % 4 of the 8-byte piece that lane
    // 4 s + j / 4 addresses).
    __device__ __forceinline__ ssm_half<E> col(const E* tile, int c0, int k0) const {
      if constexpr (kSwizzled) {
        typedef short i16x4 __attribute__((ext_vector_type(4)));
        const E* p = tile + k0 * stride + (c ^ c0);
        const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) i16x4*)(const_cast<E*>(p)));
        return __builtin_bit_cast(uint2, v);
      } else {
        const E* p = tile + k0 * stride + c0 + c;
        return make_float4(p[0], p[stride], p[2 * stride], p[3 * stride]);
      }
    }
  };
};

// A thread's place: its wave (a scalar, so that what depends on it alone costs no vector
// register), lane = 16 g + c.  fresh(), called in every turn of a loop, hides from the compiler
// that they stay the same: it would otherwise form the addresses of all operands ahead of
// the loop, some 200 of them, and spill accumulators to keep them.
struct SsmSelf {
  int thread, wave, lane, c, g;
  __device__ __forceinline__ SsmSelf() : thread(threadIdx.x) { place(); }
  __device__ __forceinline__ void fresh() {
    asm volatile("" : "+v"(thread));
    place();
  }
  __device__ __forceinline__ void place() {
    wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    lane = thread & 63, c = lane & 15, g = lane >> 4;
  }
};

constexpr int kSsmP = 64;  // columns of the state that a workgroup holds
// Tokens of a chunk: the in-chunk products grow with it, the states' traffic in
// the backward shrinks; fp32 tiles take twice the LDS.
template <typename E> constexpr int ssm_chunk() { return sizeof(E) == 2 ? 64 : 32; }

// A token-major tensor's rows on their way into a tile: K pieces of 16 bytes per
// thread, loaded a chunk ahead of their use.  Rows at or past `valid` and columns at or
// past `cols` become zeros and are never read.  VEC (rows are whole aligned pieces, further
// apart than their width and within 2^31 bytes): by buffer loads, whose bounds give the
// zeros, one address register for all pieces and no branch; a branch between loads makes the
// compiler wait for those before it, which cost three memory latencies per chunk.
// Otherwise elements one by one.
template <typename E, int ROWS, int COLS, int THREADS, bool VEC>
struct SsmRows {
  static constexpr int V = 16 / static_cast<int>(sizeof(E)), PER = COLS / V;
  static constexpr int K = ROWS * PER / THREADS, kStep = THREADS / PER;  // rows between pieces
  static_assert(ROWS * PER % THREADS == 0, "every thread moves whole pieces");
  uint4 r[K];
  const SsmSelf& me;  // addresses are formed anew from its thread number
  __device__ __forceinline__ int row() const { return me.thread / PER; }
  __device__ __forceinline__ int column() const { return me.thread % PER * V; }
  __device__ __forceinline__ explicit SsmRows(const SsmSelf& self) : me(self) {}
  __device__ __forceinline__ void load(const E* src, long long stride, int valid, int cols) {
    if constexpr (VEC) {
      const int bytes = ((valid - 1) * static_cast<int>(stride) + min(cols, COLS)) *
                        static_cast<int>(sizeof(E));
      const auto buffer =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(src), 0, bytes, 0x00020000);
      const unsigned step = kStep * static_cast<unsigned>(stride) * static_cast<unsigned>(sizeof(E));
      const unsigned at = column() < cols ? (row() * static_cast<unsigned>(stride) + column()) *
                                                static_cast<unsigned>(sizeof(E))
                                          : 0x80000000u;  // out of bounds with any step
#pragma unroll
      for (int j = 0; j < K; ++j)
        r[j] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(
                                             buffer, static_cast<int>(at + j * step), 0, 0));
    } else {
#pragma unroll
      for (int j = 0; j < K; ++j) {
        union { uint4 u; E e[V]; } v;
        v.u = make_uint4(0, 0, 0, 0);
        const int at = row() + j * kStep;
        const E* p = src + at * stride + column();
        for (int k = 0; k < V; ++k)
          if (at < valid && column() + k < cols) v.e[k] = p[k];
        r[j] = v.u;
      }
    }
  }
  // Whether one of the pieces has a value that is not finite: an exponent of all ones.
  __device__ __forceinline__ bool non_finite() const {
    if constexpr (sizeof(E) == 2) {
      typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
      u16x2 most = {};
#pragma unroll
      for (int j = 0; j < K; ++j)
        for (uint32_t w : {r[j].x, r[j].y, r[j].z, r[j].w})
          most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu));
      return max(most.x, most.y) >= 0x7F80;
    } else {
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < K; ++j)
        for (uint32_t w : {r[j].x, r[j].y, r[j].z, r[j].w}) most = max(most, w & 0x7FFFFFFFu);
      return most >= 0x7F800000u;
    }
  }
  __device__ __forceinline__ void store(E* dst) const {
#pragma unroll
    for (int j = 0; j < K; ++j)
      *reinterpret_cast<uint4*>(dst + SsmTile<E, COLS>::at(row(), column()) +
                                j * kStep * SsmTile<E, COLS>::stride) = r[j];
  }
};

// ---- steps and decays of a chunk -------------------------------------------------
// Ends a stretch that the scheduler may reorder: operand reads of later stretches are not
// moved up, where they would hold registers that the accumulators need.
__device__ __forceinline__ void ssm_stretch() { __builtin_amdgcn_sched_barrier(0); }

// Inclusive sums in fp64 over the lanes of a row of 16 by DPP shifts, and over a wave's: then
// the last lane of a row to the next row, of the first two rows to the last two.
struct Halves64 {
  int lo, hi;
};
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x) {
  const auto move = [](int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); };
  const Halves64 h = __builtin_bit_cast(Halves64, x);
  return x + __builtin_bit_cast(double, Halves64{move(h.lo), move(h.hi)});
}
__device__ __forceinline__ double scan_row(double x) {
  x = dpp_add<0x111, 0xF>(x);
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  return dpp_add<0x118, 0xF>(x);
}
__device__ __forceinline__ double scan_wave(double x) {
  x = dpp_add<0x142, 0xA>(scan_row(x));
  return dpp_add<0x143, 0xC>(x);
}
__device__ __forceinline__ double read_lane(double x, int lane) {
  const Halves64 h = __builtin_bit_cast(Halves64, x);
  return __builtin_bit_cast(double, Halves64{__builtin_amdgcn_readlane(h.lo, lane),
                                             __builtin_amdgcn_readlane(h.hi, lane)});
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A token's step and its derivative by dt.
struct SsmStep {
  double step, gate;
};
// z = dt + bias, softplus(z) and its derivative, in fp64 to 1e-10 of themselves: z in fp32 would be
// off by 2^-24 |z|, and a step or gate of e^z, z = -5, by five times its own rounding (dt_dbias
// of random bf16 calls 1.8e-7 off for 1.2e-7).  With u = e^-|z| from Taylor's series of e^f,
// |f| <= log(2) / 2, to f^9:
//   softplus(z) = max(z, 0) + log(1 + u),  log(1 + u) = 2 artanh(s), s = u / (2 + u) <= 1 / 3,
//   by its series to s^19;  the derivative is 1 / (1 + u), for z < 0 u / (1 + u).
// u = 0 where e^z is nothing in fp32: -inf and the lowest numbers, as masks use them, give 0.
__device__ __forceinline__ SsmStep ssm_step_of(double z, bool softplus) {
  if (!softplus) return {z, 1.0};
  const double a = -fabs(z), n = rint(a * 1.4426950408889634074), f = a - n * 0.69314718055994530942;
  double u = 1.0 / 362880.0;
  constexpr double kSeries[] = {1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5, 1.0, 1.0};
#pragma unroll
  for (double k : kSeries) u = fma(u, f, k);
  // (n bounded: it may be infinite or NaN, which is no int; a NaN stays in u)
  u = a < -104.0 ? 0.0 : __builtin_amdgcn_ldexp(u, static_cast<int>(fmax(n, -2000.0)));
  const double p = 1.0 + u, q = 2.0 + u, d = p * q;
  double r = __builtin_amdgcn_rcp(d);  // 1 / d, by Newton's iteration
  r = fma(fma(-d, r, 1.0), r, r);
  const double s = u * p * r, s2 = s * s;
  double l = 2.0 / 19;
#pragma unroll
  for (int k = 17; k > 0; k -= 2) l = fma(l, s2, 2.0 / k);
  return {fmax(z, 0.0) + l * s, (z < 0.0 ? u : 1.0) * q * r};
}
__device__ __forceinline__ SsmStep ssm_step_of(float dt, const float* bias, int h, bool softplus) {
  return ssm_step_of(static_cast<double>(dt) + (bias ? static_cast<double>(bias[h]) : 0.0), softplus);
}

// A first kernel forms them once for all others: per token {hi, lo, step, gate} with the
// running sum l = hi + lo of step A over the chunk in units of log 2 (summed in fp64:
// differences of l keep 2^-48 of the largest, and exp(l_t - l_s) is right where a strong
// decay stands before weak ones), and gate the derivative of step by dt.  16 heads of 131072
// tokens: 17 us, a wave waiting for its one load and then for the chain of its step and its scan.
template <typename E, int L>
__global__ __launch_bounds__(256) void ssm_logs_kernel(SsmArgs a, int NC) {
  const int per = (a.H + 3) / 4;
  const int h = (blockIdx.x % per) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int chunk = (blockIdx.x / per) % NC, b = blockIdx.x / per / NC;
  if (h >= a.H) return;
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int t = chunk * L + lane;
  const bool live = lane < L && t < len;
  SsmStep v = {0.0, 0.0};
  if (live)
    v = ssm_step_of(to_f32(static_cast<const E*>(a.dt)[b * a.db + h * a.dh + t * a.dt_t]), a.bias, h,
                    a.softplus);
  double l = v.step * (static_cast<double>(a.A[h]) * 1.4426950408889634074);
  // 2^-2000 and 2^2000 are 0 and inf in fp32: bounded, sums and their differences stay finite
  l = l < -2000.0 ? -2000.0 : (l > 2000.0 ? 2000.0 : l);  // (NaN stays)
  if (!live) l = 0.0;
  l = scan_wave(l);
  if (lane >= L) return;
  const float hi = static_cast<float>(l);
  a.logs[(static_cast<size_t>(b * a.H + h) * NC + chunk) * L + lane] =
      make_float4(hi, isfinite(hi) ? static_cast<float>(l - hi) : 0.f, static_cast<float>(v.step),
                  static_cast<float>(v.gate));
}

// A chunk's logs in LDS, with exp(l_t) (since) and exp(l_L - l_t) (left); all = exp(l_L).
struct __attribute__((aligned(16))) SsmChunkLog {
  // push: left times step
  float hi[64], lo[64], step[64], gate[64], since[64], left[64], push[64];
  float all, log;  // log: l_L, rounded

  // By one whole wave; lanes past the chunk hold a copy of its last token.
  template <int L>
  __device__ __forceinline__ void store(float4 v) {
    const int lane = threadIdx.x & 63;
    const float eh = __shfl(v.x, L - 1), el = __shfl(v.y, L - 1);
    if (lane == 0) all = exp2_fast(eh + el), log = eh + el;
    if (lane >= L) return;
    hi[lane] = v.x, lo[lane] = v.y, step[lane] = v.z, gate[lane] = v.w;
    since[lane] = exp2_fast(v.x + v.y);
    const float rest = exp2_fast((eh - v.x) + (el - v.y));
    left[lane] = rest;
    push[lane] = rest * v.z;
  }
  __device__ __forceinline__ f32x4 four(const float* p, int i) const {
    return *reinterpret_cast<const f32x4*>(p + i);
  }
  // exp(l_t - l_s) of token t and four tokens s0 ..
  __device__ __forceinline__ f32x4 decay(int t, int s0) const {
    const f32x4 d = (hi[t] - four(hi, s0)) + (lo[t] - four(lo, s0));
    return f32x4{exp2_fast(d[0]), exp2_fast(d[1]), exp2_fast(d[2]), exp2_fast(d[3])};
  }
};

template <int L>
__device__ __forceinline__ const float4* ssm_log_row(const SsmArgs& a, int bh, int NC) {
  return a.logs + static_cast<size_t>(bh) * NC * L + min(static_cast<int>(threadIdx.x & 63), L - 1);
}

// A chunk's lower-triangular 16 x 16 tiles (row tile tt >= column tile ss), numbered.
__device__ __forceinline__ void ssm_tri(int id, int& tt, int& ss) {
  tt = id >= 6 ? 3 : (id >= 3 ? 2 : (id >= 1 ? 1 : 0));
  ss = id - tt * (tt + 1) / 2;
}

// Workgroups go to the 8 XCDs in turn: numbered so that neighbours share an XCD's L2.
__device__ __forceinline__ unsigned ssm_xcd_order() {
  const unsigned n = gridDim.x, x = blockIdx.x & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (blockIdx.x >> 3);
}

// ---- forward -------------------------------------------------------------------
// A workgroup carries the state of one head (64 of its columns) over the chunks of a
// span, as accumulators: wave w holds columns 16 w ...  Per chunk a wave forms the
// weights of 16 tokens, which as accumulators are already the operand that they are
// needed as, and with them and all columns' states (shared through LDS as operands, a
// chunk behind the accumulators) these tokens' y; then the new state of its columns.
// The next chunk's rows are on their way meanwhile.  y is turned in LDS into whole lines.
// The chunk's weights and the state that y reads are rounded to bf16 once (2^-8 of a term
// each at most, as y itself is rounded), the state that is carried is not, and D x is added in fp32:
// on W's diagonal D would be rounded with it, the same factor for all tokens of a head (y 2.3e-3
// off for 1.8e-3 (rms); 131072 tokens 272 us for 279).
// 16 heads of 131072 tokens, N = P = 64, bf16: 222 us, 626 MB counted, 2.8 TB/s; bound by issue,
// vector instructions taking 62% of a SIMD's cycles and matrix ones 19%.  Rows that are not
// whole aligned pieces are read element by element: 3 times the time of the whole call.
constexpr int ssm_most(int a, int b) { return a > b ? a : b; }

template <typename E, int NP>
struct __attribute__((aligned(16))) SsmOutLds {
  static constexpr int L = ssm_chunk<E>();
  // a wave's part of st: 16 columns' states, or 16 rows of y
  static constexpr int kPart = SsmTile<E, ssm_most(NP, kSsmP)>::size(16);
  E c[SsmTile<E, NP>::size(L)], b[SsmTile<E, NP>::size(L)], x[SsmTile<E, kSsmP>::size(L)];
  E st[4 * kPart];
  SsmChunkLog log;
  int bad;  // the last chunk whose x has non-finite values
};

// The state's columns of this wave as accumulator tiles, from or to [N][P] fp32.
template <int NP>
__device__ __forceinline__ void ssm_load_state(const float* S, int N, int P, int p,
                                               f32x4 (&h)[NP / 16]) {
  const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
  for (int j = 0; j < NP / 16; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = 16 * j + 4 * g + i;
      h[j][i] = (S && n < N && p < P) ? S[static_cast<size_t>(n) * P + p] : 0.f;
    }
}
template <int NP>
__device__ __forceinline__ void ssm_store_state(float* S, int N, int P, int p,
                                                const f32x4 (&h)[NP / 16]) {
  const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
  for (int j = 0; j < NP / 16; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = 16 * j + 4 * g + i;
      if (n < N && p < P) S[static_cast<size_t>(n) * P + p] = h[j][i];
    }
}

// h <- exp(l_L) h + sum_s B_s (scale_s v_s)^T over the chunk's tokens; keys and v are
// LDS tiles, f the scales of four tokens.  bf16: the scaled values enter as hi + lo, so that
// the fp32 state keeps 2^-17 of every term: enough for what is rounded to bf16 afterwards (y);
// EXACT, for a state that is returned and for the gradients, with a third part, which keeps
// all of fp32's bits (the error of a state of 2000 tokens falls from 2e-6 to 1e-7; a
// forward that returns none would take 1.1 times as long with it).  OWN: the chunk's own
// sum first, so that the state is rounded once per chunk and not by each of the products
// added to it, whose errors the states of long memories gather (dA of 16 heads of 1024 tokens
// 4.4e-7 off for 2.1e-7), and with EXACT the smaller parts' sum apart (see ssm_add_rest); for the
// gradients and fp32.  (ssm_out_kernel's registers do not hold it:
// a prompt's call 40 us for 38.)
template <typename E, int NP, int L, bool EXACT, bool OWN, typename F>
__device__ __forceinline__ void ssm_state_update(const typename SsmTile<E, NP>::Lane& kt,
                                                 const typename SsmTile<E, kSsmP>::Lane& vt,
                                                 const E* keys, const E* v, int p0, float decay,
                                                 F f, f32x4 (&h)[NP / 16]) {
  const int g = (threadIdx.x >> 4) & 3;
  f32x4 own[OWN ? NP / 16 : 1] = {}, rest[OWN && EXACT ? NP / 16 : 1] = {};
  if constexpr (!OWN) {
#pragma unroll
    for (int j = 0; j < NP / 16; ++j) h[j] *= decay;
  }
#pragma unroll
  for (int s0 = 0; s0 < L; s0 += 32) {
    const f32x4 v0 = half_f32(vt.col(v, p0, s0)) * f(s0 + 4 * g);
    const f32x4 v1 = half_f32(vt.col(v, p0, s0 + 16)) * f(s0 + 16 + 4 * g);
    const SsmSplit<E> a(v0), b(v1);
    ssm_half<E> a2, b2;
    if constexpr (EXACT) {
      a2 = to_half<E>((v0 - half_f32(a.hi)) - half_f32(a.lo));
      b2 = to_half<E>((v1 - half_f32(b.hi)) - half_f32(b.lo));
    }
#pragma unroll
    for (int j = 0; j < NP / 16; ++j) {
      f32x4& sum = OWN ? own[OWN ? j : 0] : h[j];
      const auto k0 = kt.col(keys, 16 * j, s0);
      const auto k1 = kt.col(keys, 16 * j, s0 + 16);
      sum = mac2(k0, k1, a.hi, b.hi, sum);
      f32x4& low = OWN && EXACT ? rest[OWN && EXACT ? j : 0] : sum;
      if constexpr (sizeof(E) == 2) low = mac2(k0, k1, a.lo, b.lo, low);
      if constexpr (EXACT) low = mac2(k0, k1, a2, b2, low);
    }
    ssm_stretch();
  }
  if constexpr (OWN) {
#pragma unroll
    for (int j = 0; j < NP / 16; ++j) {
      if constexpr (EXACT) own[j] += rest[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[j][i] = fmaf(decay, h[j][i], own[j][i]);
    }
  }
}

// Workgroup -> batch, span, block of columns, head; heads of one batch and span run
// next to each other, so that their group's B and C rows come from HBM once.
struct SsmPlace {
  int b, span, pb, h;
  __device__ __forceinline__ SsmPlace(const SsmArgs& a, int spans, unsigned id) {
    const int blocks = (a.P + kSsmP - 1) / kSsmP;
    h = id % a.H, id /= a.H;
    pb = id % blocks, id /= blocks;
    span = id % spans;
    b = id / spans;
  }
};

// A 16-byte piece of a row, the first element at column p of P.
template <bool VEC, typename E>
__device__ __forceinline__ void ssm_store_piece(E* dst, uint4 v, int p, int P) {
  if constexpr (VEC) {
    if (p < P) *reinterpret_cast<uint4*>(dst) = v;
  } else {
    constexpr int V = 16 / static_cast<int>(sizeof(E));
    const RawVec<E, V> e = *reinterpret_cast<const RawVec<E, V>*>(&v);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (p + i < P) dst[i] = e.e[i];
  }
}

// Non-finite values replaced by zeros.
template <typename E>
__device__ __forceinline__ ssm_half<E> ssm_finite(ssm_half<E> h) {
  f32x4 v = half_f32(h);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = fabsf(v[i]) < INFINITY ? v[i] : 0.f;
  return to_half<E>(v);
}

// Four neighbouring results of a row, the first at column p of P.
template <bool VEC, typename E>
__device__ __forceinline__ void ssm_store4(E* dst, f32x4 v, int p, int P) {
  if constexpr (VEC) {
    if (p < P) *reinterpret_cast<ssm_half<E>*>(dst) = to_half<E>(v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < P) store_f32(dst + i, v[i]);
  }
}

template <typename E, int NP, bool VEC, bool EXACT>
__global__ __launch_bounds__(256, NP > 64 ? 2 : (sizeof(E) == 2 ? 4 : 3)) void ssm_out_kernel(SsmArgs a) {
  constexpr int L = ssm_chunk<E>(), LT = L / 16, NT = NP / 16;
  constexpr int PW = LT == 4 ? 4 : 2;  // tiles of columns of which a wave forms y
  typedef SsmTile<E, NP> KT;
  typedef SsmTile<E, kSsmP> VT;
  typedef SsmTile<E, 16 * PW> YT;
  typedef SsmOutLds<E, NP> Lds;
  static_assert(YT::size(16) <= Lds::kPart && KT::size(16) <= Lds::kPart, "a wave's part");
  __shared__ Lds m;
  typename KT::Lane kt;
  typename VT::Lane vt;
  const SsmPlace at(a, a.spans, ssm_xcd_order());
  const int b = at.b, h = at.h, bh = b * a.H + h, grp = h / (a.H / a.G);
  SsmSelf me;
  const int &wave = me.wave, &c = me.c, &g = me.g;
  const int pc = at.pb * kSsmP;
  const int NC = (a.T + L - 1) / L;
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int span_len = a.span_chunks * L;
  const int first = at.span * span_len, last = min(first + span_len, len);
  const float D = a.D ? a.D[h] : 0.f;
  const size_t NPs = static_cast<size_t>(a.N) * a.P;
  f32x4 st[NT];
  const float* from = at.span ? a.rec + (static_cast<size_t>(bh) * (a.spans - 1) + at.span - 1) * NPs
                              : (a.S_in ? a.S_in + bh * NPs : nullptr);
  ssm_load_state<NP>(from, a.N, a.P, pc + 16 * wave + c, st);
  // the rows of the next chunk to fetch, and of y
  const E* x = static_cast<const E*>(a.x) + b * a.xb + h * a.xh + pc + first * a.xt;
  const E* Bm = static_cast<const E*>(a.Bm) + b * a.bb + grp * a.bg + first * a.bt;
  const E* Cm = static_cast<const E*>(a.Cm) + b * a.cb + grp * a.cg + first * a.ct;
  const float4* logs = ssm_log_row<L>(a, bh, NC) + first;
  E* y = static_cast<E*>(a.y) + b * a.yb + h * a.yh + pc + first * a.yt;
  SsmRows<E, L, NP, 256, VEC> rc(me), rb(me);
  SsmRows<E, L, kSsmP, 256, VEC> rx(me);
  float4 rl;
  const auto fetch = [&](int t0) {
    const int rows = min(L, last - t0);
    rc.load(Cm, a.ct, rows, a.N);
    rb.load(Bm, a.bt, rows, a.N);
    rx.load(x, a.xt, rows, a.P - pc);
    if (wave == 0) rl = *logs;
    Cm += L * a.ct, Bm += L * a.bt, x += L * a.xt, logs += L;
  };
  // a chunk's rows, and the state before it, into LDS
  const auto stage = [&](int t0) {
    rc.store(m.c);
    rb.store(m.b);
    rx.store(m.x);
    if (wave == 0) m.log.template store<L>(rl);
    if (rx.non_finite()) m.bad = t0;
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<ssm_half<E>*>(m.st + wave * Lds::kPart + KT::at(c, 16 * j + 4 * g)) =
          to_half<E>(st[j]);
  };
  if (threadIdx.x == 0) m.bad = -1;
  lds_barrier();
  if (first < last) fetch(first), stage(first);
  for (int t0 = first; t0 < last; t0 += L) {
    const int rows = min(L, last - t0);
    lds_barrier();
    if (t0 + L < last) fetch(t0 + L);
    kt.fresh(), vt.fresh(), me.fresh();
    // the tile of tokens, turned with the workgroup: later tiles have more weights to form
    const int tt = (wave + blockIdx.x) % LT, q0 = LT == 4 ? 0 : PW * (wave / LT);
    const int t = 16 * tt + c;
    ssm_half<E> cr[NT], w[LT];
    bool above[4];  // the diagonal
#pragma unroll
    for (int i = 0; i < 4; ++i) above[i] = 4 * g + i > c;
#pragma unroll
    for (int k = 0; k < NT; ++k) cr[k] = kt.row(m.c, 16 * tt, 16 * k);
#pragma unroll
    for (int ss = 0; ss < LT; ++ss) {
      w[ss] = ssm_half<E>{};
      if (ss > tt) continue;
      // C B^T, rows s, columns t: as a half, row t of W
      f32x4 acc = {};
#pragma unroll
      for (int k = 0; k < NT; k += 2)
        acc = mac2(kt.row(m.b, 16 * ss, 16 * k), kt.row(m.b, 16 * ss, 16 * k + 16), cr[k], cr[k + 1], acc);
      const int s = 16 * ss + 4 * g;
      acc *= m.log.decay(t, s) * m.log.four(m.log.step, s);
      if (tt == ss) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = above[i] ? 0.f : acc[i];
      }
      w[ss] = to_half<E>(acc);
    }
    ssm_stretch();
    // y, rows p, columns t
    const float since = m.log.since[t];
    ssm_half<E> out[PW];
    const auto columns = [&](auto finite) {
#pragma unroll
      for (int j = 0; j < PW; ++j) {
        const int p0 = 16 * (q0 + j);
        const E* sp = m.st + (q0 + j) * Lds::kPart;
        f32x4 acc = {};
#pragma unroll
        for (int k = 0; k < NT; k += 2)
          acc = mac2(kt.row(sp, 0, 16 * k), kt.row(sp, 0, 16 * k + 16), cr[k], cr[k + 1], acc);
        acc *= since;
#pragma unroll
        for (int ss = 0; ss < LT; ss += 2) {
          if (ss > tt) continue;
          auto x0 = vt.col(m.x, p0, 16 * ss), x1 = vt.col(m.x, p0, 16 * ss + 16);
          if (!finite) x0 = ssm_finite<E>(x0), x1 = ssm_finite<E>(x1);
          acc = mac2(x0, x1, w[ss], w[ss + 1], acc);
        }
        const f32x4 own = half_f32(vt.row(m.x, 16 * tt, p0));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(D, own[i], acc[i]);
        if (!finite) {
          bool seen[4] = {};
#pragma nounroll
          for (int s = 0; s <= t; ++s) {
            const f32x4 v = half_f32(*reinterpret_cast<const ssm_half<E>*>(m.x + VT::at(s, p0 + 4 * g)));
#pragma unroll
            for (int i = 0; i < 4; ++i) seen[i] |= !(fabsf(v[i]) < INFINITY);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = seen[i] ? NAN : acc[i];
        }
        out[j] = to_half<E>(acc);
      }
    };
    // A non-finite x_s times the zero weight of an earlier token would be NaN: left out of
    // the products, it makes the tokens from s on NaN.
    if (__builtin_amdgcn_readfirstlane(m.bad) != t0) columns(std::true_type{});
    else columns(std::false_type{});
    ssm_stretch();
    ssm_state_update<E, NP, L, EXACT, sizeof(E) == 4>(
        kt, vt, m.b, m.x, 16 * wave, m.log.all, [&](int s) { return m.log.four(m.log.push, s); }, st);
    lds_barrier();
    // a wave's 16 rows of y, turned in its own part of st
    E* mine = m.st + wave * Lds::kPart;
#pragma unroll
    for (int j = 0; j < PW; ++j)
      *reinterpret_cast<ssm_half<E>*>(mine + YT::at(c, 16 * j + 4 * g)) = out[j];
    __builtin_amdgcn_wave_barrier();
    constexpr int V = 16 / static_cast<int>(sizeof(E)), PER = 16 * PW / V;
#pragma unroll
    for (int j = 0; j < 16 * PER / 64; ++j) {
      const int i = me.lane + 64 * j, r = 16 * tt + i / PER, col = i % PER * V;
      const uint4 v = *reinterpret_cast<const uint4*>(mine + YT::at(i / PER, col));
      if (r < rows) ssm_store_piece<VEC>(y + r * a.yt + 16 * q0 + col, v, pc + 16 * q0 + col, a.P);
    }
    __builtin_amdgcn_wave_barrier();
    y += L * a.yt;
    if (t0 + L < last) stage(t0 + L);
  }
  if (a.S_out && at.span == a.spans - 1)
    ssm_store_state<NP>(a.S_out + bh * NPs, a.N, a.P, pc + 16 * wave + c, st);
}

// ---- states of spans and chunks --------------------------------------------------
// Forward: S over keys B and values x; reverse: R over keys C and values dy, from a
// span's last chunk to its first; a launch does the first `dirs` of the two, half of its
// workgroups each.  CHUNKS = false: a span's own contribution and its decay, to rec;
// true: from the span's state in rec, every chunk's state before its tokens are added (S
// at the chunk's start, R at its end), to `chunks` (R's behind S's): records of [64
// columns][NP] fp32, one per head, block and chunk.
// Span states of 16 heads of 131072 tokens: 82 us, 333 MB counted, 4.1 TB/s, vector and
// matrix instructions issuing in 74% of the cycles.  Chunk records of 8 x 4096 tokens of 16 heads:
// 81 us, 438 MB counted (268 MB of them written), 5.4 TB/s, HBM bound.
// An accumulator tile's float4 of a lane is a piece: piece 64 (4 j + w) + lane holds rows
// 16 j + 4 g .. of column 16 w + c, so that stores are whole lines as they stand.
template <typename E, int NP>
struct __attribute__((aligned(16))) SsmStateLds {
  static constexpr int L = ssm_chunk<E>();
  E k[SsmTile<E, NP>::size(L)], v[SsmTile<E, kSsmP>::size(L)];
  SsmChunkLog log;
};

template <typename E, int NP, bool CHUNKS, bool VEC, bool EXACT>
__global__ __launch_bounds__(256) void ssm_state_kernel(SsmArgs a, f32x4* chunks, int dirs) {
  constexpr int L = ssm_chunk<E>();
  __shared__ SsmStateLds<E, NP> m;
  typename SsmTile<E, NP>::Lane kl;
  typename SsmTile<E, kSsmP>::Lane vl;
  // without CHUNKS the forward's last and the reverse's first span go nowhere
  unsigned id = ssm_xcd_order();
  const bool rev = id >= gridDim.x / dirs;
  if (rev) id -= gridDim.x / dirs;
  SsmPlace at(a, CHUNKS ? a.spans : a.spans - 1, id);
  const int slot = at.span;  // rec's, without CHUNKS
  if (!CHUNKS && rev) ++at.span;
  const int b = at.b, h = at.h, bh = b * a.H + h, grp = h / (a.H / a.G);
  SsmSelf me;
  const int &wave = me.wave, &c = me.c;
  const int pc = at.pb * kSsmP, p0 = 16 * wave, p = pc + p0 + c;
  const int NC = (a.T + L - 1) / L, blocks = (a.P + kSsmP - 1) / kSsmP;
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int span_len = a.span_chunks * L;
  const int first = at.span * span_len, last = min(first + span_len, len);
  const size_t NPs = static_cast<size_t>(a.N) * a.P;
  const int gaps = a.spans - 1;
  f32x4 st[NP / 16];
  const float* from = nullptr;
  const size_t recs = (rev ? static_cast<size_t>(a.B) * a.H * gaps : 0) + static_cast<size_t>(bh) * gaps;
  if (CHUNKS && (rev ? at.span < gaps : at.span > 0)) from = a.rec + (recs + at.span - !rev) * NPs;
  ssm_load_state<NP>(from, a.N, a.P, p, st);
  const E* v = rev ? static_cast<const E*>(a.dy) + b * a.yb + h * a.yh + pc
                   : static_cast<const E*>(a.x) + b * a.xb + h * a.xh + pc;
  const E* k = rev ? static_cast<const E*>(a.Cm) + b * a.cb + grp * a.cg
                   : static_cast<const E*>(a.Bm) + b * a.bb + grp * a.bg;
  const long long vt = rev ? a.yt : a.xt, kt = rev ? a.ct : a.bt;
  const float4* logs = ssm_log_row<L>(a, bh, NC);
  const int n = last > first ? (last - first + L - 1) / L : 0;
  const int steps = CHUNKS ? n - 1 : n;  // the state past the span's end is the next span's
  SsmRows<E, L, NP, 256, VEC> rk(me);
  SsmRows<E, L, kSsmP, 256, VEC> rv(me);
  float4 rl;
  const auto start = [&](int i) { return first + (rev ? n - 1 - i : i) * L; };
  const auto fetch = [&](int t0) {
    const int rows = min(L, last - t0);
    rk.load(k + t0 * kt, kt, rows, a.N);
    rv.load(v + t0 * vt, vt, rows, a.P - pc);
    if (wave == 0) rl = logs[t0];
  };
  if (steps > 0) fetch(start(0));
  double log_sum = 0.0;
  for (int i = 0; i < n; ++i) {
    const int t0 = start(i);
    if constexpr (CHUNKS) {
      f32x4* rec = chunks + ((static_cast<size_t>(bh + (rev ? a.B * a.H : 0)) * blocks + at.pb) * NC + t0 / L) *
                                (kSsmP * NP / 4);
#pragma unroll
      for (int j = 0; j < NP / 16; ++j) rec[(4 * j + wave) * 64 + me.lane] = st[j];
      if (i >= steps) break;
    }
    lds_barrier();
    rk.store(m.k);
    rv.store(m.v);
    if (wave == 0) m.log.template store<L>(rl);
    lds_barrier();
    if (i + 1 < steps) fetch(start(i + 1));
    kl.fresh(), vl.fresh(), me.fresh();
    if (!CHUNKS) log_sum += m.log.log;
    ssm_state_update<E, NP, L, EXACT, EXACT || sizeof(E) == 4>(
        kl, vl, m.k, m.v, p0, m.log.all,
        [&](int s) { return m.log.four(rev ? m.log.since : m.log.push, s); }, st);
  }
  if constexpr (!CHUNKS) {
    ssm_store_state<NP>(a.rec + (recs + slot) * NPs, a.N, a.P, p, st);
    if (threadIdx.x == 0 && at.pb == 0) a.rec_log[recs + slot] = log_sum;
  }
}

// rec: a span's own contribution becomes the state that enters the next span (reverse:
// the one before), in the same slot.  Grid: V elements a thread, heads, directions.  A chain
// of loads eight records deep: 12 us for 63 records of 16 heads, 10 us for 7 of 128 (four
// elements a thread; with one 2% more of a call of 131072 tokens).
template <int V>
__global__ __launch_bounds__(256) void ssm_span_scan(SsmArgs a) {
  const int NPs = a.N * a.P, gaps = a.spans - 1;
  const int e = (blockIdx.x * 256 + threadIdx.x) * V, bh = blockIdx.y;
  const bool rev = blockIdx.z;
  if (e >= NPs) return;
  float s[V] = {};
  if (!rev && a.S_in) load_vec<V>(a.S_in + static_cast<size_t>(bh) * NPs + e, s);
  const size_t recs = (static_cast<size_t>(rev) * a.B * a.H + bh) * gaps;
  float* rec = a.rec + recs * NPs + e;
  const double* log = a.rec_log + recs;
  constexpr int U = 8;  // records in flight
  for (int i = 0; i < gaps; i += U) {
    float v[U][V], d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(i + u, gaps - 1), j = rev ? gaps - 1 - k : k;
      load_vec<V>(rec + static_cast<size_t>(j) * NPs, v[u]);
      d[u] = exp2_fast(static_cast<float>(log[j]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= gaps) break;
      const int j = rev ? gaps - 1 - (i + u) : i + u;
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] = fmaf(d[u], s[k], v[u][k]);
      store_vec<V>(rec + static_cast<size_t>(j) * NPs, s);
    }
  }
}

// ---- gradients ------------------------------------------------------------------
// A workgroup takes one chunk of one group and a block of its heads in turn: dB and dC
// of the group stay in accumulators over the heads, C B^T is formed once, and the next
// head's rows and records are on their way while one is worked on.  Results stand with
// features (n, p) along an accumulator's rows and tokens along its columns, so that a
// lane holds four neighbouring features of one token; a wave forms 2 x 2 tiles where
// there are as many, each operand read serving two products.  Four waves, so that two
// workgroups share a CU and one works through the other's barriers; eight at N > 64,
// whose records leave LDS for one workgroup.
// 8 x 4096 tokens of 16 heads, N = P = 64, bf16: 190 us, 512 MB counted (268 MB of
// records), 2.7 TB/s; vector instructions take 45% of the cycles, LDS 37%, matrix
// instructions 11%, the rest are waits at the six barriers of a head, which two workgroups
// of a CU half cover.
// part: dA, dD, dbias of the chunk, [B * NC][3][H], in fp64: a head's chunks may cancel.
struct SsmGrads {
  void *dx, *ddt, *dBm, *dCm;
  float *pB, *pC;  // with several head blocks: their sums, [blocks][B][T][G][N] fp32
  double* part;
  const f32x4 *fwd, *rev;  // chunk records
  int head_block, blocks;
};

// In LDS a record stands as operand planes, bf16 ones as hi + mid + lo, all of fp32's bits: the
// gradients of A and of the steps are sums of products of S and R in which much cancels.
// With hi + lo in state, record and product (2^-17 each) 4.4% of the heads of random calls had a dA
// and 6% a dbias off by more than 1e-5 of themselves for 0.6% (a plain fp32 form: 0.5 and 1.3%); a
// training step of 8 x 4096 tokens took 368 us for 379.
template <typename E> constexpr int ssm_planes() { return sizeof(E) == 2 ? 3 : 1; }
constexpr int ssm_grad_threads(int NP) { return NP > 64 ? 512 : 256; }

template <typename E, int NP>
struct __attribute__((aligned(16))) SsmGradLds {
  static constexpr int L = ssm_chunk<E>(), kWaves = ssm_grad_threads(NP) / 64;
  E c[SsmTile<E, NP>::size(L)], b[SsmTile<E, NP>::size(L)];
  E x[SsmTile<E, kSsmP>::size(L)], dy[SsmTile<E, kSsmP>::size(L)];
  E st[ssm_planes<E>() * SsmTile<E, NP>::size(kSsmP)];
  E w[SsmTile<E, L>::size(L)], mw[SsmTile<E, L>::size(L)];
  SsmChunkLog log[2];                       // of this head and the next
  // pair sums by tile of the other index; a diagonal tile's row: its pairs across each token
  float row[4][64], col[4][64];
  float diag[64], trace[64];                // of (C B^T) M exp(l_t - l_s), of M
  float q[kWaves / 2][64], k[kWaves / 2][64];  // state terms by the waves' tiles of n, of p
  float dot[kWaves];
};

// The pieces of a chunk record that a thread moves.
template <typename E, int NP, int THREADS>
struct SsmRecord {
  static constexpr int K = kSsmP * NP / 4 / THREADS, PL = ssm_planes<E>();
  static constexpr int kStep = THREADS / 16;  // rows between pieces
  static_assert(kSsmP * NP % (4 * THREADS) == 0 && THREADS % 256 == 0, "every thread moves whole pieces");
  typedef SsmTile<E, NP> KT;
  f32x4 r[K];
  const SsmSelf& me;
  __device__ __forceinline__ explicit SsmRecord(const SsmSelf& self) : me(self) {}
  __device__ __forceinline__ void load(const f32x4* rec) {
#pragma unroll
    for (int j = 0; j < K; ++j) r[j] = rec[me.thread + j * THREADS];
  }
  // The first piece's place in a plane, and the others'.
  __device__ __forceinline__ int first() const {
    return KT::at(16 * (me.wave & 3) + me.c, 16 * (me.wave >> 2) + 4 * me.g);
  }
  static __device__ __forceinline__ int place(int first, int j) {
    return KT::kSwizzled ? first ^ j * kStep : first + j * kStep;
  }
  __device__ __forceinline__ void store(E* dst) const {
    const int o = first();
#pragma unroll
    for (int j = 0; j < K; ++j) {
      f32x4 rest = r[j];
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        const ssm_half<E> h = to_half<E>(rest);
        *reinterpret_cast<ssm_half<E>*>(dst + q * KT::size(kSsmP) + place(o, j)) = h;
        if (q + 1 < PL) rest -= half_f32(h);
      }
    }
  }
  // The sum of products of this record's values with those of another that stands in LDS.
  __device__ __forceinline__ float dot(const E* src) const {
    const int o = first();
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      f32x4 v = {};
#pragma unroll
      for (int q = PL - 1; q >= 0; --q)  // exact
        v += half_f32(*reinterpret_cast<const ssm_half<E>*>(src + q * KT::size(kSsmP) + place(o, j)));
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fmaf(r[j][i], v[i], sum);
    }
    return sum;
  }
};

// Sums over the 16 lanes c of a g, over the four g, over all.
__device__ __forceinline__ float sum_c(float v) { return sum_group<16>(v); }
__device__ __forceinline__ float sum_g(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float sum_wave(float v) { return sum_group<64>(v); }
// The sum over the lanes at and past each of a row of 16.
__device__ __forceinline__ float sum_lanes_from(float v) {
  v += dpp_move<0x101>(v);
  v += dpp_move<0x102>(v);
  v += dpp_move<0x104>(v);
  return v + dpp_move<0x108>(v);
}

__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) {
  return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3])));
}

// Adds the sums over the planes past the first to the first's, which they are kept apart from:
// the bf16 matrix instructions cut off what lies below the largest term's last bits, downwards,
// and small products added to a large sum lower it by 1.8e-9 of its size on average, products of one
// size by 1.2e-10 (64 terms).  Sums of 8 x 4096 tokens with B, C and x of mostly one sign gathered
// that: dA of a training step 0.4-1.2e-6 off for 0.7-2e-7 (371 us for 374).
template <int PLANES, int M, int N, int K>
__device__ __forceinline__ void ssm_add_rest(f32x4 (&acc)[M][N], const f32x4 (&rest)[K][N]) {
  if constexpr (PLANES > 1) {
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) acc[i][j] += rest[i][j];
  }
}

// ONE: P <= 64, a head is one block of columns, and M needs no registers between blocks (the
// training step of 8 x 4096 tokens 379 us, without the distinction 411).
template <typename E, int NP, bool VEC, bool ONE>
__global__ __launch_bounds__(ssm_grad_threads(NP), 2) void ssm_grad_kernel(SsmArgs a, SsmGrads o) {
  constexpr int L = ssm_chunk<E>(), LT = L / 16, NT = NP / 16, PT = kSsmP / 16;
  constexpr int THREADS = ssm_grad_threads(NP), WV = THREADS / 64;
  constexpr int TRI = LT * (LT + 1) / 2, TW = (TRI + WV - 1) / WV;
  // dB, dC: waves stand WN x NG over tiles of n and tokens, each with NN x TN tiles;
  // dx: WP x WS, PP x TP tiles of p and tokens
  constexpr int NG = LT == 4 && NT == 2 ? 4 : 2, WN = WV / NG, NN = NT / WN, TN = LT / NG;
  constexpr int WS = WV / 2 < LT ? WV / 2 : LT, WP = WV / WS, PP = PT / WP, TP = LT / WS;
  static_assert(WN <= WV / 2 && WP <= WV / 2, "places of the state terms");
  typedef SsmTile<E, NP> KT;
  typedef SsmTile<E, kSsmP> VT;
  typedef SsmTile<E, L> WT;
  constexpr int kRecord = kSsmP * NP / 4, kPlane = KT::size(kSsmP), kPlanes = ssm_planes<E>();
  __shared__ SsmGradLds<E, NP> m;
  typename KT::Lane kt;
  typename VT::Lane vt;
  typename WT::Lane wt;
  const int NC = (a.T + L - 1) / L, blocks = ONE ? 1 : (a.P + kSsmP - 1) / kSsmP;
  unsigned id = ssm_xcd_order();
  const int hb = id % o.blocks;
  id /= o.blocks;
  const int grp = id % a.G;
  id /= a.G;
  const int chunk = id % NC, b = id / NC;
  const int per = a.H / a.G, t0 = chunk * L, rows = min(L, a.T - t0);
  SsmSelf me;
  const int &wave = me.wave, &lane = me.lane, &c = me.c, &g = me.g;
  const int h0 = grp * per + hb * o.head_block;
  const int turns = (min((hb + 1) * o.head_block, per) - hb * o.head_block) * blocks;
  SsmRows<E, L, kSsmP, THREADS, VEC> rx(me), ry(me);
  SsmRecord<E, NP, THREADS> rs(me), rr(me);
  float4 rl;
  const auto record = [&](int turn) {
    return ((static_cast<size_t>(b * a.H + h0 + turn / blocks) * blocks + turn % blocks) * NC + chunk) *
           kRecord;
  };
  const auto fetch = [&](int turn) {
    const int h = h0 + turn / blocks, pb = turn % blocks, pc = pb * kSsmP, bh = b * a.H + h;
    rx.load(static_cast<const E*>(a.x) + b * a.xb + h * a.xh + t0 * a.xt + pc, a.xt, rows,
            a.P - pc);
    ry.load(static_cast<const E*>(a.dy) + b * a.yb + h * a.yh + t0 * a.yt + pc, a.yt, rows,
            a.P - pc);
    rs.load(o.fwd + record(turn));
    if (wave == 0) rl = ssm_log_row<L>(a, bh, NC)[t0];
  };
  {
    SsmRows<E, L, NP, THREADS, VEC> rb(me), rc(me);
    rb.load(static_cast<const E*>(a.Bm) + b * a.bb + grp * a.bg + t0 * a.bt, a.bt, rows, a.N);
    rc.load(static_cast<const E*>(a.Cm) + b * a.cb + grp * a.cg + t0 * a.ct, a.ct, rows, a.N);
    fetch(0);
    rr.load(o.rev + record(0));
    rb.store(m.b);
    rc.store(m.c);
  }
  for (int i = threadIdx.x; i < WT::size(L); i += THREADS) store_f32(m.w + i, 0.f), store_f32(m.mw + i, 0.f);
  lds_barrier();
  f32x4 cb[TW];  // C B^T: rows s, columns t, tiles wave, wave + WV, ...
  f32x4 dC[NN][TN] = {}, dB[NN][TN] = {};
#pragma unroll
  for (int j = 0; j < TW; ++j) {
    cb[j] = f32x4{};
    if (wave + WV * j < TRI) {
      int tt, ss;
      ssm_tri(wave + WV * j, tt, ss);
#pragma unroll
      for (int k = 0; k < NP; k += 32)
        cb[j] = mac2(kt.row(m.b, 16 * ss, k), kt.row(m.b, 16 * ss, k + 16),
                     kt.row(m.c, 16 * tt, k), kt.row(m.c, 16 * tt, k + 16), cb[j]);
    }
  }
  f32x4 mm[TW];  // M: rows s, columns t
  float qs[TN], ks[TP], dot = 0.f;
  for (int turn = 0; turn < turns; ++turn) {
    const int h = h0 + turn / blocks, pb = turn % blocks, pc = pb * kSsmP;
    const float D = a.D ? a.D[h] : 0.f;
    SsmChunkLog& lg = m.log[turn / blocks & 1];
    if (pb == 0) {
#pragma unroll
      for (int j = 0; j < TW; ++j) mm[j] = f32x4{};
#pragma unroll
      for (int j = 0; j < TN; ++j) qs[j] = 0.f;
#pragma unroll
      for (int j = 0; j < TP; ++j) ks[j] = 0.f;
      dot = 0.f;
    }
    // x, dy and st were last read before the barrier that ended the turn before
    rx.store(m.x);
    ry.store(m.dy);
    rs.store(m.st);
    if (wave == 0 && pb == 0) lg.template store<L>(rl);
    lds_barrier();
    kt.fresh(), vt.fresh(), wt.fresh(), me.fresh();
    bool above[4];  // the diagonal
#pragma unroll
    for (int i = 0; i < 4; ++i) above[i] = 4 * g + i > c;
#pragma unroll
    for (int j = 0; j < TW; ++j) {
      if (wave + WV * j >= TRI) break;
      int tt, ss;
      ssm_tri(wave + WV * j, tt, ss);
      const int t = 16 * tt + c, s = 16 * ss + 4 * g;
      f32x4 acc = ONE ? f32x4{} : mm[j];
#pragma unroll
      for (int k = 0; k < kSsmP; k += 32)
        acc = mac2(vt.row(m.x, 16 * ss, k), vt.row(m.x, 16 * ss, k + 16),
                   vt.row(m.dy, 16 * tt, k), vt.row(m.dy, 16 * tt, k + 16), acc);
      if (!ONE) mm[j] = acc;
      if (pb != 0 && pb + 1 != blocks) continue;
      f32x4 dec = lg.decay(t, s);
      const f32x4 step = lg.four(lg.step, s);
      if (tt == ss) {
#pragma unroll
        for (int i = 0; i < 4; ++i) dec[i] = above[i] ? 0.f : dec[i];
      }
      if (pb == 0) {  // W
        f32x4 w = cb[j] * dec * step;
        if (tt == ss) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = above[i] ? 0.f : w[i];
        }
        *reinterpret_cast<ssm_half<E>*>(m.w + WT::at(t, s)) = to_half<E>(w);
      }
      if (pb + 1 != blocks) continue;
      // M exp(l_t - l_s) step_s as an operand, and the sums of (C B^T) M exp(l_t - l_s): over
      // s with step_s (row), over t > s (col), s = t.  In a diagonal tile row holds, for
      // each token c of it, the pairs s < c <= t: sums over the lanes t >= c, then over s.
      const f32x4 f = acc * dec;
      f32x4 pair = f * cb[j];
      *reinterpret_cast<ssm_half<E>*>(m.mw + WT::at(t, s)) = to_half<E>(f * step);
      if (tt == ss) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * g + i == c) m.diag[t] = pair[i], m.trace[t] = acc[i], pair[i] = 0.f;
      }
      f32x4 part = pair * step;
      if (tt == ss) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          part[i] = sum_lanes_from(part[i]);
          part[i] = 4 * g + i < c ? part[i] : 0.f;
        }
      }
      const float row = sum_g((part[0] + part[1]) + (part[2] + part[3]));
      if (g == 0) m.row[ss][t] = row;
      f32x4 col;
#pragma unroll
      for (int i = 0; i < 4; ++i) col[i] = sum_c(pair[i]);
      if (c == 0) *reinterpret_cast<f32x4*>(&m.col[tt][s]) = col;
    }
    ssm_stretch();
    // exp(l_t) S dy_t, and its product with C_t
    int n0 = 16 * NN * (wave % WN), tn = wave / WN;  // tiles of tokens tn, tn + NG
    {
      f32x4 acc[NN][TN] = {}, rest[kPlanes > 1 ? NN : 1][TN] = {};
#pragma unroll
      for (int k = 0; k < kSsmP; k += 32) {
        ssm_half<E> y[TN][2];
#pragma unroll
        for (int j = 0; j < TN; ++j)
          y[j][0] = vt.row(m.dy, 16 * (tn + NG * j), k), y[j][1] = vt.row(m.dy, 16 * (tn + NG * j), k + 16);
#pragma unroll
        for (int i = 0; i < NN; ++i)
#pragma unroll
          for (int q = 0; q < kPlanes; ++q) {
            const auto s0 = kt.col(m.st + q * kPlane, n0 + 16 * i, k);
            const auto s1 = kt.col(m.st + q * kPlane, n0 + 16 * i, k + 16);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
              f32x4& sum = q ? rest[kPlanes > 1 ? i : 0][j] : acc[i][j];
              sum = mac2(s0, s1, y[j][0], y[j][1], sum);
            }
          }
      }
      ssm_add_rest<kPlanes>(acc, rest);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int tt = tn + NG * j;
        const float since = lg.since[16 * tt + c];
#pragma unroll
        for (int i = 0; i < NN; ++i) {
          qs[j] = fmaf(since, dot4(half_f32(kt.row(m.c, 16 * tt, n0 + 16 * i)), acc[i][j]), qs[j]);
          dC[i][j] += since * acc[i][j];
        }
      }
    }
    lds_barrier();
    dot += rr.dot(m.st);  // a thread's own pieces: it may overwrite them
    rr.store(m.st);
    ssm_stretch();
    if (turn + 1 < turns) fetch(turn + 1);
    lds_barrier();
    // exp(l_L - l_s) step_s R x_s: dB alone reads it, so R's leading bf16 is enough
    kt.fresh(), vt.fresh(), wt.fresh(), me.fresh();
    n0 = 16 * NN * (wave % WN), tn = wave / WN;
    {
      f32x4 acc[NN][TN] = {};
#pragma unroll
      for (int k = 0; k < kSsmP; k += 32) {
        ssm_half<E> x[TN][2];
#pragma unroll
        for (int j = 0; j < TN; ++j)
          x[j][0] = vt.row(m.x, 16 * (tn + NG * j), k), x[j][1] = vt.row(m.x, 16 * (tn + NG * j), k + 16);
#pragma unroll
        for (int i = 0; i < NN; ++i) {
          const auto r0 = kt.col(m.st, n0 + 16 * i, k), r1 = kt.col(m.st, n0 + 16 * i, k + 16);
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = mac2(r0, r1, x[j][0], x[j][1], acc[i][j]);
        }
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const float push = lg.push[16 * (tn + NG * j) + c];
#pragma unroll
        for (int i = 0; i < NN; ++i) dB[i][j] += push * acc[i][j];
      }
    }
    ssm_stretch();
    const int p0 = 16 * PP * (wave % WP), tp = wave / WP;  // tp, tp + WS
    {
      f32x4 acc[PP][TP] = {}, rest[kPlanes > 1 ? PP : 1][TP] = {};
#pragma unroll
      for (int k = 0; k < NP; k += 32) {
        ssm_half<E> v[TP][2];
#pragma unroll
        for (int j = 0; j < TP; ++j)
          v[j][0] = kt.row(m.b, 16 * (tp + WS * j), k), v[j][1] = kt.row(m.b, 16 * (tp + WS * j), k + 16);
#pragma unroll
        for (int i = 0; i < PP; ++i)
#pragma unroll
          for (int q = 0; q < kPlanes; ++q) {
            const auto r0 = kt.row(m.st + q * kPlane, p0 + 16 * i, k);
            const auto r1 = kt.row(m.st + q * kPlane, p0 + 16 * i, k + 16);
#pragma unroll
            for (int j = 0; j < TP; ++j) {
              f32x4& sum = q ? rest[kPlanes > 1 ? i : 0][j] : acc[i][j];
              sum = mac2(r0, r1, v[j][0], v[j][1], sum);
            }
          }
      }
      ssm_add_rest<kPlanes>(acc, rest);
      ssm_stretch();
#pragma unroll
      for (int j = 0; j < TP; ++j) {
        const int ss = tp + WS * j;
        const float left = lg.left[16 * ss + c], push = lg.push[16 * ss + c];
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          ks[j] = fmaf(left, dot4(half_f32(vt.row(m.x, 16 * ss, p0 + 16 * i)), acc[i][j]), ks[j]);
          acc[i][j] *= push;
        }
      }
      ssm_stretch();
#pragma unroll
      for (int r = 0; r < L; r += 32) {
        ssm_half<E> y[PP][2];
#pragma unroll
        for (int i = 0; i < PP; ++i)
          y[i][0] = vt.col(m.dy, p0 + 16 * i, r), y[i][1] = vt.col(m.dy, p0 + 16 * i, r + 16);
#pragma unroll
        for (int j = 0; j < TP; ++j) {
          const int ss = tp + WS * j;
          if (r + 16 < 16 * ss) continue;  // W_rs of the tiles r >= s
          const auto w0 = wt.col(m.w, 16 * ss, r), w1 = wt.col(m.w, 16 * ss, r + 16);
#pragma unroll
          for (int i = 0; i < PP; ++i) acc[i][j] = mac2(y[i][0], y[i][1], w0, w1, acc[i][j]);
        }
      }
#pragma unroll
      for (int j = 0; j < TP; ++j) {
        const int s = 16 * (tp + WS * j) + c;
        E* row = static_cast<E*>(o.dx) + ((static_cast<size_t>(b) * a.T + t0 + s) * a.H + h) * a.P;
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          const int p = pc + p0 + 16 * i + 4 * g;
          const f32x4 own = half_f32(vt.row(m.dy, 16 * (tp + WS * j), p0 + 16 * i));
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[i][j][k] = fmaf(D, own[k], acc[i][j][k]);
          if (s < rows) ssm_store4<VEC>(row + p, acc[i][j], p, a.P);
        }
      }
    }
    ssm_stretch();
    if (pb + 1 < blocks) {
      lds_barrier();
      rr.load(o.rev + record(turn + 1));
      continue;
    }
    me.fresh();
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const float q = sum_g(qs[j]);
      if (g == 0) m.q[wave % WN][16 * (tn + NG * j) + c] = q;
    }
#pragma unroll
    for (int j = 0; j < TP; ++j) {
      const float k = sum_g(ks[j]);
      if (g == 0) m.k[wave % WP][16 * (tp + WS * j) + c] = k;
    }
    dot = sum_wave(dot);
    if (lane == 0) m.dot[wave] = dot;
    lds_barrier();
    kt.fresh(), wt.fresh(), me.fresh();
    n0 = 16 * NN * (wave % WN), tn = wave / WN;
    if (turn + 1 < turns) rr.load(o.rev + record(turn + 1));
#pragma unroll
    for (int k = 0; k < L; k += 32) {
      ssm_half<E> kb[NN][2], kc[NN][2];
#pragma unroll
      for (int i = 0; i < NN; ++i) {
        kb[i][0] = kt.col(m.b, n0 + 16 * i, k), kb[i][1] = kt.col(m.b, n0 + 16 * i, k + 16);
        kc[i][0] = kt.col(m.c, n0 + 16 * i, k), kc[i][1] = kt.col(m.c, n0 + 16 * i, k + 16);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int tt = tn + NG * j;
        if (k <= 16 * tt) {
          const auto w0 = wt.row(m.mw, 16 * tt, k), w1 = wt.row(m.mw, 16 * tt, k + 16);
#pragma unroll
          for (int i = 0; i < NN; ++i) dC[i][j] = mac2(kb[i][0], kb[i][1], w0, w1, dC[i][j]);
        }
        if (k + 16 >= 16 * tt) {
          const auto w0 = wt.col(m.mw, 16 * tt, k), w1 = wt.col(m.mw, 16 * tt, k + 16);
#pragma unroll
          for (int i = 0; i < NN; ++i) dB[i][j] = mac2(kc[i][0], kc[i][1], w0, w1, dB[i][j]);
        }
      }
    }
    // the waves take turns at what one wave does
    if (wave == turn % WV) {
      // e_t = sum_{u >= t} q_u + sum_{s < t} step_s k_s + the state that passes through + the
      // pairs s < t <= u.  These, t being in tile tau: the ones of tiles ss < tau, as
      // sum_{u >= t} over all tiles (in after) less the tiles ss >= tau (later), which are the same
      // fp32 numbers and cancel in fp64; of tiles ss = tau < tt, sum_{s < t} step_s col; of the
      // diagonal tile, row.  So only rounding errors of pairs across t reach e_t: in fp32, all pairs
      // u >= t less the pairs s >= t would leave those of the whole chunk, which is the larger the
      // less the tokens cross.
      const int t = min(lane, L - 1), tau = t >> 4, at = t & 15;
      const bool in = lane < rows;
      const double step = lg.step[t];
      // all reads ahead of what selects among them: no branch, and one wait
      float from[LT - 1], to[LT - 1], of[LT - 1], qk[WN + WP];
#pragma unroll
      for (int j = 0; j < WN + WP; ++j) qk[j] = j < WN ? m.q[j][t] : m.k[j - WN][t];
#pragma unroll
      for (int j = 0; j + 1 < LT; ++j)
        from[j] = m.row[j][t], to[j] = m.col[j + 1][t], of[j] = m.row[tau][16 * (j + 1) + at];
      const float row = m.row[tau][t], own = m.col[tau][t] + m.diag[t];
      double after = 0.0, tile = 0.0, col = 0.0, k = 0.0;
#pragma unroll
      for (int j = 0; j < WN; ++j) after += qk[j];
#pragma unroll
      for (int j = WN; j < WN + WP; ++j) k += qk[j];
#pragma unroll
      for (int j = 0; j + 1 < LT; ++j) {
        after += j < tau ? from[j] : 0.f;
        col += j + 1 > tau ? to[j] : 0.f;
        tile += j + 1 > tau && 16 * (j + 1) + at < rows ? of[j] : 0.f;
      }
      const double direct = in ? own + col + k : 0.0;
      const double across = in ? step * col : 0.0, before = in ? step * k : 0.0;
      if (!in) after = tile = 0.0;
      // sum_{u >= t} after + sum_{s < t} before, from one running sum of their difference
      const double diff = scan_wave(before - after), total = read_lane(scan_wave(after), 63);
      const double tiles = scan_row(tile), sums = scan_row(across) - across;
      double later = 0.0;  // of the tiles ss >= tau
#pragma unroll
      for (int j = 0; j + 1 < LT; ++j) {
        const double all = read_lane(tiles, 16 * j + 15);
        later += j >= tau ? all : 0.0;
      }
      float through = 0.f;
#pragma unroll
      for (int j = 0; j < WV; ++j) through += m.dot[j];
      const double e = (total - later + (diff - (before - after))) + sums + row +
                       static_cast<double>(lg.all) * through;
      const double ddt = (direct + e * a.A[h]) * lg.gate[t];
      if (in)
        store_f32(static_cast<E*>(o.ddt) + (static_cast<size_t>(b) * a.T + t0 + lane) * a.H + h,
                  static_cast<float>(ddt));
      const double dA = scan_wave(in ? e * step : 0.0), db = scan_wave(in ? ddt : 0.0);
      const double dD = scan_wave(in ? m.trace[t] : 0.0);
      if (lane == 63) {
        double* part = o.part + (static_cast<size_t>(b) * NC + chunk) * 3 * a.H + h;
        part[0] = dA;
        part[a.H] = dD;
        part[2 * a.H] = db;
      }
    }
  }
  const int n0 = 16 * NN * (wave % WN), tn = wave / WN;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int t = 16 * (tn + NG * j) + c;
    if (t >= rows) break;
    const size_t at = ((static_cast<size_t>(b) * a.T + t0 + t) * a.G + grp) * a.N;
    const size_t all = static_cast<size_t>(a.B) * a.T * a.G * a.N;
#pragma unroll
    for (int i = 0; i < NN; ++i) {
      const int n = n0 + 16 * i + 4 * g;
      if (o.blocks > 1) {
        ssm_store4<VEC>(o.pB + hb * all + at + n, dB[i][j], n, a.N);
        ssm_store4<VEC>(o.pC + hb * all + at + n, dC[i][j], n, a.N);
      } else {
        ssm_store4<VEC>(static_cast<E*>(o.dBm) + at + n, dB[i][j], n, a.N);
        ssm_store4<VEC>(static_cast<E*>(o.dCm) + at + n, dC[i][j], n, a.N);
      }
    }
  }
}

// dB and dC from the sums of the head blocks.
template <typename E>
__global__ __launch_bounds__(256) void ssm_join_heads(SsmGrads o, size_t all) {
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= all) return;
  float b = 0.f, c = 0.f;
  for (int k = 0; k < o.blocks; ++k) b += o.pB[k * all + i], c += o.pC[k * all + i];
  store_f32(static_cast<E*>(o.dBm) + i, b);
  store_f32(static_cast<E*>(o.dCm) + i, c);
}

// ---- one token --------------------------------------------------------------------
// One workgroup per head: the state is read and written once (HBM bound), a thread
// holding V columns of every 256 / (columns / V)-th row; y is joined over the rows
// in LDS.  256 sequences of 16 heads, N = P = 64: 22 us, 135 MB at 6.1 TB/s (V = 1, for
// P that are no multiple of four: 25 us).
template <typename E, int V>
__global__ __launch_bounds__(256) void ssm_step_kernel(float* S, SsmArgs a) {
  __shared__ float red[256 * V];
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, grp = h / (a.H / a.G);
  const E* x = static_cast<const E*>(a.x) + b * a.xb + h * a.xh;
  const E* Bm = static_cast<const E*>(a.Bm) + b * a.bb + grp * a.bg;
  const E* Cm = static_cast<const E*>(a.Cm) + b * a.cb + grp * a.cg;
  const float step = static_cast<float>(
      ssm_step_of(to_f32(*(static_cast<const E*>(a.dt) + b * a.db + h * a.dh)), a.bias, h, a.softplus).step);
  const float decay = expf(step * a.A[h]);
  const int cols = a.P / V, lanes = 256 / cols;  // rows at once; P / V <= 256
  const int r0 = threadIdx.x / cols, pc = (threadIdx.x % cols) * V;
  float* s = S + static_cast<size_t>(blockIdx.x) * a.N * a.P + pc;
  float y[V] = {}, xv[V];
  if (r0 < lanes) {
#pragma unroll
    for (int i = 0; i < V; ++i) xv[i] = to_f32(x[pc + i]) * step;
#pragma unroll 4
    for (int n = r0; n < a.N; n += lanes) {
      float v[V];
      load_vec<V>(s + static_cast<size_t>(n) * a.P, v);
      const float bn = to_f32(Bm[n]), cn = to_f32(Cm[n]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = fmaf(decay, v[i], bn * xv[i]);
        y[i] = fmaf(cn, v[i], y[i]);
      }
      store_vec<V>(s + static_cast<size_t>(n) * a.P, v);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) red[r0 * a.P + pc + i] = y[i];
  }
  __syncthreads();
  for (int p = threadIdx.x; p < a.P; p += 256) {
    float sum = 0.f;
    for (int r = 0; r < lanes; ++r) sum += red[r * a.P + p];
    if (a.D) sum = fmaf(a.D[h], to_f32(x[p]), sum);
    store_f32(static_cast<E*>(a.y) + b * a.yb + h * a.yh + p, sum);
  }
}

// ---- launches ---------------------------------------------------------------------

inline int ssm_np(int N) { return N <= 32 ? 32 : (N <= 64 ? 64 : 128); }
inline int ssm_chunk_of(bool bf16) { return bf16 ? ssm_chunk<bf16_t>() : ssm_chunk<float>(); }

// Spans of a head: one workgroup each, so that the heads of a call with few of them
// still stand on every CU, four workgroups each where there are as many spans of four chunks:
// a span's own state costs one more pass over x and B.  (16 heads of 131072 tokens with 512,
// 768, 1024, 1536 and 2048 workgroups: 325, 310, 299, 311 and 303 us; a training step of
// 8 x 4096 tokens: 379, 379, 384, 390 and 402 us.)  Spans of two chunks only where those of
// four would leave CUs without a workgroup: with four and two, 16 heads of 500 tokens 25.1 and
// 18.9 us, of 2000 27.2 and 23.9, of 4000 34.1 and 33.2; 32 heads of 2000 30.9 and 31.0, 64
// heads of 2000 38 and 39 us.
inline void ssm_spans(int BHP, int T, int L, int& spans, int& span_chunks) {
  const int NC = (T + L - 1) / L;
  int n = (1024 + BHP - 1) / BHP;
  const int least = static_cast<long long>(BHP) * (NC / 4) < 256 ? 2 : 4;
  if (n > NC / least) n = NC / least;
  if (n < 1) n = 1;
  span_chunks = (NC + n - 1) / n;
  spans = (NC + span_chunks - 1) / span_chunks;
}

inline size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

struct SsmWorkspace {
  size_t logs, rec, log, fwd, rev, part, pB, pC, bytes;
  int spans, span_chunks, head_block, blocks;
};

inline SsmWorkspace ssm_workspace(int B, int T, int H, int G, int N, int P, bool bf16,
                                  bool backward) {
  SsmWorkspace w = {};
  const int L = ssm_chunk_of(bf16), NC = (T + L - 1) / L, blocks = (P + kSsmP - 1) / kSsmP;
  ssm_spans(B * H * blocks, T, L, w.spans, w.span_chunks);
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  w.logs = take(static_cast<size_t>(B) * H * NC * L * sizeof(float4));
  const size_t gaps = static_cast<size_t>(B) * H * (w.spans - 1);
  const int dirs = backward ? 2 : 1;
  w.rec = take(dirs * gaps * N * P * sizeof(float));
  w.log = take(dirs * gaps * sizeof(double));
  w.blocks = 1, w.head_block = H / G;
  if (backward) {
    const size_t rec = static_cast<size_t>(kSsmP) * ssm_np(N) * sizeof(float);
    const size_t all = static_cast<size_t>(B) * H * blocks * NC * rec;
    w.fwd = take(2 * all);
    w.rev = w.fwd + all;
    w.part = take(static_cast<size_t>(B) * NC * 3 * H * sizeof(double));
    // Heads of a group are split while there are fewer workgroups than the 256 CUs hold in
    // LDS, two each (N > 64: one); each split adds fp32 sums of dB and dC to write and read.
    // Training steps of B 2, T 2048, H 32, P 64, bf16, with room for 512 and for 256: N 64
    // 135 and 151 us, N 128 207 and 195 us; 1024: N 64 141, N 128 227 us.
    const long long wgs = static_cast<long long>(B) * G * NC, room = N > 64 ? 256 : 512;
    long long split = (room + wgs - 1) / wgs;
    if (split > H / G) split = H / G;
    w.head_block = static_cast<int>((H / G + split - 1) / split);
    w.blocks = (H / G + w.head_block - 1) / w.head_block;
    if (w.blocks > 1) {
      const size_t sums = static_cast<size_t>(w.blocks) * B * T * G * N * sizeof(float);
      w.pB = take(sums);
      w.pC = take(sums);
    }
  }
  w.bytes = at ? at : 256;
  return w;
}

#define KATA_TRY(CALL)                     \
  do {                                     \
    const hipError_t e_ = (CALL);          \
    if (e_ != hipSuccess) return e_;       \
  } while (0)

// The states between spans, forward (and reverse: dirs = 2).
template <typename E, int NP, bool VEC, bool EXACT>
hipError_t ssm_between_spans(const SsmArgs& a, int dirs, hipStream_t st) {
  if (a.spans < 2) return hipSuccess;
  const int blocks = (a.P + kSsmP - 1) / kSsmP;
  ssm_state_kernel<E, NP, false, VEC, EXACT>
      <<<static_cast<unsigned>(a.B) * a.H * blocks * (a.spans - 1) * dirs, 256, 0, st>>>(a, nullptr, dirs);
  KATA_TRY(hipGetLastError());
  if (a.N * a.P % 4 == 0)
    ssm_span_scan<4><<<dim3((a.N * a.P / 4 + 255) / 256, a.B * a.H, dirs), 256, 0, st>>>(a);
  else
    ssm_span_scan<1><<<dim3((a.N * a.P + 255) / 256, a.B * a.H, dirs), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <typename E>
hipError_t ssm_logs(const SsmArgs& a, hipStream_t st) {
  constexpr int L = ssm_chunk<E>();
  const int NC = (a.T + L - 1) / L;
  ssm_logs_kernel<E, L><<<static_cast<unsigned>(a.B) * NC * ((a.H + 3) / 4), 256, 0, st>>>(a, NC);
  return hipGetLastError();
}

template <typename E, int NP, bool VEC, bool EXACT>
hipError_t ssm_fwd_exact(const SsmArgs& a, hipStream_t st) {
  KATA_TRY(ssm_logs<E>(a, st));
  KATA_TRY((ssm_between_spans<E, NP, VEC, EXACT>(a, 1, st)));
  const int blocks = (a.P + kSsmP - 1) / kSsmP;
  ssm_out_kernel<E, NP, VEC, EXACT>
      <<<static_cast<unsigned>(a.B) * a.H * blocks * a.spans, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <typename E, int NP, bool VEC>
hipError_t ssm_fwd_np(const SsmArgs& a, hipStream_t st) {
  constexpr bool bf16 = sizeof(E) == 2;  // fp32 states need no parts
  return a.S_out ? ssm_fwd_exact<E, NP, VEC, bf16>(a, st) : ssm_fwd_exact<E, NP, VEC, false>(a, st);
}

template <typename E, int NP, bool VEC>
hipError_t ssm_bwd_np(const SsmArgs& a, const SsmGrads& o, f32x4* chunks, float* dA, float* dD,
                      float* dbias, hipStream_t st) {
  const int blocks = (a.P + kSsmP - 1) / kSsmP, L = ssm_chunk<E>(), NC = (a.T + L - 1) / L;
  KATA_TRY(ssm_logs<E>(a, st));
  KATA_TRY((ssm_between_spans<E, NP, VEC, sizeof(E) == 2>(a, 2, st)));
  ssm_state_kernel<E, NP, true, VEC, sizeof(E) == 2>
      <<<static_cast<unsigned>(a.B) * a.H * blocks * a.spans * 2, 256, 0, st>>>(a, chunks, 2);
  KATA_TRY(hipGetLastError());
  const unsigned grid = static_cast<unsigned>(a.B) * NC * a.G * o.blocks;
  constexpr int threads = ssm_grad_threads(NP);
  if (VEC && blocks == 1) ssm_grad_kernel<E, NP, VEC, VEC><<<grid, threads, 0, st>>>(a, o);
  else ssm_grad_kernel<E, NP, VEC, false><<<grid, threads, 0, st>>>(a, o);
  KATA_TRY(hipGetLastError());
  if (o.blocks > 1) {
    const size_t all = static_cast<size_t>(a.B) * a.T * a.G * a.N;
    ssm_join_heads<E><<<static_cast<unsigned>((all + 255) / 256), 256, 0, st>>>(o, all);
    KATA_TRY(hipGetLastError());
  }
  return launch_sum_partials(o.part, a.B * NC, 3 * a.H, {{dA, dD, dbias}, {a.H, a.H, a.H}}, st);
}

#define KATA_SSM_NP(CALL)                \
  switch (ssm_np(a.N)) {                 \
    case 32: return CALL(32);            \
    case 64: return CALL(64);            \
    default: return CALL(128);           \
  }

size_t ssm_workspace_bytes(int B, int T, int H, int G, int N, int P, bool bf16, bool backward) {
  return ssm_workspace(B, T, H, G, N, P, bf16, backward).bytes;
}

hipError_t launch_ssm_fwd(SsmArgs a, void* ws, bool bf16, hipStream_t st) {
  const SsmWorkspace w = ssm_workspace(a.B, a.T, a.H, a.G, a.N, a.P, bf16, false);
  char* base = static_cast<char*>(ws);
  a.spans = w.spans, a.span_chunks = w.span_chunks;
  a.logs = reinterpret_cast<float4*>(base + w.logs);
  a.rec = reinterpret_cast<float*>(base + w.rec);
  a.rec_log = reinterpret_cast<double*>(base + w.log);
  if (bf16) {
#define KATA_CALL(K) (a.vec ? ssm_fwd_np<bf16_t, K, true>(a, st) : ssm_fwd_np<bf16_t, K, false>(a, st))
    KATA_SSM_NP(KATA_CALL)
#undef KATA_CALL
  }
#define KATA_CALL(K) (a.vec ? ssm_fwd_np<float, K, true>(a, st) : ssm_fwd_np<float, K, false>(a, st))
  KATA_SSM_NP(KATA_CALL)
#undef KATA_CALL
}

hipError_t launch_ssm_bwd(SsmArgs a, void* dx, void* ddt, float* dA, void* dBm, void* dCm,
                          float* dD, float* dbias, void* ws, bool bf16, hipStream_t st) {
  const SsmWorkspace w = ssm_workspace(a.B, a.T, a.H, a.G, a.N, a.P, bf16, true);
  char* base = static_cast<char*>(ws);
  a.spans = w.spans, a.span_chunks = w.span_chunks;
  a.logs = reinterpret_cast<float4*>(base + w.logs);
  a.rec = reinterpret_cast<float*>(base + w.rec);
  a.rec_log = reinterpret_cast<double*>(base + w.log);
  const SsmGrads o = {dx, ddt, dBm, dCm, reinterpret_cast<float*>(base + w.pB),
                      reinterpret_cast<float*>(base + w.pC),
                      reinterpret_cast<double*>(base + w.part),
                      reinterpret_cast<const f32x4*>(base + w.fwd),
                      reinterpret_cast<const f32x4*>(base + w.rev), w.head_block, w.blocks};
  f32x4* chunks = reinterpret_cast<f32x4*>(base + w.fwd);
  if (bf16) {
#define KATA_CALL(K)                                                        \
  (a.vec ? ssm_bwd_np<bf16_t, K, true>(a, o, chunks, dA, dD, dbias, st)     \
         : ssm_bwd_np<bf16_t, K, false>(a, o, chunks, dA, dD, dbias, st))
    KATA_SSM_NP(KATA_CALL)
#undef KATA_CALL
  }
#define KATA_CALL(K)                                                       \
  (a.vec ? ssm_bwd_np<float, K, true>(a, o, chunks, dA, dD, dbias, st)     \
         : ssm_bwd_np<float, K, false>(a, o, chunks, dA, dD, dbias, st))
  KATA_SSM_NP(KATA_CALL)
#undef KATA_CALL
}
#undef KATA_SSM_NP

hipError_t launch_ssm_step(float* S, const SsmArgs& a, bool bf16, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(a.B) * a.H;
  const bool vec = a.P % 4 == 0;
  if (bf16) {
    if (vec) ssm_step_kernel<bf16_t, 4><<<grid, 256, 0, st>>>(S, a);
    else ssm_step_kernel<bf16_t, 1><<<grid, 256, 0, st>>>(S, a);
  } else {
    if (vec) ssm_step_kernel<float, 4><<<grid, 256, 0, st>>>(S, a);
    else ssm_step_kernel<float, 1><<<grid, 256, 0, st>>>(S, a);
  }
  return hipGetLastError();
}

}  // namespace kata
