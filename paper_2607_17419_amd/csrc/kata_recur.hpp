// kata_recur.hpp -- gated linear recurrence with a decay per channel and token:
//
//   rate_t = c softplus(lam) sigmoid(r_t + rb),   a_t = exp(-rate_t),
//   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t + ib) x_t,   y_t = h_t.
//
// Backward, with G_t = dy_t + a_{t+1} G_{t+1} the gradient of h_t, beta = sqrt(1 - a^2) and
// u = sigmoid(i) x:
//   drate = -G (a h_{t-1} - u a^2 / beta),   dr = drate rate (1 - sigmoid(r)),
//   dlam = sigmoid(lam) / softplus(lam) sum drate rate,
//   dx = G beta sigmoid(i),   di = G beta u (1 - sigmoid(i)).
//
// A workgroup takes a span of tokens of 128 channels: a lane two channels, a wave a run of
// tokens, whose inputs it reads once and holds in registers.  A run's tokens act on a state as
// h -> exp(-L) h + H, L the sum of their rates.  The waves' (L, H) are joined in LDS.  A span's
// is published in the workspace, and the state before it found from those of the spans before,
// in one fixed order, so that results do not depend on the order in which workgroups run.
// L and not the product of the a: where a = 1 - m 2^-24, its products round to 1 - (m + n) 2^-24
// token by token, always to the same side (state after 20000 tokens at rates of 2e-5: 1.2e-5 off).
//
// 131072 tokens of 1024 channels, bf16: 251 us, 4.3 TB/s of the 1.07 GB that are read and
// written once (three launches that form the spans' sums, join them and read everything again:
// 874); the vector units are busy 69% of the cycles (44 instructions an element, a sixth of
// them exponentials, reciprocals and roots at 2.5 times an addition's time), loads and
// arithmetic of the two workgroups of a CU overlap in part.  Training step of 8 x 4096 tokens:
// forward 75-81 us, gradients 164-175.  Runs of 8 tokens a wave: long 298 (for 268 then), training
// 257 (for 251).  fp32: 65536 tokens 206-217 us, training step of 8 x 2048 65-69 and 136-141 us, the
// gradients with one workgroup on a CU (156 registers).
#pragma once

#include "kata_block.hpp"
#include "kata_rows.hpp"

namespace kata {

// Within fp32's range, NaN as it is: so that a shut gate (a sigmoid of 0) is a rate of 0 and a gate
// of -inf stays shut, whatever finite parameters they meet.
__device__ __forceinline__ float recur_finite(float v) {
  return v > 3e38f ? 3e38f : v < -3e38f ? -3e38f : v;
}

// c softplus(lam) = c (max(lam, 0) + log(1 + e)), e = exp(-|lam|) <= 1: the logarithm as
// 2 atanh(z), z = e / (2 + e) <= 1/3, by its series (the first term left out is 2e-8 of it).
__device__ __forceinline__ float recur_slope(float lam, float c) {
  const float e = expf(-fabsf(lam)), z = e / (2.f + e), q = z * z;
  float s = fmaf(q, 1.f / 13.f, 1.f / 11.f);
  s = fmaf(q, s, 1.f / 9.f);
  s = fmaf(q, s, 1.f / 7.f);
  s = fmaf(q, s, 1.f / 5.f);
  s = fmaf(q, s, 1.f / 3.f);
  s = fmaf(q, s, 1.f);
  return recur_finite(c * (fmaxf(lam, 0.f) + 2.f * z * s));
}

// A gate's bias as part of exp(-(v + bias)) = exp2(v (-log2 e) + b) more: b = -bias log2 e rounded,
// more = exp2 of what the rounding left out, so that gates and biases that cancel leave no error
// (without it, |bias| 2^-24 of the exponential).  v + bias formed first is an instruction more: training
// step 255 us for 251, 131072 tokens 272 for 268.
constexpr float kLog2e = 1.44269504088896341f;
struct RecurBias {
  float b, more;
};
__device__ __forceinline__ RecurBias recur_bias(float bias) {
  const float b = recur_finite(-kLog2e * bias);
  return {b, __builtin_amdgcn_exp2f(fminf(fmaxf(fmaf(-kLog2e, bias, -b), -100.f), 100.f))};
}
// sigmoid of a gate and what is left of 1, both off by a few (1 + |v + bias|) 2^-24 of themselves.
__device__ __forceinline__ float recur_sigmoid(float v, const RecurBias& b) {
  return __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(fmaf(v, -kLog2e, b.b)), b.more, 1.f));
}
__device__ __forceinline__ void recur_sigmoid(float v, const RecurBias& b, float& sig, float& rest) {
  const float e = __builtin_amdgcn_exp2f(fmaf(v, -kLog2e, b.b)) * b.more;
  sig = __builtin_amdgcn_rcpf(1.f + e);
  rest = e < 1.f ? e * sig : 1.f - sig;
}

// Small rates make a near 1, where exp's own error is that of many tokens' product and
// 1 - a^2 cancels: below 1/8, 1 - a is formed first, by its series (the first term left out
// is 1e-9 of the sum), and a from it.  near (of the whole wave): all rates are below 1/8.
constexpr float kRecurNear = 0.125f;
__device__ __forceinline__ float recur_less(float w) {
  float s = fmaf(w, -1.f / 720.f, 1.f / 120.f);
  s = fmaf(w, -s, 1.f / 24.f);
  s = fmaf(w, -s, 1.f / 6.f);
  s = fmaf(w, -s, 0.5f);
  s = fmaf(w, -s, 1.f);
  return w * s;
}
__device__ __forceinline__ void recur_decay(float rate, bool near, float& a, float& beta) {
  float less = recur_less(rate);
  a = 1.f - less;
  if (!near) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * rate);
    const bool small = rate < kRecurNear;
    less = small ? less : 1.f - e;
    a = small ? a : e;
  }
  beta = __builtin_amdgcn_sqrtf(less * (1.f + a));
}
// How tokens whose rates sum to L act on a state, in one number that is no NaN: exp(-L), or
// -(1 - exp(-L)) where that is the more exact one.  exp(-L) as a square (off by 5 2^-24), so that small
// ones are fp32's subnormal numbers, which exp2 itself flushes (shifting its argument where it is low
// takes three instructions more, training step 242 us for 239); 0 as the least of them, so that the sign
// tells which it is.
__device__ __forceinline__ float recur_factor(float L) {
  const float root = __builtin_amdgcn_exp2f(-0.5f * kLog2e * L);
  return L < kRecurNear ? -recur_less(L) : fmaxf(root * root, 0x1p-149f);
}
__device__ __forceinline__ float recur_act(float factor, float h, float H) {
  const float f = fmaf(factor, h, H);
  return factor > 0.f ? f : h + f;
}

// Two channels' constants, slope = c softplus(lam).
struct RecurChannel {
  float slope[2];
  RecurBias rb[2], ib[2];
  bool near;  // of the whole wave
};
__device__ __forceinline__ RecurChannel recur_channel(const RecurArgs& s, int c) {
  RecurChannel p;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int at = min(c + k, s.D - 1);
    p.slope[k] = s.slopes ? s.slopes[at] : recur_slope(s.lam[at], s.c);
    p.rb[k] = recur_bias(s.rb ? s.rb[at] : 0.f);
    p.ib[k] = recur_bias(s.ib ? s.ib[at] : 0.f);
  }
  p.near = __all(p.slope[0] < kRecurNear && p.slope[1] < kRecurNear);
  return p;
}

// Channels c, c + 1 of a row (VEC: both there and aligned as a pair), raw.
template <bool VEC, typename E>
__device__ __forceinline__ RawVec<E, 2> recur_load(const E* row, int c, int D) {
  if constexpr (VEC) {
    if constexpr (sizeof(E) == 2)
      return __builtin_bit_cast(RawVec<E, 2>, *reinterpret_cast<const uint32_t*>(row + min(c, D - 2)));
    else
      return load_raw<E, 2>(row + min(c, D - 2));
  } else {
    return RawVec<E, 2>{{row[min(c, D - 1)], row[min(c + 1, D - 1)]}};
  }
}
// The same value, as far as the compiler can tell another: what was formed from it is formed again.
template <typename E>
__device__ __forceinline__ void recur_forget(RawVec<E, 2>& v) {
  struct Words { uint32_t w[sizeof(E) / 2]; };
  Words u = __builtin_bit_cast(Words, v);
#pragma unroll
  for (int k = 0; k < static_cast<int>(sizeof(E)) / 2; ++k) asm volatile("" : "+v"(u.w[k]));
  v = __builtin_bit_cast(RawVec<E, 2>, u);
}
template <bool VEC, typename E>
__device__ __forceinline__ void recur_store(E* row, int c, int D, const float (&v)[2]) {
  if constexpr (VEC) {
    if (c < D) {
      if constexpr (sizeof(E) == 2) *reinterpret_cast<uint32_t*>(row + c) = pack_bf16x2(v[0], v[1]);
      else *reinterpret_cast<float2*>(row + c) = make_float2(v[0], v[1]);
    }
  } else {
    if (c < D) store_f32(row + c, v[0]);
    if (c + 1 < D) store_f32(row + c + 1, v[1]);
  }
}

// rate, a and beta u of a token.
template <typename E>
__device__ __forceinline__ void recur_token(const RecurChannel& p, const RawVec<E, 2>& x,
                                            const RawVec<E, 2>& r, const RawVec<E, 2>& i,
                                            float (&rate)[2], float (&a)[2], float (&b)[2]) {
  float xv[2], rv[2], iv[2];
  raw_f32<E, 2>(x, xv);
  raw_f32<E, 2>(r, rv);
  raw_f32<E, 2>(i, iv);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float beta;
    rate[k] = p.slope[k] * recur_sigmoid(rv[k], p.rb[k]);
    recur_decay(rate[k], p.near, a[k], beta);
    b[k] = beta * (recur_sigmoid(iv[k], p.ib[k]) * xv[k]);
  }
}

// In the place of tokens past a sequence's end: a gate shut (a rate of 0), an input of 0, so
// that they leave the state as it is.
template <typename E>
__device__ __forceinline__ RawVec<E, 2> recur_pair(float v) {
  RawVec<E, 2> p;
  store_f32(&p.e[0], v);
  store_f32(&p.e[1], v);
  return p;
}

__device__ __forceinline__ int recur_length(const RecurArgs& s, int b) {
  return s.lengths ? min(max(s.lengths[b], 0), s.T) : s.T;
}

// ---- the chain of spans -----------------------------------------------------------
// A column is 128 channels of a sequence; its spans follow each other (backward: from the last
// on) in an order.  A word of 64 bits for each span and channel holds (L, H), and one for
// each sixteenth span (state behind it, 0); all ones: not there yet, which no such word is.  It
// is written and read as one relaxed atomic, so it needs no fence.  Workgroups take their spans
// from a counter, order by order: one that waits does so for workgroups that took theirs
// before it and are running, so every wait ends.  Should one not, it gives up after
// seconds, and its states are NaN.

constexpr int kRecurGroup = 16;
constexpr uint64_t kRecurNone = ~0ull;

__device__ __forceinline__ uint64_t recur_word(float lo, float hi) {
  return static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo);
}
__device__ __forceinline__ float recur_lo(uint64_t w) { return __uint_as_float(static_cast<uint32_t>(w)); }
__device__ __forceinline__ float recur_hi(uint64_t w) { return __uint_as_float(static_cast<uint32_t>(w >> 32)); }
__device__ __forceinline__ uint64_t recur_peek(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void recur_publish(uint64_t* p, uint64_t w) {
  __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t recur_wait(const uint64_t* p, uint64_t w) {
  for (int n = 0; w == kRecurNone && n < (1 << 22); ++n) {
    __builtin_amdgcn_s_sleep(2);
    w = recur_peek(p);
  }
  return w == kRecurNone ? recur_word(__builtin_nanf(""), __builtin_nanf("")) : w;
}

struct RecurTurn {
  int order, col;
};
__device__ __forceinline__ RecurTurn recur_turn(const RecurArgs& s, unsigned* shared) {
  if (threadIdx.x == 0) *shared = atomicAdd(s.ticket, 1u);
  __syncthreads();
  const unsigned id = __builtin_amdgcn_readfirstlane(*shared);
  const unsigned order = id / s.cols;
  return {static_cast<int>(order), static_cast<int>(id - order * s.cols)};
}

// The state before the span of this order, of channel threadIdx.x of the first 128 threads;
// publishes the span's own (L, H).  first: the state before order 0.  All threads of the
// workgroup fetch the words of the group's spans before, into `found`; they are joined to one
// (L, H) before the state behind the last group is waited for, so that a link of the chain is one
// multiply-add from word to word (131072 tokens of 128 channels 69 us; joined span by span behind
// it 113 us).
__device__ __forceinline__ float recur_before(const RecurArgs& s, const RecurTurn& t, float L, float H, float first,
                                              uint64_t (*found)[kRecurCols]) {
  const int ch = threadIdx.x % kRecurCols, q = threadIdx.x / kRecurCols;
  uint64_t* mine = s.words + (static_cast<size_t>(t.col) * s.spans + t.order) * kRecurCols + ch;
  if (q == 0) recur_publish(mine, recur_word(fmaxf(L, 0.f), H));  // (a NaN L goes with a NaN H)
  const int groups = s.spans / kRecurGroup, g = t.order / kRecurGroup, n = t.order % kRecurGroup;
  const uint64_t* back = mine - static_cast<size_t>(n) * kRecurCols;  // the group's first span
  uint64_t w[kRecurGroup / 4];
#pragma unroll
  for (int k = 0; k < kRecurGroup / 4; ++k)
    if (4 * k + q < n) w[k] = recur_peek(back + (4 * k + q) * kRecurCols);
#pragma unroll
  for (int k = 0; k < kRecurGroup / 4; ++k)
    if (4 * k + q < n) found[4 * k + q][ch] = recur_wait(back + (4 * k + q) * kRecurCols, w[k]);
  __syncthreads();
  if (q != 0) return 0.f;
  uint64_t* ends = s.words + (static_cast<size_t>(s.cols) * s.spans + static_cast<size_t>(t.col) * groups) * kRecurCols + ch;
  const uint64_t* end = ends + static_cast<size_t>(g - 1) * kRecurCols;  // (g > 0) behind the last group
  uint64_t behind = 0;
  if (g > 0) behind = recur_peek(end);
  float Lb = 0.f, Hb = 0.f;
  for (int k = 0; k < n; ++k) {
    const float Lk = recur_lo(found[k][ch]);
    Hb = recur_act(recur_factor(Lk), Hb, recur_hi(found[k][ch]));
    Lb += Lk;
  }
  const float by = recur_factor(Lb), all = recur_factor(Lb + L), Ha = recur_act(recur_factor(L), Hb, H);
  const float h = g > 0 ? recur_lo(recur_wait(end, behind)) : first;
  if (n == kRecurGroup - 1)
    recur_publish(ends + static_cast<size_t>(g) * kRecurCols, recur_word(recur_act(all, h, Ha), 0.f));
  return recur_act(by, h, Hb);
}

// No words yet, no turn taken: 16 bytes a thread, the first 256 bytes zero; and the channels'
// slopes, which each lane of the spans' workgroups would form again (7% of their instructions).
__global__ __launch_bounds__(256) void recur_clear_kernel(uint4* ws, size_t n, const float* lam, float c,
                                                          float* slopes, int D) {
  const size_t id = blockIdx.x * 256ull + threadIdx.x;
  const uint32_t v = id < 16 ? 0u : ~0u;
  if (id < n) ws[id] = make_uint4(v, v, v, v);
  else if (id - n < static_cast<size_t>(D)) slopes[id - n] = recur_slope(lam[id - n], c);
}

// ---- forward ------------------------------------------------------------------------

constexpr int kRecurRun = 16;                                // tokens of a wave
constexpr int kRecurWaves = 8;
constexpr int kRecurFwdSpan = kRecurRun * kRecurWaves;       // tokens of a workgroup
constexpr int kRecurBackRun = 8;
static_assert(kRecurBackRun * kRecurWaves == kRecurSpan && kRecurFwdSpan % kRecurSpan == 0, "");

// CHAIN: the sequences have more than one span.
template <typename E, bool VEC, bool CHAIN>
__global__ __launch_bounds__(64 * kRecurWaves, 4) void recur_fwd_kernel(RecurArgs s) {
  __shared__ float2 act[kRecurWaves][kRecurCols];
  __shared__ float sums[kRecurWaves][kRecurCols];
  __shared__ uint64_t found[CHAIN ? kRecurGroup : 1][kRecurCols];
  __shared__ float from[kRecurCols];
  __shared__ unsigned turn;
  RecurTurn at = {0, static_cast<int>(blockIdx.x)};
  if constexpr (CHAIN) at = recur_turn(s, &turn);
  const int b = at.col / s.tiles, c0 = (at.col - b * s.tiles) * kRecurCols;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int c = c0 + lane * 2, t0 = at.order * kRecurFwdSpan + wave * kRecurRun;
  const int len = recur_length(s, b), ch = threadIdx.x, col = c0 + ch;  // (ch: of the first 128 threads)
  const size_t state = static_cast<size_t>(b) * s.D;
  if (len == 0 && at.order == 0 && s.h_out && ch < kRecurCols && col < s.D)
    s.h_out[state + col] = s.h_in ? s.h_in[state + col] : 0.f;
  if (at.order * kRecurFwdSpan >= len) return;
  const E* x = static_cast<const E*>(s.x) + b * s.xb;
  const E* r = static_cast<const E*>(s.r) + b * s.rb_;
  const E* i = static_cast<const E*>(s.i) + b * s.ib_;
  RawVec<E, 2> xs[kRecurRun], rs[kRecurRun], is[kRecurRun];
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    const long long t = min(t0 + k, len - 1);
    xs[k] = recur_load<VEC>(x + t * s.xt, c, s.D);
    rs[k] = recur_load<VEC>(r + t * s.rt, c, s.D);
    is[k] = recur_load<VEC>(i + t * s.it, c, s.D);
  }
  __builtin_amdgcn_sched_barrier(0);  // the loads first
  const RecurChannel p = recur_channel(s, c);
  float a[kRecurRun][2], bu[kRecurRun][2], L[2] = {0.f, 0.f}, H[2] = {0.f, 0.f};
  if (t0 + kRecurRun > len) {
#pragma unroll
    for (int k = 0; k < kRecurRun; ++k)
      if (t0 + k >= len) {
        rs[k] = recur_pair<E>(-__builtin_inff());
        xs[k] = is[k] = recur_pair<E>(0.f);
      }
  }
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    float rate[2];
    recur_token<E>(p, xs[k], rs[k], is[k], rate, a[k], bu[k]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      L[e] += rate[e];
      H[e] = fmaf(a[k][e], H[e], bu[k][e]);
    }
    __builtin_amdgcn_sched_barrier(0);  // tokens one by one: more of them at once spill
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    act[wave][lane * 2 + e] = make_float2(recur_factor(L[e]), H[e]);
    sums[wave][lane * 2 + e] = L[e];
  }
  __syncthreads();
  float first = ch < kRecurCols && s.h_in && col < s.D ? s.h_in[state + col] : 0.f;
  if constexpr (CHAIN) {
    float all = 0.f, own = 0.f;
    if (ch < kRecurCols) {
#pragma unroll
      for (int w = 0; w < kRecurWaves; ++w) {
        all += sums[w][ch];
        own = recur_act(act[w][ch].x, own, act[w][ch].y);
      }
    }
    first = recur_before(s, at, all, own, first, found);
  }
  if (ch < kRecurCols) from[ch] = first;
  __syncthreads();
  float h[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    h[e] = from[lane * 2 + e];
    for (int w = 0; w < wave; ++w) h[e] = recur_act(act[w][lane * 2 + e].x, h[e], act[w][lane * 2 + e].y);
  }
  if (s.starts && t0 % kRecurSpan == 0 && t0 < len)
    recur_store<false>(s.starts + (static_cast<size_t>(b) * ((s.T + kRecurSpan - 1) / kRecurSpan) + t0 / kRecurSpan) * s.D,
                       c, s.D, h);
  if (!s.y) return;
  E* y = static_cast<E*>(s.y) + b * s.yb;
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
#pragma unroll
    for (int e = 0; e < 2; ++e) h[e] = fmaf(a[k][e], h[e], bu[k][e]);
    if (t0 + k < len) recur_store<VEC>(y + static_cast<long long>(t0 + k) * s.yt, c, s.D, h);
  }
  if (s.h_out && t0 < len && len <= t0 + kRecurRun) recur_store<false>(s.h_out + state, c, s.D, h);
}

// ---- gradients ------------------------------------------------------------------------

template <typename E, bool VEC, bool CHAIN>
__global__ __launch_bounds__(64 * kRecurWaves, sizeof(E) == 2 ? 4 : 2) void recur_bwd_kernel(RecurArgs s) {
  __shared__ float2 act[kRecurWaves][kRecurCols];
  __shared__ float sums[kRecurWaves][kRecurCols], back[kRecurWaves][kRecurCols];
  // the words found, then the sums over tokens
  __shared__ __align__(16) char both[sizeof(uint64_t) * kRecurGroup * kRecurCols];
  uint64_t(*found)[kRecurCols] = reinterpret_cast<uint64_t(*)[kRecurCols]>(both);
  float(*red)[3][kRecurCols] = reinterpret_cast<float(*)[3][kRecurCols]>(both);
  static_assert(sizeof(float) * kRecurWaves * 3 * kRecurCols <= sizeof(both), "");
  __shared__ float from[kRecurCols];
  __shared__ unsigned turn;
  RecurTurn at = {0, static_cast<int>(blockIdx.x)};
  if constexpr (CHAIN) at = recur_turn(s, &turn);
  const int b = at.col / s.tiles, c0 = (at.col - b * s.tiles) * kRecurCols;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int len = recur_length(s, b), ch = threadIdx.x, col = c0 + ch;  // (ch: of the first 128 threads)
  const int n = (len + kRecurSpan - 1) / kRecurSpan;
  const size_t state = static_cast<size_t>(b) * s.D;
  if (at.order >= n) {  // the spans past the end
    if (ch < kRecurCols && col < s.D) {
      for (int k = 0; k < 3; ++k) s.part[((static_cast<size_t>(b) * s.spans + at.order) * 3 + k) * s.D + col] = 0.f;
      if (n == 0 && at.order == 0 && s.dh_in) s.dh_in[state + col] = s.dh_out ? s.dh_out[state + col] : 0.f;
    }
    return;
  }
  const int which = n - 1 - at.order, c = c0 + lane * 2, t0 = which * kRecurSpan + wave * kRecurBackRun;
  const size_t span = static_cast<size_t>(b) * s.spans + which;
  const E* x = static_cast<const E*>(s.x) + b * s.xb;
  const E* r = static_cast<const E*>(s.r) + b * s.rb_;
  const E* i = static_cast<const E*>(s.i) + b * s.ib_;
  const E* dy = static_cast<const E*>(s.dy) + b * s.yb;
  RawVec<E, 2> xs[kRecurBackRun], rs[kRecurBackRun], is[kRecurBackRun], gs[kRecurBackRun];
#pragma unroll
  for (int k = 0; k < kRecurBackRun; ++k) {
    const long long t = min(t0 + k, len - 1);
    xs[k] = recur_load<VEC>(x + t * s.xt, c, s.D);
    rs[k] = recur_load<VEC>(r + t * s.rt, c, s.D);
    is[k] = recur_load<VEC>(i + t * s.it, c, s.D);
    gs[k] = recur_load<VEC>(dy + t * s.yt, c, s.D);
  }
  __builtin_amdgcn_sched_barrier(0);  // the loads first
  const RecurChannel p = recur_channel(s, c);
  float L[2] = {0.f, 0.f}, H[2] = {0.f, 0.f}, R[2] = {0.f, 0.f};
  float a[kRecurBackRun][2], rate[kRecurBackRun][2];
  float before[kRecurBackRun][2];  // the state before a token, from a zero state at the run's first
  if (t0 + kRecurBackRun > len) {
#pragma unroll
    for (int k = 0; k < kRecurBackRun; ++k)
      if (t0 + k >= len) {
        rs[k] = recur_pair<E>(-__builtin_inff());
        xs[k] = is[k] = gs[k] = recur_pair<E>(0.f);
      }
  }
#pragma unroll
  for (int k = 0; k < kRecurBackRun; ++k) {
    float xv[2], rv[2], iv[2];
    raw_f32<E, 2>(xs[k], xv);
    raw_f32<E, 2>(rs[k], rv);
    raw_f32<E, 2>(is[k], iv);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float beta;
      rate[k][e] = p.slope[e] * recur_sigmoid(rv[e], p.rb[e]);
      recur_decay(rate[k][e], p.near, a[k][e], beta);
      const float bu = beta * (recur_sigmoid(iv[e], p.ib[e]) * xv[e]);
      before[k][e] = H[e];
      L[e] += rate[k][e];
      H[e] = fmaf(a[k][e], H[e], bu);
    }
    __builtin_amdgcn_sched_barrier(0);  // tokens one by one: more of them at once spill
  }
#pragma unroll
  for (int k = kRecurBackRun - 1; k >= 0; --k) {
    float g[2];
    raw_f32<E, 2>(gs[k], g);
#pragma unroll
    for (int e = 0; e < 2; ++e) R[e] = a[k][e] * (g[e] + R[e]);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    act[wave][lane * 2 + e] = make_float2(recur_factor(L[e]), H[e]);
    sums[wave][lane * 2 + e] = L[e];
    back[wave][lane * 2 + e] = R[e];
  }
  __syncthreads();
  {
    float first = ch < kRecurCols && s.dh_out && col < s.D ? s.dh_out[state + col] : 0.f;
    float all = 0.f, own = 0.f;
    if (ch < kRecurCols) {
#pragma unroll
      for (int w = kRecurWaves - 1; w >= 0; --w) {
        all += sums[w][ch];
        own = recur_act(act[w][ch].x, own, back[w][ch]);
      }
    }
    if constexpr (CHAIN) first = recur_before(s, at, all, own, first, found);
    if (ch < kRecurCols) {
      from[ch] = first;
      if (which == 0 && s.dh_in && col < s.D) s.dh_in[state + col] = recur_act(recur_factor(all), first, own);
    }
  }
  __syncthreads();
  float h[2], g[2], sum[3][2] = {};
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int l = lane * 2 + e;
    h[e] = s.starts[span * s.D + min(c + e, s.D - 1)];
    for (int w = 0; w < wave; ++w) h[e] = recur_act(act[w][l].x, h[e], act[w][l].y);
    g[e] = from[l];
    for (int w = kRecurWaves - 1; w > wave; --w) g[e] = recur_act(act[w][l].x, g[e], back[w][l]);
  }
  // what the state before the run's first token has become is added to the states before each
#pragma unroll
  for (int k = 0; k < kRecurBackRun; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      before[k][e] += h[e];
      h[e] *= a[k][e];
    }
  E* dx = static_cast<E*>(s.dx) + b * s.dxb;
  E* dr = static_cast<E*>(s.dr) + b * s.drb;
  E* di = static_cast<E*>(s.di) + b * s.dib;
#pragma unroll
  for (int k = kRecurBackRun - 1; k >= 0; --k) {
    if (t0 + k >= len) continue;
    // the gates once more: kept, they would halve the waves of a CU (training step 276 us)
    float xv[2], rv[2], iv[2], dyv[2], ox[2], orr[2], oi[2];
    for (auto* v : {&xs[k], &rs[k], &is[k], &gs[k]}) recur_forget<E>(*v);
    asm volatile("" : "+v"(rate[k][0]), "+v"(rate[k][1]));
    raw_f32<E, 2>(xs[k], xv);
    raw_f32<E, 2>(rs[k], rv);
    raw_f32<E, 2>(is[k], iv);
    raw_f32<E, 2>(gs[k], dyv);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float take, left, sig, rest, same, beta;
      recur_sigmoid(iv[e], p.ib[e], take, left);
      recur_sigmoid(rv[e], p.rb[e], sig, rest);
      recur_decay(rate[k][e], p.near, same, beta);
      const float u = take * xv[e], G = dyv[e] + g[e], ag = a[k][e] * G;
      // rate / beta -> 0 with the rate
      const float ratio = beta > 0.f ? rate[k][e] * __builtin_amdgcn_rcpf(beta) : 0.f;
      // (a shut state, a = 0, meets its rate before anything else, so that no product is 0 inf)
      const float by_rate = ag * (u * a[k][e] * ratio) - ag * rate[k][e] * before[k][e];
      const float du = G * beta;
      ox[e] = du * take;
      orr[e] = by_rate * rest;
      oi[e] = du * u * left;
      sum[0][e] += by_rate;
      sum[1][e] += orr[e];
      sum[2][e] += oi[e];
      g[e] = ag;
    }
    const long long t = t0 + k;
    recur_store<VEC>(dx + t * s.dxt, c, s.D, ox);
    recur_store<VEC>(dr + t * s.drt, c, s.D, orr);
    recur_store<VEC>(di + t * s.dit, c, s.D, oi);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) red[wave][k][lane * 2 + e] = sum[k][e];
  __syncthreads();
  if (ch >= kRecurCols || col >= s.D) return;
  // sigmoid(lam) / softplus(lam)
  const float lam = s.lam[col];
  const float per = lam < -15.f ? 1.f : 1.f / ((1.f + expf(-lam)) * recur_slope(lam, 1.f));
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kRecurWaves; ++w) v += red[w][k][ch];
    s.part[(span * 3 + k) * s.D + col] = k == 0 ? v * per : v;
  }
}

// One token of every sequence.
template <typename E, bool VEC>
__global__ __launch_bounds__(256) void recur_step_kernel(float* __restrict__ h, RecurArgs s, int pairs) {
  const long long id = blockIdx.x * 256LL + threadIdx.x;
  if (id >= static_cast<long long>(pairs) * s.B) return;
  const int b = static_cast<int>(id / pairs), c = 2 * static_cast<int>(id - 1LL * b * pairs);
  const RawVec<E, 2> x = recur_load<VEC>(static_cast<const E*>(s.x) + b * s.xb, c, s.D);
  const RawVec<E, 2> r = recur_load<VEC>(static_cast<const E*>(s.r) + b * s.rb_, c, s.D);
  const RawVec<E, 2> i = recur_load<VEC>(static_cast<const E*>(s.i) + b * s.ib_, c, s.D);
  float* state = h + static_cast<long long>(b) * s.D;
  float hv[2] = {state[c], state[min(c + 1, s.D - 1)]}, rate[2], a[2], u[2];
  recur_token<E>(recur_channel(s, c), x, r, i, rate, a, u);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    hv[e] = fmaf(a[e], hv[e], u[e]);
    if (c + e < s.D) state[c + e] = hv[e];
  }
  recur_store<VEC>(static_cast<E*>(s.y) + b * s.yb, c, s.D, hv);
}

// ---- launches ---------------------------------------------------------------

int recur_spans(int T) { return (T + kRecurSpan - 1) / kRecurSpan; }

// Bytes of the chain of `spans` spans of each column: the counter, the words; then the slopes.
inline size_t recur_word_bytes(int B, int D, int spans) {
  const size_t cols = static_cast<size_t>(B) * ((D + kRecurCols - 1) / kRecurCols);
  return 256 + cols * (spans + spans / kRecurGroup) * kRecurCols * sizeof(uint64_t);
}
inline size_t recur_chain_bytes(int B, int D, int spans) {
  if (spans < 2) return 0;
  return recur_word_bytes(B, D, spans) + ((D * sizeof(float) + 255) & ~static_cast<size_t>(255));
}
// A chain; gradients: partial sums, and the states before the spans.
size_t recur_workspace_bytes(int B, int T, int D, bool backward) {
  const int fwd = (T + kRecurFwdSpan - 1) / kRecurFwdSpan, bwd = recur_spans(T);
  const size_t chain = recur_chain_bytes(B, D, backward ? bwd : fwd);
  const size_t rows = backward ? 4 * static_cast<size_t>(B) * bwd * D * sizeof(float) : 0;
  const size_t all = (chain + rows + 255) & ~static_cast<size_t>(255);
  return all ? all : 256;
}

template <typename E>
bool recur_vec(const RecurArgs& s) {
  const long long all = s.xb | s.xt | s.rb_ | s.rt | s.ib_ | s.it | s.yb | s.yt | s.dxb | s.dxt |
                        s.drb | s.drt | s.dib | s.dit;
  return s.D % 2 == 0 && all % 2 == 0 &&
         ptr_aligned({s.x, s.r, s.i, s.dy, s.y, s.dx, s.dr, s.di}, 2 * sizeof(E));
}

// The chain in `ws`, cleared, and the slopes; the grid.
inline hipError_t recur_chain(RecurArgs& s, int spans, void* ws, unsigned& blocks, hipStream_t st) {
  s.spans = spans;
  s.tiles = (s.D + kRecurCols - 1) / kRecurCols;
  s.cols = s.B * s.tiles;
  s.ticket = static_cast<unsigned*>(ws);
  s.words = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + 256);
  blocks = static_cast<unsigned>(static_cast<long long>(s.cols) * spans);
  s.slopes = nullptr;
  if (spans < 2) return hipSuccess;
  const size_t words = recur_word_bytes(s.B, s.D, spans), n = words / 16;
  float* slopes = reinterpret_cast<float*>(static_cast<char*>(ws) + words);
  s.slopes = slopes;
  recur_clear_kernel<<<static_cast<unsigned>((n + s.D + 255) / 256), 256, 0, st>>>(
      static_cast<uint4*>(ws), n, s.lam, s.c, slopes, s.D);
  return hipGetLastError();
}

template <typename E, bool VEC>
hipError_t recur_fwd_v(RecurArgs s, void* ws, hipStream_t st) {
  unsigned blocks;
  const hipError_t e = recur_chain(s, (s.T + kRecurFwdSpan - 1) / kRecurFwdSpan, ws, blocks, st);
  if (e != hipSuccess) return e;
  if (s.spans > 1) recur_fwd_kernel<E, VEC, true><<<blocks, 64 * kRecurWaves, 0, st>>>(s);
  else recur_fwd_kernel<E, VEC, false><<<blocks, 64 * kRecurWaves, 0, st>>>(s);
  return hipGetLastError();
}

template <typename E, bool VEC>
hipError_t recur_bwd_v(RecurArgs s, float* const (&sums)[3], void* ws, hipStream_t st) {
  const int spans = recur_spans(s.T);
  float* rows = reinterpret_cast<float*>(static_cast<char*>(ws) + recur_chain_bytes(s.B, s.D, spans));
  s.part = rows;
  hipError_t e;
  if (!s.starts) {
    // the forward's chain first, in the same place (it is the shorter one)
    RecurArgs f = s;
    f.y = nullptr, f.h_out = nullptr;
    f.starts = s.starts = rows + 3 * static_cast<size_t>(s.B) * spans * s.D;
    e = recur_fwd_v<E, VEC>(f, ws, st);
    if (e != hipSuccess) return e;
  }
  unsigned blocks;
  e = recur_chain(s, spans, ws, blocks, st);
  if (e != hipSuccess) return e;
  if (spans > 1) recur_bwd_kernel<E, VEC, true><<<blocks, 64 * kRecurWaves, 0, st>>>(s);
  else recur_bwd_kernel<E, VEC, false><<<blocks, 64 * kRecurWaves, 0, st>>>(s);
  e = hipGetLastError();
  if (e != hipSuccess || (!sums[0] && !sums[1] && !sums[2])) return e;
  return launch_sum_partials(s.part, s.B * spans, 3 * s.D,
                             {{sums[0], sums[1], sums[2]}, {s.D, s.D, s.D}}, st);
}

hipError_t launch_recur_fwd(const RecurArgs& s, void* ws, bool bf16, hipStream_t st) {
  if (bf16) return recur_vec<bf16_t>(s) ? recur_fwd_v<bf16_t, true>(s, ws, st) : recur_fwd_v<bf16_t, false>(s, ws, st);
  return recur_vec<float>(s) ? recur_fwd_v<float, true>(s, ws, st) : recur_fwd_v<float, false>(s, ws, st);
}

hipError_t launch_recur_bwd(const RecurArgs& s, float* dlam, float* drb, float* dib, void* ws, bool bf16,
                            hipStream_t st) {
  float* const sums[3] = {dlam, drb, dib};
  if (bf16)
    return recur_vec<bf16_t>(s) ? recur_bwd_v<bf16_t, true>(s, sums, ws, st)
                                : recur_bwd_v<bf16_t, false>(s, sums, ws, st);
  return recur_vec<float>(s) ? recur_bwd_v<float, true>(s, sums, ws, st)
                             : recur_bwd_v<float, false>(s, sums, ws, st);
}

hipError_t launch_recur_step(float* h, const RecurArgs& s, bool bf16, hipStream_t st) {
  const int pairs = (s.D + 1) / 2;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(pairs) * s.B + 255) / 256);
#define KATA_STEP(E, VEC) recur_step_kernel<E, VEC><<<blocks, 256, 0, st>>>(h, s, pairs)
  if (bf16) {
    if (recur_vec<bf16_t>(s)) KATA_STEP(bf16_t, true);
    else KATA_STEP(bf16_t, false);
  } else {
    if (recur_vec<float>(s)) KATA_STEP(float, true);
    else KATA_STEP(float, false);
  }
#undef KATA_STEP
  return hipGetLastError();
}

}  // namespace kata
