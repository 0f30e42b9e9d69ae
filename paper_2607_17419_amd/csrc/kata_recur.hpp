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
// A workgroup takes a span of 128 tokens of 128 channels: a lane two channels, a wave 16
// tokens.  Each wave's tokens act on a state as h -> exp(-L) h + H, L the sum of their rates; the
// waves' and the spans' (L, H) are joined in order, whatever order workgroups run in.  L and not
// the product of the a: where a = 1 - m 2^-24, its products round to 1 - (m + n) 2^-24 token
// by token, always to the same side (state after 20000 tokens at rates of 2e-5: 1.2e-5 off).
#pragma once

#include "kata_block.hpp"
#include "kata_rows.hpp"

namespace kata {

// c softplus(lam)
__device__ __forceinline__ float recur_slope(float lam, float c) {
  return c * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam))));
}

// sigmoid(x) and 1 - sigmoid(x), both to a few 2^-24 of themselves.
__device__ __forceinline__ void recur_sigmoid(float x, float& sig, float& rest) {
  const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * x);
  sig = __builtin_amdgcn_rcpf(1.f + e);
  rest = e < 1.f ? e * sig : 1.f - sig;
}
// Small rates make a near 1, where exp's own error is that of many tokens' product and
// 1 - a^2 cancels: below 1/4, 1 - a is formed first, by its series (the first term left out
// is 1e-8 of the sum), and a from it.
__device__ __forceinline__ float recur_less(float w) {
  float s = fmaf(w, -1.f / 5040.f, 1.f / 720.f);
  s = fmaf(w, -s, 1.f / 120.f);
  s = fmaf(w, -s, 1.f / 24.f);
  s = fmaf(w, -s, 1.f / 6.f);
  s = fmaf(w, -s, 0.5f);
  s = fmaf(w, -s, 1.f);
  return w * s;
}
__device__ __forceinline__ void recur_decay(float rate, float& a, float& beta) {
  const float small = recur_less(rate), e = __builtin_amdgcn_exp2f(-1.44269504088896341f * rate);
  const bool near = rate < 0.25f;
  const float less = near ? small : 1.f - e;  // 1 - a
  a = near ? 1.f - small : e;
  beta = __builtin_amdgcn_sqrtf(less * (1.f + a));
}

// How tokens whose rates sum to L act on a state, in one number: exp(-L), or -(1 - exp(-L)) where
// that is the more exact one.
__device__ __forceinline__ float recur_factor(float L) {
  const float w = L;
  float a, beta;
  recur_decay(w, a, beta);
  return w < 0.25f ? -recur_less(w) : fmaxf(a, 0x1p-126f);
}
__device__ __forceinline__ float recur_act(float factor, float h, float H) {
  const float f = fmaf(factor, h, H);
  return factor > 0.f ? f : h + f;
}

// V channels' constants.
template <int V>
struct RecurChannel {
  float slope[V], rb[V], ib[V];
};
template <int V>
__device__ __forceinline__ RecurChannel<V> recur_channel(const RecurArgs& s, int c) {
  RecurChannel<V> p;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int at = min(c + k, s.D - 1);
    p.slope[k] = recur_slope(s.lam[at], s.c);
    p.rb[k] = s.rb ? s.rb[at] : 0.f;
    p.ib[k] = s.ib ? s.ib[at] : 0.f;
  }
  return p;
}

// Channels c, c + 1 of a row (VEC: both there and aligned as a pair), raw.
template <bool VEC, typename E>
__device__ __forceinline__ RawVec<E, 2> recur_load(const E* row, int c, int D) {
  if constexpr (VEC) return load_raw<E, 2>(row + min(c, D - 2));
  else return RawVec<E, 2>{{row[min(c, D - 1)], row[min(c + 1, D - 1)]}};
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
__device__ __forceinline__ void recur_token(const RecurChannel<2>& p, const RawVec<E, 2>& x,
                                            const RawVec<E, 2>& r, const RawVec<E, 2>& i,
                                            float (&rate)[2], float (&a)[2], float (&b)[2]) {
  float xv[2], rv[2], iv[2];
  raw_f32<E, 2>(x, xv);
  raw_f32<E, 2>(r, rv);
  raw_f32<E, 2>(i, iv);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float beta;
    rate[k] = p.slope[k] * sigmoid(rv[k] + p.rb[k]);
    recur_decay(rate[k], a[k], beta);
    b[k] = beta * (sigmoid(iv[k] + p.ib[k]) * xv[k]);
  }
}

__device__ __forceinline__ int recur_length(const RecurArgs& s, int b) {
  return s.lengths ? min(max(s.lengths[b], 0), s.T) : s.T;
}

constexpr int kRecurRun = 16;    // tokens of a wave
constexpr int kRecurWaves = kRecurSpan / kRecurRun;

struct RecurPlace {
  int b, span, c, lane, wave, t0, len;
};
__device__ __forceinline__ RecurPlace recur_place(const RecurArgs& s) {
  RecurPlace p;
  const int tile = blockIdx.x % s.tiles, rest = blockIdx.x / s.tiles;
  p.b = rest % s.B, p.span = rest / s.B;
  p.lane = threadIdx.x & 63, p.wave = threadIdx.x >> 6;
  p.c = tile * kRecurCols + p.lane * 2;
  p.t0 = p.span * kRecurSpan + p.wave * kRecurRun;
  p.len = recur_length(s, p.b);
  return p;
}

// FINAL: y and the last state from the states before the spans; else a span's (L, H).
template <typename E, bool VEC, bool FINAL>
__global__ __launch_bounds__(64 * kRecurWaves) void recur_fwd_kernel(RecurArgs s) {
  __shared__ float2 act[kRecurWaves][kRecurCols];
  const RecurPlace at = recur_place(s);
  const size_t span = static_cast<size_t>(at.b) * s.spans + at.span;
  if (FINAL && at.span == 0 && at.len == 0 && s.h_out && at.wave == 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (at.c + k < s.D) {
        const size_t e = static_cast<size_t>(at.b) * s.D + at.c + k;
        s.h_out[e] = s.h_in ? s.h_in[e] : 0.f;
      }
  }
  if (at.span * kRecurSpan >= at.len) return;
  const E* x = static_cast<const E*>(s.x) + at.b * s.xb;
  const E* r = static_cast<const E*>(s.r) + at.b * s.rb_;
  const E* i = static_cast<const E*>(s.i) + at.b * s.ib_;
  RawVec<E, 2> xs[kRecurRun], rs[kRecurRun], is[kRecurRun];
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    const long long t = min(at.t0 + k, at.len - 1);
    xs[k] = recur_load<VEC>(x + t * s.xt, at.c, s.D);
    rs[k] = recur_load<VEC>(r + t * s.rt, at.c, s.D);
    is[k] = recur_load<VEC>(i + t * s.it, at.c, s.D);
  }
  const RecurChannel<2> p = recur_channel<2>(s, at.c);
  float a[kRecurRun][2], b[kRecurRun][2], L[2] = {0.f, 0.f}, H[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    float rate[2];
    recur_token<E>(p, xs[k], rs[k], is[k], rate, a[k], b[k]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (at.t0 + k >= at.len) rate[e] = 0.f, a[k][e] = 1.f, b[k][e] = 0.f;
      L[e] += rate[e];
      H[e] = fmaf(a[k][e], H[e], b[k][e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) act[at.wave][at.lane * 2 + e] = make_float2(FINAL ? recur_factor(L[e]) : L[e], H[e]);
  __syncthreads();
  if constexpr (!FINAL) {
    const int c = threadIdx.x, col = at.c - at.lane * 2 + c;
    if (c >= kRecurCols || col >= s.D) return;
    float2 all = act[0][c];
#pragma unroll
    for (int w = 1; w < kRecurWaves; ++w) {
      const float2 m = act[w][c];
      all = make_float2(all.x + m.x, recur_act(recur_factor(m.x), all.y, m.y));
    }
    s.sums[span * 2 * s.D + col] = all.x;
    s.sums[(span * 2 + 1) * s.D + col] = all.y;
  } else {
    E* y = static_cast<E*>(s.y) + at.b * s.yb;
    float h[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      h[e] = s.starts[span * s.D + min(at.c + e, s.D - 1)];
      for (int w = 0; w < at.wave; ++w) {
        const float2 m = act[w][at.lane * 2 + e];
        h[e] = recur_act(m.x, h[e], m.y);
      }
    }
#pragma unroll
    for (int k = 0; k < kRecurRun; ++k) {
#pragma unroll
      for (int e = 0; e < 2; ++e) h[e] = fmaf(a[k][e], h[e], b[k][e]);
      if (at.t0 + k < at.len) recur_store<VEC>(y + (at.t0 + k) * s.yt, at.c, s.D, h);
    }
    if (s.h_out && at.t0 < at.len && at.len <= at.t0 + kRecurRun) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (at.c + e < s.D) s.h_out[static_cast<size_t>(at.b) * s.D + at.c + e] = h[e];
    }
  }
}

// States between spans: forward from h_in into starts; REVERSE the values a_t G_t behind each
// span from the last on, and dh_in.
template <bool REVERSE>
__global__ __launch_bounds__(256) void recur_join_kernel(RecurArgs s) {
  const long long id = blockIdx.x * 256LL + threadIdx.x;
  if (id >= static_cast<long long>(s.B) * s.D) return;
  const int b = static_cast<int>(id / s.D), c = static_cast<int>(id - 1LL * b * s.D);
  const int len = recur_length(s, b), n = (len + kRecurSpan - 1) / kRecurSpan;
  const float* first = REVERSE ? s.dh_out : s.h_in;
  const float* __restrict__ sums = s.sums;
  float* __restrict__ out = REVERSE ? s.behind : s.starts;
  float h = first ? first[id] : 0.f;
  const size_t base = static_cast<size_t>(b) * s.spans;
#pragma unroll 8
  for (int k = 0; k < n; ++k) {
    const size_t span = base + (REVERSE ? n - 1 - k : k);
    const float L = sums[span * 2 * s.D + c], H = sums[(span * 2 + 1) * s.D + c];
    out[span * s.D + c] = h;
    h = recur_act(recur_factor(L), h, H);
  }
  if (REVERSE && s.dh_in) s.dh_in[id] = h;
}

// Gradients.  FINAL from the states before the spans and the values behind them; else a span's
// (L, R): the value a_t G_t of its first token from one behind it.
template <typename E, bool VEC, bool FINAL>
__global__ __launch_bounds__(64 * kRecurWaves) void recur_bwd_kernel(RecurArgs s) {
  __shared__ float2 act[kRecurWaves][kRecurCols];
  __shared__ float back[FINAL ? kRecurWaves : 1][kRecurCols];
  __shared__ float red[FINAL ? kRecurWaves : 1][3][kRecurCols];
  const RecurPlace at = recur_place(s);
  const size_t span = static_cast<size_t>(at.b) * s.spans + at.span;
  const int c = threadIdx.x, col = at.c - at.lane * 2 + c;  // of the sums over waves
  if (at.span * kRecurSpan >= at.len) {
    if (FINAL && c < kRecurCols && col < s.D)
      for (int k = 0; k < 3; ++k) s.part[(span * 3 + k) * s.D + col] = 0.f;
    return;
  }
  const E* x = static_cast<const E*>(s.x) + at.b * s.xb;
  const E* r = static_cast<const E*>(s.r) + at.b * s.rb_;
  const E* i = static_cast<const E*>(s.i) + at.b * s.ib_;
  const E* dy = static_cast<const E*>(s.dy) + at.b * s.yb;
  RawVec<E, 2> xs[FINAL ? kRecurRun : 1], rs[kRecurRun], is[FINAL ? kRecurRun : 1], gs[kRecurRun];
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    const long long t = min(at.t0 + k, at.len - 1);
    rs[k] = recur_load<VEC>(r + t * s.rt, at.c, s.D);
    gs[k] = recur_load<VEC>(dy + t * s.yt, at.c, s.D);
    if constexpr (FINAL) {
      xs[k] = recur_load<VEC>(x + t * s.xt, at.c, s.D);
      is[k] = recur_load<VEC>(i + t * s.it, at.c, s.D);
    }
  }
  const RecurChannel<2> p = recur_channel<2>(s, at.c);
  float L[2] = {0.f, 0.f}, H[2] = {0.f, 0.f}, R[2] = {0.f, 0.f};
  float before[FINAL ? kRecurRun : 1][2];
  float a[kRecurRun][2];
#pragma unroll
  for (int k = 0; k < kRecurRun; ++k) {
    const bool there = at.t0 + k < at.len;
    float b[2] = {0.f, 0.f}, rate[2];
    if constexpr (FINAL) {
      recur_token<E>(p, xs[k], rs[k], is[k], rate, a[k], b);
    } else {
      float rv[2], beta;
      raw_f32<E, 2>(rs[k], rv);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        rate[e] = p.slope[e] * sigmoid(rv[e] + p.rb[e]);
        recur_decay(rate[e], a[k][e], beta);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (!there) rate[e] = 0.f, a[k][e] = 1.f, b[e] = 0.f;
      if constexpr (FINAL) before[k][e] = H[e];  // from a zero state at the wave's first token
      L[e] += rate[e];
      H[e] = fmaf(a[k][e], H[e], b[e]);
    }
  }
#pragma unroll
  for (int k = kRecurRun - 1; k >= 0; --k) {
    float g[2];
    raw_f32<E, 2>(gs[k], g);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (at.t0 + k < at.len) R[e] = a[k][e] * (g[e] + R[e]);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    act[at.wave][at.lane * 2 + e] = make_float2(FINAL ? recur_factor(L[e]) : L[e], FINAL ? H[e] : R[e]);
    if constexpr (FINAL) back[at.wave][at.lane * 2 + e] = R[e];
  }
  __syncthreads();
  if constexpr (!FINAL) {
    if (c >= kRecurCols || col >= s.D) return;
    float2 all = act[kRecurWaves - 1][c];
#pragma unroll
    for (int w = kRecurWaves - 2; w >= 0; --w) {
      const float2 m = act[w][c];
      all = make_float2(all.x + m.x, recur_act(recur_factor(m.x), all.y, m.y));
    }
    s.sums[span * 2 * s.D + col] = all.x;
    s.sums[(span * 2 + 1) * s.D + col] = all.y;
  } else {
    float h[2], g[2], sum[3][2] = {};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int ch = min(at.c + e, s.D - 1), l = at.lane * 2 + e;
      h[e] = s.starts[span * s.D + ch];
      for (int w = 0; w < at.wave; ++w) h[e] = recur_act(act[w][l].x, h[e], act[w][l].y);
      g[e] = s.behind[span * s.D + ch];
      for (int w = kRecurWaves - 1; w > at.wave; --w) g[e] = recur_act(act[w][l].x, g[e], back[w][l]);
    }
    // the states before each token: what the state before the wave's first has become is added
#pragma unroll
    for (int k = 0; k < kRecurRun; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        before[k][e] += h[e];
        h[e] *= a[k][e];
      }
    E* dx = static_cast<E*>(s.dx) + at.b * s.dxb;
    E* dr = static_cast<E*>(s.dr) + at.b * s.drb;
    E* di = static_cast<E*>(s.di) + at.b * s.dib;
#pragma unroll
    for (int k = kRecurRun - 1; k >= 0; --k) {
      if (at.t0 + k >= at.len) continue;
      float xv[2], rv[2], iv[2], dyv[2], ox[2], orr[2], oi[2];
      raw_f32<E, 2>(xs[k], xv);
      raw_f32<E, 2>(rs[k], rv);
      raw_f32<E, 2>(is[k], iv);
      raw_f32<E, 2>(gs[k], dyv);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sig, rest, take, left, beta, same;
        recur_sigmoid(rv[e] + p.rb[e], sig, rest);
        recur_sigmoid(iv[e] + p.ib[e], take, left);
        const float rate = p.slope[e] * sig, u = take * xv[e];
        recur_decay(rate, same, beta);
        const float G = dyv[e] + g[e], ak = a[k][e];
        // rate / beta -> 0 with the rate
        const float ratio = beta > 0.f ? rate * __builtin_amdgcn_rcpf(beta) : 0.f;
        const float by_rate = -G * ak * (rate * before[k][e] - u * ak * ratio);
        const float du = G * beta;
        ox[e] = du * take;
        orr[e] = by_rate * rest;
        oi[e] = du * u * left;
        sum[0][e] += by_rate;
        sum[1][e] += orr[e];
        sum[2][e] += oi[e];
        g[e] = ak * G;
      }
      const long long t = at.t0 + k;
      recur_store<VEC>(dx + t * s.dxt, at.c, s.D, ox);
      recur_store<VEC>(dr + t * s.drt, at.c, s.D, orr);
      recur_store<VEC>(di + t * s.dit, at.c, s.D, oi);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) red[at.wave][k][at.lane * 2 + e] = sum[k][e];
    __syncthreads();
    if (c >= kRecurCols || col >= s.D) return;
    // sigmoid(lam) / softplus(lam)
    const float lam = s.lam[col];
    const float per = lam < -15.f ? 1.f : 1.f / ((1.f + expf(-lam)) * recur_slope(lam, 1.f));
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kRecurWaves; ++w) v += red[w][k][c];
      s.part[(span * 3 + k) * s.D + col] = k == 0 ? v * per : v;
    }
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
  recur_token<E>(recur_channel<2>(s, c), x, r, i, rate, a, u);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    hv[e] = fmaf(a[e], hv[e], u[e]);
    if (c + e < s.D) state[c + e] = hv[e];
  }
  recur_store<VEC>(static_cast<E*>(s.y) + b * s.yb, c, s.D, hv);
}

// ---- launches ---------------------------------------------------------------

int recur_spans(int T) { return (T + kRecurSpan - 1) / kRecurSpan; }

// The spans' (L, H) or (L, R), the states before or values behind them; gradients: partial sums,
// and the states before the spans.
size_t recur_workspace_bytes(int B, int T, int D, bool backward) {
  const size_t rows = static_cast<size_t>(B) * recur_spans(T) * D * sizeof(float);
  return ((backward ? 7 : 3) * rows + 255) & ~static_cast<size_t>(255);
}

template <typename E>
bool recur_vec(const RecurArgs& s) {
  const long long all = s.xb | s.xt | s.rb_ | s.rt | s.ib_ | s.it | s.yb | s.yt | s.dxb | s.dxt |
                        s.drb | s.drt | s.dib | s.dit;
  return s.D % 2 == 0 && all % 2 == 0 &&
         ptr_aligned({s.x, s.r, s.i, s.dy, s.y, s.dx, s.dr, s.di}, 2 * sizeof(E));
}

inline unsigned recur_blocks(const RecurArgs& s) {
  return static_cast<unsigned>(static_cast<long long>(s.B) * s.spans * s.tiles);
}
inline unsigned recur_join_blocks(const RecurArgs& s) {
  return static_cast<unsigned>((static_cast<long long>(s.B) * s.D + 255) / 256);
}

// The states before the spans, from s.sums on.
template <typename E, bool VEC>
hipError_t recur_states(const RecurArgs& s, hipStream_t st) {
  recur_fwd_kernel<E, VEC, false><<<recur_blocks(s), 64 * kRecurWaves, 0, st>>>(s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  recur_join_kernel<false><<<recur_join_blocks(s), 256, 0, st>>>(s);
  return hipGetLastError();
}

template <typename E, bool VEC>
hipError_t recur_fwd_v(const RecurArgs& s, hipStream_t st) {
  const hipError_t e = recur_states<E, VEC>(s, st);
  if (e != hipSuccess) return e;
  recur_fwd_kernel<E, VEC, true><<<recur_blocks(s), 64 * kRecurWaves, 0, st>>>(s);
  return hipGetLastError();
}

template <typename E, bool VEC>
hipError_t recur_bwd_v(const RecurArgs& s, bool have_starts, float* const (&sums)[3], hipStream_t st) {
  hipError_t e = have_starts ? hipSuccess : recur_states<E, VEC>(s, st);
  if (e != hipSuccess) return e;
  recur_bwd_kernel<E, VEC, false><<<recur_blocks(s), 64 * kRecurWaves, 0, st>>>(s);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  recur_join_kernel<true><<<recur_join_blocks(s), 256, 0, st>>>(s);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  recur_bwd_kernel<E, VEC, true><<<recur_blocks(s), 64 * kRecurWaves, 0, st>>>(s);
  e = hipGetLastError();
  if (e != hipSuccess || (!sums[0] && !sums[1] && !sums[2])) return e;
  return launch_sum_partials(s.part, s.B * s.spans, 3 * s.D,
                             {{sums[0], sums[1], sums[2]}, {s.D, s.D, s.D}}, st);
}

hipError_t launch_recur_fwd(RecurArgs s, void* ws, bool bf16, hipStream_t st) {
  s.spans = recur_spans(s.T), s.tiles = (s.D + kRecurCols - 1) / kRecurCols;
  const size_t rows = static_cast<size_t>(s.B) * s.spans * s.D;
  s.sums = static_cast<float*>(ws);
  if (!s.starts) s.starts = s.sums + 2 * rows;
  if (bf16) return recur_vec<bf16_t>(s) ? recur_fwd_v<bf16_t, true>(s, st) : recur_fwd_v<bf16_t, false>(s, st);
  return recur_vec<float>(s) ? recur_fwd_v<float, true>(s, st) : recur_fwd_v<float, false>(s, st);
}

hipError_t launch_recur_bwd(RecurArgs s, float* dlam, float* drb, float* dib, void* ws, bool bf16,
                            hipStream_t st) {
  s.spans = recur_spans(s.T), s.tiles = (s.D + kRecurCols - 1) / kRecurCols;
  const size_t rows = static_cast<size_t>(s.B) * s.spans * s.D;
  s.sums = static_cast<float*>(ws);
  s.behind = s.sums + 2 * rows;
  s.part = s.behind + rows;
  const bool have = s.starts != nullptr;
  if (!have) s.starts = s.part + 3 * rows;
  float* const sums[3] = {dlam, drb, dib};
  if (bf16)
    return recur_vec<bf16_t>(s) ? recur_bwd_v<bf16_t, true>(s, have, sums, st)
                                : recur_bwd_v<bf16_t, false>(s, have, sums, st);
  return recur_vec<float>(s) ? recur_bwd_v<float, true>(s, have, sums, st)
                             : recur_bwd_v<float, false>(s, have, sums, st);
}

hipError_t launch_recur_step(float* h, RecurArgs s, bool bf16, hipStream_t st) {
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
