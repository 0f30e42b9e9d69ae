// kata_conv.hpp -- causal depthwise convolution of W = 2..4 taps over the
// channels of a projection, with bias and SiLU:
//
//   pre[t] = bias + sum_{j<W} w[j] x[t - (W-1) + j],   y = pre sigmoid(pre) or pre,
//
// x before the first token being the W-1 rows of `state` (or zeros).  Backward:
// dpre = dy act'(pre), dx[t] = sum_j w[j] dpre[t + W-1 - j],
// dw[j] = sum_t dpre[t] x[t - (W-1) + j], dbias = sum_t dpre[t].
//
// All three kernels are bound by HBM: x (and dy) read once and y (dx) written
// once.  A thread owns V neighbouring channels and walks a run of tokens with
// the last W-1 rows in registers, so that only the run's first rows are read
// twice; channels go along the lanes, so every row of a wave is one piece.
// 8 x 4096 tokens of 1152 channels, W = 4, bf16: forward 36 us (165 MB counted, 4.6 TB/s),
// gradients 55 us (259 MB, 4.7 TB/s) and 5 us for their sums; both together 95 us, with rows
// that are not aligned 104 us.  One token of 256 sequences: 3.2 us, its launch's latency.
#pragma once

#include "kata_index.hpp"
#include "kata_rows.hpp"

namespace kata {

// Channels c .. c+V-1 of token t >= -(W-1): before the first token the state's rows.
template <typename E, int W, int V>
__device__ __forceinline__ void conv_row(const E* x, const E* state, const ConvShape& s, int b,
                                         int t, int c, float (&v)[V]) {
  if (t >= 0) {
    load_vec<V>(x + b * s.xb + t * s.xt + c, v);
  } else if (state) {
    load_vec<V>(state + (static_cast<long long>(b) * (W - 1) + (W - 1 + t)) * s.D + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
  }
}

// w[c][j] of V channels as wv[j][i]
template <int W, int V>
__device__ __forceinline__ void conv_weights(const float* w, int c, float (&wv)[W][V]) {
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < W; ++j) wv[j][i] = w[static_cast<size_t>(c + i) * W + j];
}

template <typename E, int W, int V, int R>
__global__ __launch_bounds__(256) void conv_fwd_kernel(const E* __restrict__ x,
                                                       const float* __restrict__ w,
                                                       const float* __restrict__ bias,
                                                       const E* __restrict__ state,
                                                       const int* __restrict__ lengths,
                                                       E* __restrict__ y,
                                                       E* __restrict__ state_out, ConvShape s,
                                                       int groups, int runs) {
  const long long id = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  const long long per = static_cast<long long>(groups) * runs;
  if (id >= per * s.B) return;
  const ConvPlace at = conv_place(id, groups, runs);
  const int b = at.b, run = at.run, c = at.group * V;
  const int len = lengths ? min(max(lengths[b], 0), s.T) : s.T;
  const int t0 = run * R, t1 = min(t0 + R, len);
  if (state_out && run == 0) {
    // the last W-1 rows of the state's rows followed by x[0 .. len)
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      float v[V];
      conv_row<E, W, V>(x, state, s, b, len - (W - 1) + j, c, v);
      store_vec<V>(state_out + (static_cast<long long>(b) * (W - 1) + j) * s.D + c, v);
    }
  }
  if (t0 >= t1) return;
  float wv[W][V], bv[V], past[W][V];
  conv_weights<W, V>(w, c, wv);
#pragma unroll
  for (int i = 0; i < V; ++i) bv[i] = bias ? bias[c + i] : 0.f;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_row<E, W, V>(x, state, s, b, t0 - (W - 1) + j, c, past[j]);
  const E* xp = x + b * s.xb + c;
  E* yp = y + b * s.yb + c;
  // four tokens at a time, the next four on their way (past the end: the last one again)
  RawVec<E, V> next[4];
  const auto fetch = [&](int t) {
#pragma unroll
    for (int k = 0; k < 4; ++k) next[k] = load_raw<E, V>(xp + min(t + k, t1 - 1) * s.xt);
  };
  fetch(t0);
  for (int t = t0; t < t1; t += 4) {
    RawVec<E, V> now[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) now[k] = next[k];
    if (t + 4 < t1) fetch(t + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      raw_f32<E, V>(now[k], past[W - 1]);
      float out[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float p = bv[i];
#pragma unroll
        for (int j = 0; j < W; ++j) p = fmaf(wv[j][i], past[j][i], p);
        out[i] = s.silu ? p * sigmoid(p) : p;
      }
      if (t + k < t1) store_vec<V>(yp + (t + k) * s.yt, out);
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) past[j][i] = past[j + 1][i];
    }
  }
}

// One token of every sequence: the state's rows move up by one.
template <typename E, int W, int V>
__global__ __launch_bounds__(256) void conv_step_kernel(E* __restrict__ state,
                                                        const E* __restrict__ x,
                                                        const float* __restrict__ w,
                                                        const float* __restrict__ bias,
                                                        E* __restrict__ y, ConvShape s,
                                                        int groups) {
  const long long id = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (id >= static_cast<long long>(groups) * s.B) return;
  const int b = static_cast<int>(id / groups), c = static_cast<int>(id - 1LL * b * groups) * V;
  E* sp = state + static_cast<long long>(b) * (W - 1) * s.D + c;
  float wv[W][V], rows[W][V], out[V];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) load_vec<V>(sp + static_cast<long long>(j) * s.D, rows[j]);
  load_vec<V>(x + b * s.xb + c, rows[W - 1]);
  conv_weights<W, V>(w, c, wv);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float p = bias ? bias[c + i] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) p = fmaf(wv[j][i], rows[j][i], p);
    out[i] = s.silu ? p * sigmoid(p) : p;
  }
  store_vec<V>(y + b * s.yb + c, out);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) store_vec<V>(sp + static_cast<long long>(j) * s.D, rows[j + 1]);
}

// Gradients.  A workgroup holds 64 channel groups (lanes) and takes runs of R
// tokens, one per wave at a time; pre is formed again from x, dpre of the W-1
// tokens past a run once more for its last dx.  dw and dbias are summed in
// registers over the runs of a wave, over the four waves in LDS, and written as
// one partial sum per workgroup, [D*W] then [D], for sum_partials.
//
// Runs of 32 tokens read 3/32 of the rows twice, runs of 8 3/8 of them; the short ones are
// for calls whose long runs are fewer than a wave for each of the 1024 SIMDs.  D 1152 bf16,
// runs of 32 and of 8: 100 tokens 17 and 9.1 us, 2000 18 and 12, 6000 (940 waves) 21 and 21,
// 12000 26 and 30, 32768 49 and 64.
inline int conv_bwd_run(int B, int T, int D) {
  const long long waves = (static_cast<long long>(T) + 31) / 32 * B * ((D + 255) / 256);
  return waves >= 1024 ? 32 : 8;
}

template <typename E, int W, int V, int R>
__global__ __launch_bounds__(256) void conv_bwd_kernel(const E* __restrict__ x,
                                                       const float* __restrict__ w,
                                                       const float* __restrict__ bias,
                                                       const E* __restrict__ dy,
                                                       E* __restrict__ dx,
                                                       float* __restrict__ part, ConvShape s,
                                                       int runs) {
  __shared__ float red[4][64][V * (W + 1)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = (blockIdx.x * 64 + lane) * V;
  const bool mine = c < s.D;
  float dw[W][V] = {}, db[V] = {};
  if (mine) {
    float wv[W][V], bv[V];
    conv_weights<W, V>(w, c, wv);
#pragma unroll
    for (int i = 0; i < V; ++i) bv[i] = bias ? bias[c + i] : 0.f;
    const long long all = static_cast<long long>(runs) * s.B;
    for (long long k = blockIdx.y * 4 + wave; k < all; k += 4LL * gridDim.y) {
      const int b = static_cast<int>(k / runs), t0 = static_cast<int>(k - 1LL * b * runs) * R;
      const int t1 = min(t0 + R, s.T);
      const E* xp = x + b * s.xb + c;
      const E* gp = dy + b * s.gb + c;
      E* dp = dx + b * s.yb + c;
      float past[W][V], g[W][V] = {};  // x[u-W+1 .. u]; dpre[u-W+1 .. u]
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        conv_row<E, W, V>(x, static_cast<const E*>(nullptr), s, b, t0 - (W - 1) + j, c, past[j]);
      // four tokens at a time, the next four on their way (past the end: the last one again,
      // with a dpre of zero)
      RawVec<E, V> nx[4], ng[4];
      const auto fetch = [&](int u) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = min(u + k, s.T - 1);
          nx[k] = load_raw<E, V>(xp + at * s.xt);
          ng[k] = load_raw<E, V>(gp + at * s.gt);
        }
      };
      const int end = t1 + W - 1;
      fetch(t0);
      for (int u0 = t0; u0 < end; u0 += 4) {
        RawVec<E, V> rx[4], rg[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) rx[k] = nx[k], rg[k] = ng[k];
        if (u0 + 4 < end) fetch(u0 + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int u = u0 + k;
          float gy[V], out[V];
          raw_f32<E, V>(rx[k], past[W - 1]);
          raw_f32<E, V>(rg[k], gy);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if (s.silu) {
              float p = bv[i];
#pragma unroll
              for (int j = 0; j < W; ++j) p = fmaf(wv[j][i], past[j][i], p);
              const float sg = sigmoid(p);
              gy[i] *= sg * fmaf(p, 1.f - sg, 1.f);
            }
            if (u >= s.T) gy[i] = 0.f;
            g[W - 1][i] = gy[i];
            float a = 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) a = fmaf(wv[j][i], g[W - 1 - j][i], a);
            out[i] = a;
          }
          if (u < t1) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
              db[i] += gy[i];
#pragma unroll
              for (int j = 0; j < W; ++j) dw[j][i] = fmaf(gy[i], past[j][i], dw[j][i]);
            }
          }
          if (u - (W - 1) >= t0 && u < end) store_vec<V>(dp + (u - (W - 1)) * s.yt, out);
#pragma unroll
          for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) past[j][i] = past[j + 1][i], g[j][i] = g[j + 1][i];
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int j = 0; j < W; ++j) red[wave][lane][i * W + j] = dw[j][i];
    red[wave][lane][V * W + i] = db[i];
  }
  __syncthreads();
  if (wave != 0 || !mine) return;
  float* row = part + static_cast<size_t>(blockIdx.y) * s.D * (W + 1);
#pragma unroll
  for (int i = 0; i < V * (W + 1); ++i) {
    const float a = red[0][lane][i] + red[1][lane][i] + (red[2][lane][i] + red[3][lane][i]);
    if (i < V * W) row[static_cast<size_t>(c) * W + i] = a;
    else row[static_cast<size_t>(s.D) * W + c + (i - V * W)] = a;
  }
}

// ---- launches ---------------------------------------------------------------

template <typename E>
constexpr int conv_vec() { return 16 / static_cast<int>(sizeof(E)); }

template <typename E, int W, int V>
hipError_t conv_fwd_runs(const E* x, const float* w, const float* bias, const E* state,
                         const int* lengths, E* y, E* state_out, const ConvShape& s,
                         hipStream_t st) {
  const int groups = s.D / V;
  // Runs of 16 tokens read 3/16 of the rows twice, runs of 4 3/4 of them (from the L2);
  // the short ones are for calls whose long runs would leave SIMDs without a wave.  D 1152
  // bf16, runs of 16 and of 4: 500 tokens 7.8 and 4.4 us, 2000 8.3 and 6.2, 6000 10.0 and
  // 10.7; a training step of 32768 tokens 95 and 108.
  const long long threads16 = static_cast<long long>(groups) * ((s.T + 15) / 16) * s.B;
  const bool wide = threads16 >= 256 * 256;
  const int R = wide ? 16 : 4;
  const int runs = (s.T + R - 1) / R;
  const long long blocks = (static_cast<long long>(groups) * runs * s.B + 255) / 256;
  const dim3 grid(static_cast<unsigned>(blocks));
  if (wide)
    conv_fwd_kernel<E, W, V, 16><<<grid, 256, 0, st>>>(x, w, bias, state, lengths, y, state_out, s,
                                                       groups, runs);
  else
    conv_fwd_kernel<E, W, V, 4><<<grid, 256, 0, st>>>(x, w, bias, state, lengths, y, state_out, s,
                                                      groups, runs);
  return hipGetLastError();
}

// Whether rows of V-channel pieces are aligned: channels, strides, base addresses.
template <typename E, int V>
bool conv_vec_ok(const ConvShape& s, std::initializer_list<const void*> p) {
  if (s.D % V || s.xb % V || s.xt % V || s.yb % V || s.yt % V || s.gb % V || s.gt % V) return false;
  return ptr_aligned(p, V * static_cast<int>(sizeof(E)));
}

#define KATA_CONV_TAPS(CALL)            \
  switch (W) {                          \
    case 2: return CALL(2);             \
    case 3: return CALL(3);             \
    default: return CALL(4);            \
  }

template <typename E>
hipError_t conv_fwd_e(const void* x, const float* w, const float* bias, const void* state,
                      const int* lengths, void* y, void* state_out, const ConvShape& s, int W,
                      hipStream_t st) {
  constexpr int V = conv_vec<E>();
  const bool vec = conv_vec_ok<E, V>(s, {x, state, y, state_out});
#define KATA_CALL(K)                                                                             \
  (vec ? conv_fwd_runs<E, K, V>(static_cast<const E*>(x), w, bias, static_cast<const E*>(state), \
                                lengths, static_cast<E*>(y), static_cast<E*>(state_out), s, st)  \
       : conv_fwd_runs<E, K, 1>(static_cast<const E*>(x), w, bias, static_cast<const E*>(state), \
                                lengths, static_cast<E*>(y), static_cast<E*>(state_out), s, st))
  KATA_CONV_TAPS(KATA_CALL)
#undef KATA_CALL
}

template <typename E, int W, int V>
hipError_t conv_step_v(E* state, const E* x, const float* w, const float* bias, E* y,
                       const ConvShape& s, hipStream_t st) {
  const int groups = s.D / V;
  const long long blocks = (static_cast<long long>(groups) * s.B + 255) / 256;
  conv_step_kernel<E, W, V><<<static_cast<unsigned>(blocks), 256, 0, st>>>(state, x, w, bias, y, s,
                                                                           groups);
  return hipGetLastError();
}

template <typename E>
hipError_t conv_step_e(void* state, const void* x, const float* w, const float* bias, void* y,
                       const ConvShape& s, int W, hipStream_t st) {
  constexpr int V = conv_vec<E>();
  const bool vec = conv_vec_ok<E, V>(s, {x, state, y});
#define KATA_CALL(K)                                                                              \
  (vec ? conv_step_v<E, K, V>(static_cast<E*>(state), static_cast<const E*>(x), w, bias,          \
                              static_cast<E*>(y), s, st)                                          \
       : conv_step_v<E, K, 1>(static_cast<E*>(state), static_cast<const E*>(x), w, bias,          \
                              static_cast<E*>(y), s, st))
  KATA_CONV_TAPS(KATA_CALL)
#undef KATA_CALL
}

// Workgroups along the runs: one run per wave up to 256 workgroups, whose partial
// sums are then a few percent of the traffic (training step of 32768 tokens: 95 us; up
// to 128 97 us, up to 512 95 us).
inline int conv_bwd_slices(int B, int T, int D) {
  const int R = conv_bwd_run(B, T, D);
  const long long runs = (static_cast<long long>(T) + R - 1) / R * B;
  const long long n = (runs + 3) / 4;
  return static_cast<int>(n < 256 ? n : 256);
}

size_t conv_bwd_workspace_bytes(int B, int T, int D, int W) {
  return (static_cast<size_t>(conv_bwd_slices(B, T, D)) * D * (W + 1) * sizeof(float) + 255) &
         ~static_cast<size_t>(255);
}

template <typename E, int W, int V>
hipError_t conv_bwd_v(const E* x, const float* w, const float* bias, const E* dy, E* dx, float* dw,
                      float* db, void* ws, const ConvShape& s, hipStream_t st) {
  float* part = static_cast<float*>(ws);
  const int R = conv_bwd_run(s.B, s.T, s.D);
  const int runs = (s.T + R - 1) / R, slices = conv_bwd_slices(s.B, s.T, s.D);
  const dim3 grid((s.D + 64 * V - 1) / (64 * V), slices);
  if (R == 32) conv_bwd_kernel<E, W, V, 32><<<grid, 256, 0, st>>>(x, w, bias, dy, dx, part, s, runs);
  else conv_bwd_kernel<E, W, V, 8><<<grid, 256, 0, st>>>(x, w, bias, dy, dx, part, s, runs);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_sum_partials(part, slices, s.D * (W + 1),
                             {{dw, db, nullptr}, {s.D * W, s.D, 0}}, st);
}

template <typename E>
hipError_t conv_bwd_e(const void* x, const float* w, const float* bias, const void* dy, void* dx,
                      float* dw, float* db, void* ws, const ConvShape& s, int W, hipStream_t st) {
  const bool vec = conv_vec_ok<E, 4>(s, {x, dy, dx});
#define KATA_CALL(K)                                                                             \
  (vec ? conv_bwd_v<E, K, 4>(static_cast<const E*>(x), w, bias, static_cast<const E*>(dy),       \
                             static_cast<E*>(dx), dw, db, ws, s, st)                             \
       : conv_bwd_v<E, K, 1>(static_cast<const E*>(x), w, bias, static_cast<const E*>(dy),       \
                             static_cast<E*>(dx), dw, db, ws, s, st))
  KATA_CONV_TAPS(KATA_CALL)
#undef KATA_CALL
}
#undef KATA_CONV_TAPS

hipError_t launch_conv_fwd(const void* x, const float* w, const float* bias, const void* state,
                           const int* lengths, void* y, void* state_out, const ConvShape& s, int W,
                           bool bf16, hipStream_t st) {
  return bf16 ? conv_fwd_e<bf16_t>(x, w, bias, state, lengths, y, state_out, s, W, st)
              : conv_fwd_e<float>(x, w, bias, state, lengths, y, state_out, s, W, st);
}
hipError_t launch_conv_step(void* state, const void* x, const float* w, const float* bias, void* y,
                            const ConvShape& s, int W, bool bf16, hipStream_t st) {
  return bf16 ? conv_step_e<bf16_t>(state, x, w, bias, y, s, W, st)
              : conv_step_e<float>(state, x, w, bias, y, s, W, st);
}
hipError_t launch_conv_bwd(const void* x, const float* w, const float* bias, const void* dy,
                           void* dx, float* dw, float* db, void* ws, const ConvShape& s, int W,
                           bool bf16, hipStream_t st) {
  return bf16 ? conv_bwd_e<bf16_t>(x, w, bias, dy, dx, dw, db, ws, s, W, st)
              : conv_bwd_e<float>(x, w, bias, dy, dx, dw, db, ws, s, W, st);
}

}  // namespace kata
