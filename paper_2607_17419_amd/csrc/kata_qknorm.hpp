// kata_qknorm.hpp -- norms of query and key heads with the position rotation in
// the same pass, from the token-major rows a projection writes to the head-major
// [B][H][T][d] that the attention entry points read:
//
//   hat = x / sqrt(mean(x^2) + eps)   (RMS; L2: sum for mean; none: hat = x)
//   y   = R(pos) (w hat),             R turning pair i by the angle pos freq[i].
//
// Backward, with e = R(pos)^T dy: dw = sum e hat, g = w e,
//   dx = (g - hat mean(g hat)) / sqrt(mean(x^2) + eps)   (L2: sum for mean).
//
// Bound by HBM: x read and y written once (131072 tokens of 16 + 4 heads of 64, bf16: 141 us,
// 671 MB at 4.8 TB/s; gradients of 32768 tokens of 16 + 16 heads 113 us, 537 MB at
// 4.8 TB/s).  A group of lanes holds one token; a lane holds four "slots" of two coordinates
// (a rotated pair, or two coordinates past the rotation) for every head in turn, so an
// angle's sine and cosine are formed once per token and not per head, and the sum of squares
// crosses only the group's lanes.  Angles: the turns pos freq / 2 pi are taken in fp64 and
// their fraction rounded to fp32 once: off by 2^-52 of the angle, which is more than fp32's
// rounding of a turn from positions of 2^28 on (fp32 angles are off by 0.06 rad at 10^6).
#pragma once

#include <type_traits>

#include "kata_rows.hpp"

namespace kata {

constexpr int kNormSlots = 4;  // slots of a lane

// The coordinates of slot u: rotated pair u < r/2, then the d - r others two by two.
struct NormSlots {
  int d, r, pairs;
  __device__ __forceinline__ void at(int u, int& e0, int& e1) const {
    const int rh = r >> 1;
    if (u < rh) {
      e0 = pairs ? 2 * u : u;
      e1 = pairs ? 2 * u + 1 : u + rh;
    } else {
      const int i = u - rh, mh = (d - r + 1) >> 1;
      e0 = r + i;
      e1 = r + mh + i;
      if (i >= mh) e0 = d;
      if (i >= mh || e1 > d) e1 = d;  // d: no such coordinate
    }
  }
};

// A lane's eight coordinates, (a, b) of each slot.  VEC: its four slots are four
// consecutive coordinates twice (or, as pairs, eight), aligned.
template <bool VEC, typename E>
__device__ __forceinline__ void norm_load(const E* p, const int (&e0)[4], const int (&e1)[4],
                                          int d, bool paired, float (&a)[4], float (&b)[4]) {
  if constexpr (VEC) {
    float u[4], v[4];
    load_vec<4>(p + e0[0], u);
    load_vec<4>(p + (paired ? e0[0] + 4 : e1[0]), v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = paired ? (i < 2 ? u[2 * i] : v[2 * i - 4]) : u[i];
      b[i] = paired ? (i < 2 ? u[2 * i + 1] : v[2 * i - 3]) : v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = e0[i] < d ? to_f32(p[e0[i]]) : 0.f;
      b[i] = e1[i] < d ? to_f32(p[e1[i]]) : 0.f;
    }
  }
}

template <bool VEC, typename E>
__device__ __forceinline__ void norm_store(E* p, const int (&e0)[4], const int (&e1)[4], int d,
                                           bool paired, const float (&a)[4], const float (&b)[4]) {
  if constexpr (VEC) {
    float u[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = paired ? ((i & 1) ? b[i >> 1] : a[i >> 1]) : a[i];
      v[i] = paired ? ((i & 1) ? b[2 + (i >> 1)] : a[2 + (i >> 1)]) : b[i];
    }
    store_vec<4>(p + e0[0], u);
    store_vec<4>(p + (paired ? e0[0] + 4 : e1[0]), v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e0[i] < d) store_f32(p + e0[i], a[i]);
      if (e1[i] < d) store_f32(p + e1[i], b[i]);
    }
  }
}

// cos and sin of this lane's rotated slots at a position; (1, 0) past the rotation.
__device__ __forceinline__ void norm_angles(const double* freq, int rh, int u0, int pos,
                                            float (&co)[4], float (&si)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    co[i] = 1.f, si[i] = 0.f;
    if (u0 + i < rh) {
      const double turns = pos * (freq[u0 + i] * 0.15915494309189533577);  // 1 / 2 pi
      sincospif(2.f * static_cast<float>(turns - rint(turns)), &si[i], &co[i]);
    }
  }
}

// A lane's coordinates of a head's row as they stand in memory; VEC as in norm_load.
template <bool VEC, typename E>
struct NormRow {
  RawVec<E, 4> u, v;
  __device__ __forceinline__ void load(const E* p, const int (&e0)[4], const int (&e1)[4], int d,
                                       bool paired) {
    if constexpr (VEC) {
      u = load_raw<E, 4>(p + e0[0]);
      v = load_raw<E, 4>(p + (paired ? e0[0] + 4 : e1[0]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u.e[i] = e0[i] < d ? p[e0[i]] : E{};
        v.e[i] = e1[i] < d ? p[e1[i]] : E{};
      }
    }
  }
  __device__ __forceinline__ void get(bool paired, float (&a)[4], float (&b)[4]) const {
    float x[4], y[4];
    raw_f32<E, 4>(u, x);
    raw_f32<E, 4>(v, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = VEC && paired ? (i < 2 ? x[2 * i] : y[2 * i - 4]) : x[i];
      b[i] = VEC && paired ? (i < 2 ? x[2 * i + 1] : y[2 * i - 3]) : y[i];
    }
  }
};

template <int LANES, bool VEC, typename E>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(const E* __restrict__ q,
                                                          const E* __restrict__ k,
                                                          const float* __restrict__ wq,
                                                          const float* __restrict__ wk,
                                                          const int* __restrict__ pos,
                                                          const double* __restrict__ freq,
                                                          E* __restrict__ yq, E* __restrict__ yk,
                                                          NormArgs n) {
  const int l = threadIdx.x & (LANES - 1);
  const long long token =
      static_cast<long long>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const long long tokens = static_cast<long long>(n.B) * n.T;
  if (token >= tokens) return;  // whole groups leave: sums cross a group's lanes only
  const int b = static_cast<int>(token / n.T), t = static_cast<int>(token - 1LL * b * n.T);
  const int u0 = l * kNormSlots, rh = n.r >> 1, U = (n.d + 1) >> 1;
  const bool live = u0 < U;
  const bool paired = n.pairs && u0 < rh;
  int e0[4], e1[4];
  const NormSlots slots{n.d, n.r, n.pairs};
#pragma unroll
  for (int i = 0; i < 4; ++i) slots.at(u0 + i, e0[i], e1[i]);
  const float scale = n.norm == kNormRms ? 1.f / static_cast<float>(n.d) : 1.f;
  const int h0 = blockIdx.y * n.split, h1 = min(h0 + n.split, n.side[0].H + n.side[1].H);
  float co[4], si[4];
  bool angles = false;
#pragma unroll
  for (int key = 0; key < 2; ++key) {
    const NormSide& s = n.side[key];
    const int from = max(h0 - (key ? n.side[0].H : 0), 0), to = min(h1 - (key ? n.side[0].H : 0), s.H);
    if (from >= to) continue;
    const E* x = (key ? k : q) + b * s.xb + t * s.xt;
    E* y = (key ? yk : yq) + (static_cast<long long>(b) * s.H * n.T + t) * n.d;
    const float* w = key ? wk : wq;
    // four heads at a time, the next four on their way (past the last: it again)
    NormRow<VEC, E> next[4];
    const auto fetch = [&](int h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) next[i].load(x + min(h + i, to - 1) * s.xh, e0, e1, n.d, paired);
    };
    if (live) fetch(from);
    if (!angles) norm_angles(freq, rh, u0, pos ? pos[token] : t, co, si);
    angles = true;
    float wa[4] = {1.f, 1.f, 1.f, 1.f}, wc[4] = {1.f, 1.f, 1.f, 1.f};
    if (w && live) norm_load<false>(w, e0, e1, n.d, false, wa, wc);
    for (int h = from; h < to; h += 4) {
      NormRow<VEC, E> now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) now[i] = next[i];
      if (live && h + 4 < to) fetch(h + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (h + j >= to) break;  // the same for all lanes
        float a[4] = {}, c[4] = {};
        if (live) now[j].get(paired, a, c);
        if (n.norm != kNormNone) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ss = fmaf(a[i], a[i], fmaf(c[i], c[i], ss));
          const float inv = __builtin_amdgcn_rsqf(fmaf(sum_group<LANES>(ss), scale, n.eps));
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] *= inv, c[i] *= inv;
        }
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] *= wa[i], c[i] *= wc[i];
          const float ta = fmaf(a[i], co[i], -c[i] * si[i]);
          c[i] = fmaf(a[i], si[i], c[i] * co[i]);
          a[i] = ta;
        }
        norm_store<VEC>(y + static_cast<long long>(h + j) * n.T * n.d, e0, e1, n.d, paired, a, c);
      }
    }
  }
}

// Gradients; dx has x's strides' layout of its own (NormArgs ds), dy is
// head-major fp32 or E.  A workgroup walks tokens, and of them the heads of its row of the
// grid; the sums of dw stay in registers until the end, then are joined over the
// workgroup's token groups in LDS and written as one partial sum per workgroup: wq's d,
// then wk's.
template <int LANES, bool VEC, typename E, typename Y>
__global__ __launch_bounds__(256) void qk_norm_bwd_kernel(
    const E* __restrict__ q, const E* __restrict__ k, const float* __restrict__ wq,
    const float* __restrict__ wk, const int* __restrict__ pos, const double* __restrict__ freq,
    const Y* __restrict__ dyq, const Y* __restrict__ dyk, E* __restrict__ dxq,
    E* __restrict__ dxk, float* __restrict__ part, NormArgs n, NormSide dq, NormSide dk) {
  __shared__ float red[256][17];  // [thread][2 sides x 8], padded
  const int l = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
  const int groups = 256 / LANES;
  const long long tokens = static_cast<long long>(n.B) * n.T;
  const int u0 = l * kNormSlots, rh = n.r >> 1, U = (n.d + 1) >> 1;
  const bool live = u0 < U;
  const bool paired = n.pairs && u0 < rh;
  int e0[4], e1[4];
  const NormSlots slots{n.d, n.r, n.pairs};
#pragma unroll
  for (int i = 0; i < 4; ++i) slots.at(u0 + i, e0[i], e1[i]);
  const float scale = n.norm == kNormRms ? 1.f / static_cast<float>(n.d) : 1.f;
  const int h0 = blockIdx.y * n.split, h1 = min(h0 + n.split, n.side[0].H + n.side[1].H);
  float dwa[2][4] = {}, dwc[2][4] = {};
  for (long long token = static_cast<long long>(blockIdx.x) * groups + group; token < tokens;
       token += static_cast<long long>(gridDim.x) * groups) {
    const int b = static_cast<int>(token / n.T), t = static_cast<int>(token - 1LL * b * n.T);
    float co[4], si[4];
    norm_angles(freq, rh, u0, pos ? pos[token] : t, co, si);
#pragma unroll
    for (int key = 0; key < 2; ++key) {
      const NormSide& s = n.side[key];
      const NormSide& ds = key ? dk : dq;
      const int from = max(h0 - (key ? n.side[0].H : 0), 0), to = min(h1 - (key ? n.side[0].H : 0), s.H);
      if (from >= to) continue;
      const float* w = key ? wk : wq;
      float wa[4], wc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) wa[i] = wc[i] = 1.f;
      if (w && live) norm_load<false>(w, e0, e1, n.d, false, wa, wc);
      const E* x0 = (key ? k : q) + b * s.xb + t * s.xt;
      E* dx0 = (key ? dxk : dxq) + b * ds.xb + t * ds.xt;
      const Y* dy0 = (key ? dyk : dyq) + (static_cast<long long>(b) * s.H * n.T + t) * n.d;
      for (int h = from; h < to; ++h) {
        float a[4] = {}, c[4] = {}, ga[4] = {}, gc[4] = {};
        if (live) {
          norm_load<VEC>(x0 + h * s.xh, e0, e1, n.d, paired, a, c);
          norm_load<VEC>(dy0 + static_cast<long long>(h) * n.T * n.d, e0, e1, n.d, paired, ga, gc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // R^T
          const float ta = fmaf(ga[i], co[i], gc[i] * si[i]);
          gc[i] = fmaf(gc[i], co[i], -ga[i] * si[i]);
          ga[i] = ta;
        }
        float inv = 1.f;
        if (n.norm != kNormNone) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ss = fmaf(a[i], a[i], fmaf(c[i], c[i], ss));
          inv = __builtin_amdgcn_rsqf(fmaf(sum_group<LANES>(ss), scale, n.eps));
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] *= inv, c[i] *= inv;  // hat
          dwa[key][i] = fmaf(ga[i], a[i], dwa[key][i]);
          dwc[key][i] = fmaf(gc[i], c[i], dwc[key][i]);
          ga[i] *= wa[i], gc[i] *= wc[i];
          dot = fmaf(ga[i], a[i], fmaf(gc[i], c[i], dot));
        }
        if (n.norm != kNormNone) {
          dot = sum_group<LANES>(dot) * scale;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ga[i] = inv * fmaf(-a[i], dot, ga[i]);
            gc[i] = inv * fmaf(-c[i], dot, gc[i]);
          }
        }
        if (live) norm_store<VEC>(dx0 + h * ds.xh, e0, e1, n.d, paired, ga, gc);
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int key = 0; key < 2; ++key)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      red[threadIdx.x][key * 8 + i] = dwa[key][i];
      red[threadIdx.x][key * 8 + 4 + i] = dwc[key][i];
    }
  __syncthreads();
  // thread (lane l', value v) adds its column over the groups, in order
  for (int i = threadIdx.x; i < LANES * 16; i += 256) {
    const int ll = i >> 4, v = i & 15;
    float acc = 0.f;
    for (int g = 0; g < groups; ++g) acc += red[g * LANES + ll][v];
    int c0, c1;
    slots.at(ll * kNormSlots + (v & 3), c0, c1);
    const int e = (v & 4) ? c1 : c0;
    if (ll * kNormSlots + (v & 3) < U && e < n.d)
      part[(static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 2 * n.d + (v >> 3) * n.d + e] = acc;
  }
}

// ---- launches ---------------------------------------------------------------

template <typename F>
void norm_with_lanes(int d, F f) {
  switch (norm_lanes(d)) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    case 16: return f(std::integral_constant<int, 16>{});
    default: return f(std::integral_constant<int, 32>{});
  }
}

// Four consecutive coordinates at a time: the rotated halves (or pairs) and the
// other coordinates' halves are whole pieces, and every row starts on one.  One by one, the
// call of 131072 tokens takes 456 us for 143.
inline bool norm_vec_ok(int d, int r, std::initializer_list<long long> strides) {
  if ((r / 2) % 4 || (d - r) % 8) return false;
  for (long long s : strides)
    if (s % 4) return false;
  return true;
}

// Heads of a workgroup: all heads of a token in one lane group share its angles; with few
// tokens the heads are split until about two workgroups stand on every CU.  16 + 16 heads of
// 64, split and not: 256 tokens forward 4.0 and 12 us, 2000 6.1 and 13 us;
// backward 100 tokens 6.8 and 22 us, 2000 14 and 29 us.
inline int norm_split(long long blocks, int H) {
  const long long splits = (512 + blocks - 1) / blocks;
  const int n = static_cast<int>(splits < H ? splits : H);
  return (H + n - 1) / n;
}

template <typename E>
hipError_t qk_norm_fwd_e(const E* q, const E* k, const float* wq, const float* wk, const int* pos,
                         const double* freq, E* yq, E* yk, NormArgs n, hipStream_t st) {
  constexpr int bytes = 4 * static_cast<int>(sizeof(E));
  const long long tokens = static_cast<long long>(n.B) * n.T;
  const int per = 256 / norm_lanes(n.d), H = n.side[0].H + n.side[1].H;
  const long long blocks = (tokens + per - 1) / per;
  n.split = norm_split(blocks, H);
  const dim3 grid(static_cast<unsigned>(blocks), (H + n.split - 1) / n.split);
  const NormSide &a = n.side[0], &c = n.side[1];
  const bool vec = norm_vec_ok(n.d, n.r, {a.xb, a.xt, a.xh, c.xb, c.xt, c.xh}) &&
                   ptr_aligned({q, k, yq, yk}, bytes);
  norm_with_lanes(n.d, [&](auto lanes) {
    constexpr int kLanes = decltype(lanes)::value;
    if (vec)
      qk_norm_fwd_kernel<kLanes, true, E><<<grid, 256, 0, st>>>(q, k, wq, wk, pos, freq, yq, yk, n);
    else
      qk_norm_fwd_kernel<kLanes, false, E><<<grid, 256, 0, st>>>(q, k, wq, wk, pos, freq, yq, yk, n);
  });
  return hipGetLastError();
}

// Workgroups of the backward along the tokens, two per CU at the most and with equal walks;
// each (of each part of the heads) writes one partial sum of dw.  8 x 4096 tokens, 16 + 16
// heads of 64: 89 us (512), 99 (768: unequal walks), 141 (256), 90 (1024).
inline int norm_bwd_blocks(int B, int T, int d) {
  const long long per = 256 / norm_lanes(d);
  const long long n = (static_cast<long long>(B) * T + per - 1) / per, walk = (n + 511) / 512;
  return static_cast<int>((n + walk - 1) / walk);
}

size_t norm_bwd_workspace_bytes(int B, int T, int H, int d) {
  const int blocks = norm_bwd_blocks(B, T, d), split = norm_split(blocks, H);
  const size_t parts = static_cast<size_t>(blocks) * ((H + split - 1) / split);
  return (parts * 2 * d * sizeof(float) + 255) & ~static_cast<size_t>(255);
}

template <typename E, typename Y>
hipError_t qk_norm_bwd_e(const E* q, const E* k, const float* wq, const float* wk, const int* pos,
                         const double* freq, const Y* dyq, const Y* dyk, E* dxq, E* dxk,
                         float* dwq, float* dwk, void* ws, NormArgs n, const NormSide& dq,
                         const NormSide& dk, hipStream_t st) {
  constexpr int bytes = 4 * static_cast<int>(sizeof(E));
  constexpr int ybytes = 4 * static_cast<int>(sizeof(Y));
  const int blocks = norm_bwd_blocks(n.B, n.T, n.d), H = n.side[0].H + n.side[1].H;
  n.split = norm_split(blocks, H);
  const dim3 grid(blocks, (H + n.split - 1) / n.split);
  float* part = dwq || dwk ? static_cast<float*>(ws) : nullptr;
  const NormSide &a = n.side[0], &c = n.side[1];
  const bool vec = norm_vec_ok(n.d, n.r, {a.xb, a.xt, a.xh, c.xb, c.xt, c.xh, dq.xb, dq.xt, dq.xh,
                                          dk.xb, dk.xt, dk.xh}) &&
                   ptr_aligned({q, k, dxq, dxk}, bytes) && ptr_aligned({dyq, dyk}, ybytes);
  norm_with_lanes(n.d, [&](auto lanes) {
    constexpr int kLanes = decltype(lanes)::value;
    if (vec)
      qk_norm_bwd_kernel<kLanes, true, E, Y><<<grid, 256, 0, st>>>(
          q, k, wq, wk, pos, freq, dyq, dyk, dxq, dxk, part, n, dq, dk);
    else
      qk_norm_bwd_kernel<kLanes, false, E, Y><<<grid, 256, 0, st>>>(
          q, k, wq, wk, pos, freq, dyq, dyk, dxq, dxk, part, n, dq, dk);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  return launch_sum_partials(part, grid.x * grid.y, 2 * n.d, {{dwq, dwk, nullptr}, {n.d, n.d, 0}}, st);
}

hipError_t launch_qk_norm_fwd(const void* q, const void* k, const float* wq, const float* wk,
                              const int* pos, const double* freq, void* yq, void* yk,
                              const NormArgs& n, bool bf16, hipStream_t st) {
  if (bf16)
    return qk_norm_fwd_e<bf16_t>(static_cast<const bf16_t*>(q), static_cast<const bf16_t*>(k), wq,
                                 wk, pos, freq, static_cast<bf16_t*>(yq),
                                 static_cast<bf16_t*>(yk), n, st);
  return qk_norm_fwd_e<float>(static_cast<const float*>(q), static_cast<const float*>(k), wq, wk,
                              pos, freq, static_cast<float*>(yq), static_cast<float*>(yk), n, st);
}

template <typename E, typename Y>
hipError_t qk_norm_bwd_p(const void* q, const void* k, const float* wq, const float* wk,
                         const int* pos, const double* freq, const void* dyq, const void* dyk,
                         void* dxq, void* dxk, float* dwq, float* dwk, void* ws, const NormArgs& n,
                         const NormSide& dq, const NormSide& dk, hipStream_t st) {
  return qk_norm_bwd_e<E, Y>(static_cast<const E*>(q), static_cast<const E*>(k), wq, wk, pos, freq,
                             static_cast<const Y*>(dyq), static_cast<const Y*>(dyk),
                             static_cast<E*>(dxq), static_cast<E*>(dxk), dwq, dwk, ws, n, dq, dk,
                             st);
}

hipError_t launch_qk_norm_bwd(const void* q, const void* k, const float* wq, const float* wk,
                              const int* pos, const double* freq, const void* dyq, const void* dyk,
                              void* dxq, void* dxk, float* dwq, float* dwk, void* ws,
                              const NormArgs& n, const NormSide& dq, const NormSide& dk, bool bf16,
                              bool dy_bf16, hipStream_t st) {
  if (!bf16)
    return qk_norm_bwd_p<float, float>(q, k, wq, wk, pos, freq, dyq, dyk, dxq, dxk, dwq, dwk, ws,
                                       n, dq, dk, st);
  if (dy_bf16)
    return qk_norm_bwd_p<bf16_t, bf16_t>(q, k, wq, wk, pos, freq, dyq, dyk, dxq, dxk, dwq, dwk,
                                         ws, n, dq, dk, st);
  return qk_norm_bwd_p<bf16_t, float>(q, k, wq, wk, pos, freq, dyq, dyk, dxq, dxk, dwq, dwk, ws, n,
                                      dq, dk, st);
}

}  // namespace kata
