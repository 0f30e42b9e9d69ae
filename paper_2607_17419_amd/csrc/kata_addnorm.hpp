// kata_addnorm.hpp -- root-mean-square norm of a row with the residual's addition:
//
//   s = x + res (rounded once to the activations' type),  inv = 1 / sqrt(mean(s^2) + eps),
//   y = s inv w,
//
// y in the activations' type, as e4m3 codes with a scale for each 128 columns, or both.
// Backward, from s: hat = s inv, g = w dy,
//   dx = dsum + inv (g - hat mean(g hat)),   dw = sum over rows of dy hat.
//
// HBM bound: a row stays in the registers of one to sixteen waves from its load to its
// store, eight neighbouring columns a lane, so every tensor is read or written once (but in the
// gradients of rows of more than 16384 columns, which spill).  32768 rows of 1024, bf16: forward 46 us
// (268 MB, 5.8 TB/s), to codes 44 us (236 MB, 5.4 TB/s), gradients 48 us (268 MB, 5.6 TB/s; 51 us
// where all of dy is 0) and 5 us for their sums; 256 rows to 8 bits 4 us, the launch's latency.
// 2048 rows of 16384: 55 and 58 us, 1024 of 32768: 57 and 270.
#pragma once

#include "kata_f8.hpp"

namespace kata {

template <int CTRL>
__device__ __forceinline__ double dpp_move64(double x) {
  struct Two { float lo, hi; };
  const Two t = __builtin_bit_cast(Two, x);
  return __builtin_bit_cast(double, Two{dpp_move<CTRL>(t.lo), dpp_move<CTRL>(t.hi)});
}
__device__ __forceinline__ float wave_sum(float x) { return sum_group<64>(x); }
__device__ __forceinline__ double wave_sum(double x) {
  x += dpp_move64<0xB1>(x);
  x += dpp_move64<0x4E>(x);
  x += dpp_move64<0x141>(x);
  x += dpp_move64<0x140>(x);
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
// Sums over the WAVES waves of a row (a workgroup, or one wave), the same in every lane; `at`
// holds them for each wave and is free again after the next barrier.
template <int WAVES, int N, typename F>
__device__ __forceinline__ void row_sum(F (&v)[N], F (*at)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) at[threadIdx.x >> 6][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = F(0);
#pragma unroll 4  // (all sixteen at once in fp64 take the registers of the row)
      for (int w = 0; w < WAVES; ++w) v[k] += at[w][k];
    }
  }
}
// 1 / sqrt(x) to a few 2^-53: the hardware's, and one step of Newton's.
__device__ __forceinline__ double row_rsqrt(double x) {
  const double r = __builtin_amdgcn_rsq(x);
  return r * fma(-0.5 * x * r, r, 1.5);
}

// WAVES waves a row; ITER pieces of 512 * WAVES columns.  Squares are summed in fp64: a tenth of
// the time that the row's bytes take, and what decides between codes is then exact.
template <typename E, int WAVES, int ITER, bool VEC>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void add_norm_kernel(
    const E* x, const E* res, const float* __restrict__ w, E* sum, E* __restrict__ y,
    uint8_t* __restrict__ q, float* __restrict__ scale, AddNormArgs s) {
  __shared__ double at[WAVES][1];
  const long long m = WAVES == 1 ? blockIdx.x * 4LL + (threadIdx.x >> 6) : blockIdx.x;
  if (m >= s.M) return;  // (with more than one wave never)
  const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  float v[ITER][8];
#pragma unroll
  for (int k = 0; k < ITER; ++k) load8<VEC>(x + m * s.x_row, (k * 64 * WAVES + lane) * 8, s.D, v[k]);
  if (res) {
    float r[ITER][8];
#pragma unroll
    for (int k = 0; k < ITER; ++k)
      load8<VEC>(res + m * s.res_row, (k * 64 * WAVES + lane) * 8, s.D, r[k]);
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[k][i] += r[k][i];
        if constexpr (sizeof(E) == 2) v[k][i] = static_cast<float>(static_cast<__bf16>(v[k][i]));
      }
      if (sum) store8<VEC>(sum + m * s.sum_row, (k * 64 * WAVES + lane) * 8, s.D, v[k]);
    }
  }
  double total[1] = {0.0};
#pragma unroll
  for (int k = 0; k < ITER; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) total[0] = fma(static_cast<double>(v[k][i]), static_cast<double>(v[k][i]), total[0]);
  row_sum<WAVES>(total, at);
  const double inv64 = row_rsqrt(total[0] / s.D + s.eps);
  const float inv = static_cast<float>(inv64);
  const int kb = (s.D + kF8Block - 1) / kF8Block;
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int c = (k * 64 * WAVES + lane) * 8;
    float wv[8], out[8];
    if (w) {
      load8<VEC>(w, c, s.D, wv);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) wv[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = v[k][i] * inv * wv[i];
    if (y) store8<VEC>(y + m * s.y_row, c, s.D, out);
    if (q) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t = fmaxf(t, fabsf(out[i]));
      const float sc = f8_scale(max_row16(t)), by = 1.f / sc;
      if ((lane & 15) == 0 && c < s.D) scale[m * kb + c / kF8Block] = sc;
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] *= by;
      // out and the block's largest value are off by up to 2.5 steps of fp32 each, their quotient by 6.
      // The row's factor stands in both and is left out: s w 448 is exact in fp64 (51 bits), so that its
      // quotient by the block's largest s w is a middle only where it is one.
      if (__any(f8_near_middle<8>(out))) {
        double exact[8], top = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          exact[i] = static_cast<double>(v[k][i]) * wv[i];
          top = fmax(top, fabs(exact[i]));
        }
        top = fmax(top, dpp_move64<0xB1>(top));
        top = fmax(top, dpp_move64<0x4E>(top));
        top = fmax(top, dpp_move64<0x141>(top));
        top = fmax(top, dpp_move64<0x140>(top));
        const bool least = !(f8_most(top * inv64) > f8_most(0.0));  // (a NaN row too)
        const double times = least ? inv64 * 0x1p126 : 448.0;
        if (least) top = 1.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = f8_odd(exact[i] * times / top);
      }
      store8_codes<VEC>(q + m * s.q_row, c, s.D, f8_pack8(out));
    }
  }
}

// A workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (in fours with one wave a
// row) and keeps its sums of dw in registers; part: [gridDim.x][D].  Squares are summed in fp32,
// and once more, scaled, in rows whose squares may have left its range (in fp64 at once:
// training step 101 -> 129 us, a wave less on each SIMD).
template <typename E, typename G, int WAVES, int ITER, bool VEC>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES,
                             ITER == 1 ? (WAVES == 1 ? 6 : 5) : WAVES == 16 || ITER == 2 ? 4 : 2) void add_norm_bwd_kernel(
    const E* __restrict__ sum, const float* __restrict__ w, const G* __restrict__ dy,
    const E* __restrict__ dsum, E* __restrict__ dx, float* __restrict__ part, AddNormArgs s) {
  __shared__ float at[2][WAVES][2];
  __shared__ double far[2][WAVES][2];
  __shared__ float red[WAVES == 1 ? 3 : 1][WAVES == 1 ? 64 * ITER * 8 : 1];
  const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  float dw[ITER][8] = {}, wv[ITER][8];
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    if (w) {
      load8<VEC>(w, (k * 64 * WAVES + lane) * 8, s.D, wv[k]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) wv[k][i] = 1.f;
    }
  }
  const long long step = WAVES == 1 ? gridDim.x * 4LL : gridDim.x;
  int turn = 0;
  for (long long m = WAVES == 1 ? blockIdx.x * 4LL + (threadIdx.x >> 6) : blockIdx.x; m < s.M;
       m += step, turn ^= 1) {
    float v[ITER][8], g[ITER][8], d[ITER][8], sums[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      const int c = (k * 64 * WAVES + lane) * 8;
      load8<VEC>(sum + m * s.x_row, c, s.D, v[k]);
      load8<VEC>(dy + m * s.res_row, c, s.D, g[k]);
      if (dsum) {
        load8<VEC>(dsum + m * s.sum_row, c, s.D, d[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[k][i] = 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < ITER; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sums[0] = fmaf(v[k][i], v[k][i], sums[0]);
        sums[1] = fmaf(v[k][i], g[k][i] * wv[k][i], sums[1]);
      }
    row_sum<WAVES>(sums, at[turn]);
    float inv = 1.f / sqrtf(sums[0] / s.D + s.eps);
    float dot = sums[1] * (inv / s.D);  // mean(g hat)
    // the same in the whole row.  (A sum above 1e-30 has lost less than 2^-35 of itself to
    // subnormal parts; one of 0 may have been smaller, or a row without gradients.)
    const float size = fabsf(sums[1]);
    if (!(sums[0] > 1e-20f && sums[0] < 1e38f && size > 1e-30f && size < 1e38f)) {
      double total[2] = {0.0, 0.0};
#pragma unroll
      for (int k = 0; k < ITER; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double one = v[k][i];
          total[0] = fma(one, one, total[0]);
          total[1] = fma(one, static_cast<double>(g[k][i] * wv[k][i]), total[1]);
        }
      row_sum<WAVES>(total, far[turn]);
      const double inv64 = row_rsqrt(total[0] / s.D + s.eps);
      inv = static_cast<float>(inv64);
      dot = static_cast<float>(total[1] * inv64 / s.D);
    }
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float hat = v[k][i] * inv;
        dw[k][i] = fmaf(g[k][i], hat, dw[k][i]);
        v[k][i] = fmaf(inv, g[k][i] * wv[k][i] - hat * dot, d[k][i]);
      }
      store8<VEC>(dx + m * s.y_row, (k * 64 * WAVES + lane) * 8, s.D, v[k]);
    }
  }
  if (!part) return;
  if constexpr (WAVES == 1) {
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < ITER; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (wave) red[wave - 1][(k * 8 + i) * 64 + lane] = dw[k][i];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 0; k < ITER; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = (k * 8 + i) * 64 + lane;
        dw[k][i] = (dw[k][i] + red[0][e]) + (red[1][e] + red[2][e]);
      }
  }
  float* row = part + static_cast<size_t>(blockIdx.x) * s.D;
#pragma unroll
  for (int k = 0; k < ITER; ++k) store8<VEC>(row, (k * 64 * WAVES + lane) * 8, s.D, dw[k]);
}

// ---- launches ---------------------------------------------------------------

// A row to one wave where there are rows for two waves on each of the 1024 SIMDs, so that
// sums need no barrier; fewer or wider rows to four waves, the widest to sixteen (whose gradients
// spill from 16385 columns on: 173 of the 256 values that a lane holds).
inline int add_norm_waves(int M, int D) { return D > 8192 ? 16 : D > 2048 || M < 2048 ? 4 : 1; }

// Pieces of 512 * waves columns: CALL(waves, pieces).
#define KATA_ADD_NORM_SHAPE(CALL)                              \
  const int per = 512 * add_norm_waves(s.M, s.D);              \
  const int pieces = (s.D + per - 1) / per;                    \
  if (per == 512) {                                            \
    if (pieces == 1) { CALL(1, 1); }                           \
    else if (pieces == 2) { CALL(1, 2); }                      \
    else { CALL(1, 4); }                                       \
  } else if (per == 2048) {                                    \
    if (pieces == 1) { CALL(4, 1); }                           \
    else if (pieces == 2) { CALL(4, 2); }                      \
    else { CALL(4, 4); }                                       \
  } else {                                                     \
    if (pieces == 2) { CALL(16, 2); }                          \
    else { CALL(16, 4); }                                      \
  }

// Whether rows are whole aligned pieces of eight elements.
inline bool add_norm_vec(const AddNormArgs& s, std::initializer_list<const void*> p) {
  return s.D % 8 == 0 && s.x_row % 8 == 0 && s.res_row % 8 == 0 && s.sum_row % 8 == 0 &&
         s.y_row % 8 == 0 && s.q_row % 8 == 0 && ptr_aligned(p, 16);
}

template <typename E>
hipError_t add_norm_e(const void* x, const void* res, const float* w, void* sum, void* y, void* q,
                      float* scale, const AddNormArgs& s, hipStream_t st) {
  const bool vec = add_norm_vec(s, {x, res, w, sum, y}) && ptr_aligned({q}, 8);
#define KATA_CALL(WV, IT)                                                                          \
  const unsigned blocks = static_cast<unsigned>(WV == 1 ? (s.M + 3LL) / 4 : s.M);                  \
  const int threads = WV == 1 ? 256 : 64 * WV;                                                     \
  if (vec)                                                                                         \
    add_norm_kernel<E, WV, IT, true><<<blocks, threads, 0, st>>>(                                  \
        static_cast<const E*>(x), static_cast<const E*>(res), w, static_cast<E*>(sum),             \
        static_cast<E*>(y), static_cast<uint8_t*>(q), scale, s);                                   \
  else                                                                                             \
    add_norm_kernel<E, WV, IT, false><<<blocks, threads, 0, st>>>(                                 \
        static_cast<const E*>(x), static_cast<const E*>(res), w, static_cast<E*>(sum),             \
        static_cast<E*>(y), static_cast<uint8_t*>(q), scale, s);
  KATA_ADD_NORM_SHAPE(KATA_CALL)
#undef KATA_CALL
  return hipGetLastError();
}

// Workgroups of the gradients: four for each CU, and no more than leave eight rows to each.
inline int add_norm_bwd_slices(int M, int D) {
  const int rows = add_norm_waves(M, D) == 1 ? 32 : 8;
  const long long n = (static_cast<long long>(M) + rows - 1) / rows;
  return static_cast<int>(n < 1024 ? n : 1024);
}

size_t add_norm_bwd_workspace_bytes(int M, int D) {
  return (static_cast<size_t>(add_norm_bwd_slices(M, D)) * D * sizeof(float) + 255) &
         ~static_cast<size_t>(255);
}

template <typename E, typename G>
hipError_t add_norm_bwd_e(const void* sum, const float* w, const void* dy, const void* dsum, void* dx,
                          float* dw, void* ws, const AddNormArgs& s, hipStream_t st) {
  const bool vec = add_norm_vec(s, {sum, w, dy, dsum, dx});
  const int slices = add_norm_bwd_slices(s.M, s.D);
  float* part = dw ? static_cast<float*>(ws) : nullptr;
#define KATA_CALL(WV, IT)                                                                        \
  const int threads = WV == 1 ? 256 : 64 * WV;                                                   \
  if (vec)                                                                                       \
    add_norm_bwd_kernel<E, G, WV, IT, true><<<slices, threads, 0, st>>>(                         \
        static_cast<const E*>(sum), w, static_cast<const G*>(dy), static_cast<const E*>(dsum),   \
        static_cast<E*>(dx), part, s);                                                           \
  else                                                                                           \
    add_norm_bwd_kernel<E, G, WV, IT, false><<<slices, threads, 0, st>>>(                        \
        static_cast<const E*>(sum), w, static_cast<const G*>(dy), static_cast<const E*>(dsum),   \
        static_cast<E*>(dx), part, s);
  KATA_ADD_NORM_SHAPE(KATA_CALL)
#undef KATA_CALL
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dw) return e;
  return launch_sum_partials(part, slices, s.D, {{dw, nullptr, nullptr}, {s.D, 0, 0}}, st);
}
#undef KATA_ADD_NORM_SHAPE

hipError_t launch_add_norm(const void* x, const void* res, const float* w, void* sum, void* y,
                           void* q, float* scale, const AddNormArgs& s, bool bf16, hipStream_t st) {
  return bf16 ? add_norm_e<bf16_t>(x, res, w, sum, y, q, scale, s, st)
              : add_norm_e<float>(x, res, w, sum, y, q, scale, s, st);
}
hipError_t launch_add_norm_bwd(const void* sum, const float* w, const void* dy, const void* dsum,
                               void* dx, float* dw, void* ws, const AddNormArgs& s, bool bf16,
                               bool dy_bf16, hipStream_t st) {
  if (!bf16) return add_norm_bwd_e<float, float>(sum, w, dy, dsum, dx, dw, ws, s, st);
  return dy_bf16 ? add_norm_bwd_e<bf16_t, bf16_t>(sum, w, dy, dsum, dx, dw, ws, s, st)
                 : add_norm_bwd_e<bf16_t, float>(sum, w, dy, dsum, dx, dw, ws, s, st);
}

}  // namespace kata
