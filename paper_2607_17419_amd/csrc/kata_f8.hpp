// kata_f8.hpp -- codes of 8 bits (e4m3: sign, 4 bits of exponent, 3 of mantissa; largest
// 448, no infinity) with an fp32 scale for each block, and the quantiser:
//
//   scale = max(max |x| over the block / 448, 2^-126),   q = e4m3(x / scale),
//
// rounded to nearest, ties to even.  x / scale is at most 448 (1 + 2^-22), which rounds to
// 448, so nothing saturates.  The quotient is formed in fp32 as x (1 / scale), and where that
// comes so near to the middle between two codes that its own roundings could decide between
// them, for the eight values of each lane of the wave once more in fp64, as x 448 / max |x| (one
// value in 10^5: a few instructions each to look, and hardly ever more).  Quotients of bf16
// inputs of the quantiser often are such middles exactly (0.2% of them), so that waves would
// hardly ever get by without; they stay as fp32 gives them.  A NaN is left
// out of the maximum and becomes a NaN code; an infinity makes its block's scale infinite and its own code NaN.
//
// 32768 x 1024 of bf16 to rows and transposed: 34 us (134 MB, 4.0 TB/s; the read, the codes' arithmetic
// and the writes follow each other in all workgroups alike); with twice the waves on a CU the same.
//
// Blocks are 128 columns of one row (KATA_BLOCK_ROWS) or 128 x 128.  A workgroup holds a
// 128 x 128 tile of x in registers, 8 x 8 values a thread, so that the rows' codes and those
// of the transposed tile come from one read of x; transposed codes go through LDS to whole
// 128-byte rows.
#pragma once

#include "kata_block.hpp"
#include "kata_rows.hpp"

namespace kata {

constexpr float kF8Top = 448.f;

__device__ __forceinline__ float f8_scale(float top) { return fmaxf(top / kF8Top, 0x1p-126f); }

// Four values as codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return static_cast<uint32_t>(r);
}

// Largest magnitude over groups of 16 lanes, in every lane.
__device__ __forceinline__ float max_row16(float x) {
  x = fmaxf(x, dpp_move<0xB1>(x));
  x = fmaxf(x, dpp_move<0x4E>(x));
  x = fmaxf(x, dpp_move<0x141>(x));
  return fmaxf(x, dpp_move<0x140>(x));
}

// Eight neighbouring elements of a row of n, c the first; zeros past its end.
template <bool VEC, typename E>
__device__ __forceinline__ void load8(const E* row, int c, int n, float (&v)[8]) {
  if constexpr (VEC) {
    if (c < n) {
      load_vec<8>(row + c, v);
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n ? to_f32(row[c + i]) : 0.f;
  }
}
template <bool VEC, typename E>
__device__ __forceinline__ void store8(E* row, int c, int n, const float (&v)[8]) {
  if constexpr (VEC) {
    if (c < n) store_vec<8>(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) store_f32(row + c + i, v[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void store8_codes(uint8_t* row, int c, int n, uint2 q) {
  if constexpr (VEC) {
    if (c < n) *reinterpret_cast<uint2*>(row + c) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) row[c + i] = static_cast<uint8_t>((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
  }
}
// Whether one of eight quotients is within N fp32 steps of a middle between two codes, which have
// 20 bits less.  Below the normal range, 2^-6, codes are as far apart as just above it.
template <int N>
__device__ __forceinline__ bool f8_near_middle(const float (&v)[8]) {
  uint32_t least = ~0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float m = fabsf(v[i]), t = m < 0x1p-6f ? m + 0x1p-6f : m;
    least = min(least, (__float_as_uint(t) - (0x80000u - N)) & 0xFFFFFu);
  }
  return least <= 2 * N;
}
// fp64 to the fp32 that rounds to the same code: to odd where it is not exact.
__device__ __forceinline__ float f8_odd(double v) {
  const float f = static_cast<float>(v);
  const double d = fabs(v) - fabs(static_cast<double>(f));
  uint32_t b = __float_as_uint(f);
  if (d < 0.0) b = (b - 1u) | 1u;
  else if (d > 0.0) b |= 1u;
  return __uint_as_float(b);
}
// The largest magnitude of a block, or what it is at the least scale.
__device__ __forceinline__ double f8_most(double top) { return fmax(top, 448.0 * 0x1p-126); }
__device__ __forceinline__ uint2 f8_pack8(const float (&v)[8]) {
  return make_uint2(f8_pack4(v[0], v[1], v[2], v[3]), f8_pack4(v[4], v[5], v[6], v[7]));
}
// Codes of eight values of a block whose largest magnitude is `top`, inv = 1 / its scale.
template <bool EXACT>
__device__ __forceinline__ uint2 f8_codes8(const float (&x)[8], float inv, float top) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = x[i] * inv;
  if constexpr (EXACT) {
    if (__any(f8_near_middle<4>(v))) {
      // x 448 is exact, so that its quotient by the largest is a middle where x / scale is one
      // (by a rounded top / 448, an eighth of them would fall to either side)
      const double most = f8_most(top);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = f8_odd(x[i] * 448.0 / most);
    }
  }
  return f8_pack8(v);
}

// ROWS: rows of a block (1 or 128).  VEC: x in whole aligned pieces of eight elements;
// VQ, VT: codes of q and of qt in aligned pieces of 8 and 16.
template <typename E, int ROWS, bool VEC, bool VQ, bool VT>
__global__ __launch_bounds__(256) void f8_quant_kernel(const E* __restrict__ x,
                                                       uint8_t* __restrict__ q,
                                                       float* __restrict__ scale,
                                                       uint8_t* __restrict__ qt,
                                                       float* __restrict__ scale_t, F8QuantArgs s) {
  constexpr bool EXACT = sizeof(E) == 4;
  __shared__ float top[4][kF8Block];
  __shared__ uint2 turned[kF8Block][17];  // [column][eight rows], a piece of padding
  const int col = threadIdx.x & 15, group = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int tm = blockIdx.x / s.kt, tk = blockIdx.x - tm * s.kt;
  const int m0 = tm * kF8Block + group * 8, k0 = tk * kF8Block + col * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (m0 + i < s.M) {
      load8<VEC>(x + (m0 + i) * s.x_row, k0, s.K, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
  const int kb = (s.K + kF8Block - 1) / kF8Block, mb = (s.M + kF8Block - 1) / kF8Block;
  float block_inv = 0.f, block_top = 0.f;
  if constexpr (ROWS != 1) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) t = fmaxf(t, fabsf(v[i][j]));
    t = max_row16(t);
    t = fmaxf(t, __shfl_xor(t, 16));
    t = fmaxf(t, __shfl_xor(t, 32));
    if ((threadIdx.x & 63) == 0) top[0][wave] = t;
    __syncthreads();
    t = fmaxf(fmaxf(top[0][0], top[0][1]), fmaxf(top[0][2], top[0][3]));
    const float sc = f8_scale(t);
    block_inv = 1.f / sc, block_top = t;
    if (threadIdx.x == 0) {
      if (scale) scale[static_cast<size_t>(tm) * kb + tk] = sc;
      if (scale_t) scale_t[static_cast<size_t>(tk) * mb + tm] = sc;
    }
  }
  if (q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float inv = block_inv, t = block_top;
      if constexpr (ROWS == 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t = fmaxf(t, fabsf(v[i][j]));
        t = max_row16(t);
        const float sc = f8_scale(t);
        inv = 1.f / sc;
        if (col == 0 && m0 + i < s.M) scale[static_cast<size_t>(m0 + i) * kb + tk] = sc;
      }
      if (m0 + i < s.M) store8_codes<VQ>(q + (m0 + i) * s.q_row, k0, s.K, f8_codes8<EXACT>(v[i], inv, t));
    }
  }
  if (!qt) return;
  const auto column_top = [&](int c) {
    return ROWS == 1 ? fmaxf(fmaxf(top[0][c], top[1][c]), fmaxf(top[2][c], top[3][c])) : block_top;
  };
  float inv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) inv[j] = block_inv;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t = fmaxf(t, fabsf(v[i][j]));
      t = fmaxf(t, __shfl_xor(t, 16));
      t = fmaxf(t, __shfl_xor(t, 32));
      if ((threadIdx.x & 48) == 0) top[wave][col * 8 + j] = t;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col * 8 + j;
      const float sc = f8_scale(column_top(c));
      inv[j] = 1.f / sc;
      if (group == 0 && k0 + j < s.K) scale_t[static_cast<size_t>(k0 + j) * mb + tm] = sc;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float down[8] = {v[0][j], v[1][j], v[2][j], v[3][j], v[4][j], v[5][j], v[6][j], v[7][j]};
    turned[col * 8 + j][group] = f8_codes8<EXACT>(down, inv[j], column_top(col * 8 + j));
  }
  __syncthreads();
  // eight lanes write a transposed row's 128 bytes
  const int part = threadIdx.x & 7;
#pragma unroll
  for (int r = threadIdx.x >> 3; r < kF8Block; r += 32) {
    const int k = tk * kF8Block + r, m = tm * kF8Block + part * 16;
    if (k >= s.K) continue;
    uint8_t* row = qt + k * s.qt_row;
    const uint2 a = turned[r][2 * part], b = turned[r][2 * part + 1];
    if (VT && m + 16 <= s.M) {
      *reinterpret_cast<uint4*>(row + m) = make_uint4(a.x, a.y, b.x, b.y);
    } else {
      store8_codes<false>(row, m, s.M, a);
      store8_codes<false>(row, m + 8, s.M, b);
    }
  }
}

template <typename E, int ROWS>
hipError_t f8_quant_e(const E* x, uint8_t* q, float* scale, uint8_t* qt, float* scale_t,
                      const F8QuantArgs& s, hipStream_t st) {
  const long long tiles = ((s.M + 127LL) / 128) * s.kt;
  const bool vec = s.K % 8 == 0 && s.x_row % 8 == 0 && ptr_aligned({x}, 16);
  const bool vq = s.K % 8 == 0 && s.q_row % 8 == 0 && ptr_aligned({q}, 8);
  const bool vt = s.qt_row % 16 == 0 && ptr_aligned({qt}, 16);
  const dim3 grid(static_cast<unsigned>(tiles));
#define KATA_QUANT(A, B, C) \
  f8_quant_kernel<E, ROWS, A, B, C><<<grid, 256, 0, st>>>(x, q, scale, qt, scale_t, s)
  if (vec && vq && vt) KATA_QUANT(true, true, true);
  else if (vec) KATA_QUANT(true, false, false);
  else if (vt) KATA_QUANT(false, false, true);
  else KATA_QUANT(false, false, false);
#undef KATA_QUANT
  return hipGetLastError();
}

hipError_t launch_f8_quant(const void* x, void* q, float* scale, void* qt, float* scale_t, int rows,
                           F8QuantArgs s, bool bf16, hipStream_t st) {
  s.kt = (s.K + kF8Block - 1) / kF8Block;
  uint8_t *qb = static_cast<uint8_t*>(q), *tb = static_cast<uint8_t*>(qt);
  if (bf16) {
    const bf16_t* p = static_cast<const bf16_t*>(x);
    return rows == 1 ? f8_quant_e<bf16_t, 1>(p, qb, scale, tb, scale_t, s, st)
                     : f8_quant_e<bf16_t, kF8Block>(p, qb, scale, tb, scale_t, s, st);
  }
  const float* p = static_cast<const float*>(x);
  return rows == 1 ? f8_quant_e<float, 1>(p, qb, scale, tb, scale_t, s, st)
                   : f8_quant_e<float, kF8Block>(p, qb, scale, tb, scale_t, s, st);
}

}  // namespace kata
