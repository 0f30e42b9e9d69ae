// kata_f8_gemm.hpp -- product of e4m3 operands with a scale for each block of 128:
//
//   c[m][n] = sum over blocks kb of sa[m][kb] sb[n / rows][kb] p[m][n][kb],
//   p = sum over the block's 128 k of a[m][k] b[n][k],
//
// rows = 128 (a weight's 128 x 128 blocks) or 1 (rows of another activation).  p is formed from
// zero by matrix instructions, scaled and added to the fp32 accumulator by the vector unit.  The
// matrix operands are exchanged (b's rows for the result's rows), so that a lane holds four
// neighbouring columns of one row of c and one scale of a.
//
// The instruction for e4m3 (v_mfma_f32_16x16x128_f8f6f4, 4.5 PFLOP/s measured from registers)
// adds groups of eight products (k = 8 j .. 8 j + 7) after cutting each, towards zero, to a
// multiple of 2^-13 of the power of two below the group's largest: products of ordinary
// operands come out within 1.3e-5 of themselves, all within 7 x 2^-13 of the sum of the
// groups' largest magnitudes.  A result in bf16 (steps of 2^-8) is formed so.  One in fp32 is
// formed from the same codes as f16 (exact: 2^-9 .. 448) by v_mfma_f32_16x16x32_f16, whose
// products and sums keep fp32's bits, at half of the rate.
#pragma once

#include "kata_f8.hpp"
#include "kata_quad.hpp"

namespace kata {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 f8_mfma(const i32x8& a, const i32x8& b) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 0x7F7F7F7F, 0,
                                                          0x7F7F7F7F);
}

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Eight codes (two words) as f16.
__device__ __forceinline__ f16x8 f8_as_f16(int lo, int hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// An operand of 16 rows of a block: its codes, or four operands in f16.
template <bool F16>
struct F8Operand {
  i32x8 v;
  __device__ __forceinline__ explicit F8Operand(const i32x8& codes) : v(codes) {}
};
template <>
struct F8Operand<true> {
  f16x8 v[4];
  __device__ __forceinline__ explicit F8Operand(const i32x8& codes) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = f8_as_f16(codes[2 * k], codes[2 * k + 1]);
  }
};
__device__ __forceinline__ f32x4 f8_block(const F8Operand<false>& a, const F8Operand<false>& b) {
  return f8_mfma(a.v, b.v);
}
__device__ __forceinline__ f32x4 f8_block(const F8Operand<true>& a, const F8Operand<true>& b) {
  f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[k], b.v[k], p, 0, 0, 0);
  return p;
}

// 16 codes of a row of K from k on, zeros past its end.
template <bool VEC>
__device__ __forceinline__ uint4 f8_chunk(const uint8_t* row, int k, int K) {
  if (VEC && k + 16 <= K) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t w[4] = {0, 0, 0, 0};
  if (k < K) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (k + i < K) w[i >> 2] |= static_cast<uint32_t>(row[k + i]) << (8 * (i & 3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ i32x8 f8_operand(uint4 lo, uint4 hi) {
  struct Two { uint4 a, b; };
  return __builtin_bit_cast(i32x8, Two{lo, hi});
}

// Four neighbouring columns of a row of the result.
template <typename E>
__device__ __forceinline__ void f8_store4(E* row, int n, int N, bool whole, const float (&v)[4]) {
  if (whole && n + 4 <= N) {
    store_vec<4>(row + n, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) store_f32(row + n + i, v[i]);
  }
}

// ---- tiles --------------------------------------------------------------------
// A staged row is its 128 codes of one block; its 16-byte chunk c lies at chunk
// c ^ ((row >> 1) & 7), so that the 16 rows of a fragment read meet no bank conflict.

__device__ __forceinline__ int f8_swz(int row) { return (row >> 1) & 7; }

// Rows 8 i .. 8 i + 7 of a tile, one 16-byte chunk a lane, by registers: any alignment, any K.
template <bool VEC>
__device__ __forceinline__ void f8_stage_slow(const uint8_t* src, long long ld, int row0, int rows,
                                              int k0, int K, int i, char* lds) {
  const int lane = threadIdx.x & 63, r = i * 8 + (lane >> 3), pos = lane & 7;
  const int at = min(row0 + r, rows - 1);
  const uint4 v = f8_chunk<VEC>(src + at * ld, k0 + 16 * (pos ^ f8_swz(r)), K);
  *reinterpret_cast<uint4*>(lds + i * 1024 + lane * 16) = v;
}
// The same of a whole block of aligned rows, straight to LDS.
__device__ __forceinline__ void f8_stage_fast(const uint8_t* src, long long ld, int row0, int rows,
                                              int k0, int i, char* lds) {
  const int lane = threadIdx.x & 63, r = i * 8 + (lane >> 3), pos = lane & 7;
  const int at = min(row0 + r, rows - 1);
  qd_copy16(src + at * ld + k0 + 16 * (pos ^ f8_swz(r)), lds + i * 1024);
}

// Fragment of 16 rows: lane l holds chunks 2 (l / 16) and the next of row l % 16.
__device__ __forceinline__ i32x8 f8_fragment(const char* tile, int row0) {
  const int lane = threadIdx.x & 63, r = row0 + (lane & 15), g = lane >> 4, z = f8_swz(r);
  const char* row = tile + r * 128;
  return f8_operand(*reinterpret_cast<const uint4*>(row + 16 * ((2 * g) ^ z)),
                    *reinterpret_cast<const uint4*>(row + 16 * ((2 * g + 1) ^ z)));
}

// BM x BN tiles of c; WM x WN waves.  ROWS: rows of a block of b.  FAST: aligned rows.
template <typename E, int BM, int BN, int WM, int WN, int ROWS, bool FAST>
__global__ __launch_bounds__(64 * WM * WN) void f8_tile_kernel(F8GemmArgs s) {
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int STAGE = (BM + BN) * 128;
  constexpr bool F16 = sizeof(E) == 4;
  __shared__ __align__(16) char lds[2 * STAGE];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int tiles = s.tm * s.tn, split = blockIdx.x / tiles;
  int id = blockIdx.x - split * tiles;
  const int tn = id / s.tm, tm = id - tn * s.tm;
  const int m0 = tm * BM, n0 = tn * BN, wm = wave % WM, wn = wave / WM;
  const int first = split * s.per, last = min(first + s.per, s.kb);
  const int whole = s.K / 128;  // blocks without a tail

  const auto stage = [&](int kb, char* to) {
    const bool fast = FAST && kb < whole;
#pragma unroll
    for (int j = 0; j < (BM + BN) / 8 / WAVES; ++j) {
      const int i = j * WAVES + wave;
      const bool is_a = i < BM / 8;
      const uint8_t* src = is_a ? s.a : s.b;
      const long long ld = is_a ? s.a_row : s.b_row;
      const int row0 = is_a ? m0 : n0, rows = is_a ? s.M : s.N;
      const int at = is_a ? i : i - BM / 8;
      char* tile = is_a ? to : to + BM * 128;
      if (fast) f8_stage_fast(src, ld, row0, rows, kb * 128, at, tile);
      else f8_stage_slow<FAST>(src, ld, row0, rows, kb * 128, s.K, at, tile);
    }
  };

  f32x4 acc[TM][TN] = {};
  stage(first, lds);
  for (int kb = first; kb < last; ++kb) {
    char* now = lds + ((kb - first) & 1) * STAGE;
    // scales of this block
    float sa[TM], sb[TN][ROWS == 1 ? 4 : 1];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = min(m0 + (wm * TM + i) * 16 + (lane & 15), s.M - 1);
      sa[i] = s.sa[static_cast<size_t>(m) * s.kb + kb];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = n0 + (wn * TN + j) * 16;
      if constexpr (ROWS == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sb[j][e] = s.sb[static_cast<size_t>(min(n + 4 * (lane >> 4) + e, s.N - 1)) * s.kb + kb];
      } else {
        sb[j][0] = s.sb[static_cast<size_t>(min(n, s.N - 1) / kF8Block) * s.kb + kb];
      }
    }
    wait_vmcnt<0>();
    __syncthreads();
    if (kb + 1 < last) stage(kb + 1, lds + ((kb + 1 - first) & 1) * STAGE);
    i32x8 fb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = f8_fragment(now + BM * 128, (wn * TN + j) * 16);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const F8Operand<F16> fa(f8_fragment(now, (wm * TM + i) * 16));
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const f32x4 p = f8_block(F8Operand<F16>(fb[j]), fa);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][j][e] = fmaf(p[e], sa[i] * sb[j][ROWS == 1 ? e : 0], acc[i][j][e]);
      }
    }
  }
  const bool pieces = s.part ? s.N % 4 == 0
                             : s.c_row % 4 == 0 &&
                                   (reinterpret_cast<uintptr_t>(s.c) & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + (wm * TM + i) * 16 + (lane & 15);
    if (m >= s.M) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = n0 + (wn * TN + j) * 16 + 4 * (lane >> 4);
      const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
      if (s.part)
        f8_store4(s.part + (static_cast<size_t>(split) * s.M + m) * s.N, n, s.N, pieces, v);
      else
        f8_store4(static_cast<E*>(s.c) + m * s.c_row, n, s.N, pieces, v);
    }
  }
}

// The sum of the splits' parts, in order.
template <typename E>
__global__ __launch_bounds__(256) void f8_join_kernel(F8GemmArgs s) {
  const long long id = (blockIdx.x * 256LL + threadIdx.x), all = static_cast<long long>(s.M) * s.N;
  if (id >= all) return;
  float v = s.part[id];
  for (int k = 1; k < s.splits; ++k) v += s.part[k * all + id];
  const long long m = id / s.N;
  store_f32(static_cast<E*>(s.c) + m * s.c_row + (id - m * s.N), v);
}

// ---- few rows of a --------------------------------------------------------------
// A workgroup forms 16 columns of c of all rows (16 MT of them); its eight waves take every
// eighth block of K, both operands straight from memory to registers, and are joined in LDS.
template <typename E, int MT, int ROWS>
__global__ __launch_bounds__(512) void f8_rows_kernel(F8GemmArgs s) {
  constexpr bool F16 = sizeof(E) == 4;
  constexpr int U = MT <= 2 ? 4 : 2;  // blocks on their way at once
  __shared__ float red[8][MT][64][4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const uint8_t* brow = s.b + min(n0 + r, s.N - 1) * s.b_row;
  f32x4 acc[MT] = {};
  for (int kb0 = wave; kb0 < s.kb; kb0 += 8 * U) {
    uint4 fb[U][2], fa[U][MT][2];
    float sa[U][MT], sb[U][ROWS == 1 ? 4 : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = kb0 + 8 * u, k = kb * 128 + g * 32;  // (past the end: zeros)
      const int kc = min(kb, s.kb - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) fb[u][h] = f8_chunk<true>(brow, k + 16 * h, s.K);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int m = min(i * 16 + r, s.M - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) fa[u][i][h] = f8_chunk<true>(s.a + m * s.a_row, k + 16 * h, s.K);
        sa[u][i] = s.sa[static_cast<size_t>(m) * s.kb + kc];
      }
      if constexpr (ROWS == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sb[u][e] = s.sb[static_cast<size_t>(min(n0 + 4 * g + e, s.N - 1)) * s.kb + kc];
      } else {
        sb[u][0] = s.sb[static_cast<size_t>(n0 / kF8Block) * s.kb + kc];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb0 + 8 * u >= s.kb) break;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const f32x4 p = f8_block(F8Operand<F16>(f8_operand(fb[u][0], fb[u][1])),
                                 F8Operand<F16>(f8_operand(fa[u][i][0], fa[u][i][1])));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][e] = fmaf(p[e], sa[u][i] * sb[u][ROWS == 1 ? e : 0], acc[i][e]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][i][lane][e] = acc[i][e];
  __syncthreads();
  const bool pieces =
      s.c_row % 4 == 0 && (reinterpret_cast<uintptr_t>(s.c) & (4 * sizeof(E) - 1)) == 0;
  if (wave >= MT) return;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v[e] += red[w][wave][lane][e];
  }
  const int m = wave * 16 + r;
  if (m < s.M) f8_store4(static_cast<E*>(s.c) + m * s.c_row, n0 + 4 * g, s.N, pieces, v);
}

// ---- launches ---------------------------------------------------------------

struct F8Plan {
  int rows_tiles;  // > 0: few rows, this many pieces of 16
  int big;         // 256 x 256 tiles (else 128 x 128)
  int splits, per;
};

// Splits of K where the tiles leave CUs idle.
inline F8Plan f8_plan(int M, int N, int K, bool fast) {
  const int kb = (K + 127) / 128;
  F8Plan p = {0, 0, 1, kb};
  if (fast && M <= 64) {
    p.rows_tiles = (M + 15) / 16;
    return p;
  }
  const long long big = ((M + 255LL) / 256) * ((N + 255LL) / 256);
  p.big = big >= 256;
  const long long tiles = p.big ? big : ((M + 127LL) / 128) * ((N + 127LL) / 128);
  if (tiles < 256) {
    long long n = 512 / tiles;
    if (n > kb / 2) n = kb / 2;  // two blocks at least
    if (n > 32) n = 32;
    if (n > 1) {
      p.per = static_cast<int>((kb + n - 1) / n);
      p.splits = (kb + p.per - 1) / p.per;
    }
  }
  return p;
}

inline bool f8_fast(const void* a, const void* b, long long a_row, long long b_row) {
  return a_row % 16 == 0 && b_row % 16 == 0 && ptr_aligned({a, b}, 16);
}

// For any alignment: the splits do not depend on it.
size_t f8_gemm_workspace_bytes(int M, int N, int K) {
  const F8Plan p = f8_plan(M, N, K, false), f = f8_plan(M, N, K, true);
  const long long splits = p.splits > f.splits ? p.splits : f.splits;
  return splits == 1 ? 256
                     : (static_cast<size_t>(splits) * M * N * sizeof(float) + 255) &
                           ~static_cast<size_t>(255);
}

template <typename E, int ROWS>
hipError_t f8_gemm_e(F8GemmArgs s, void* ws, hipStream_t st) {
  const bool fast = f8_fast(s.a, s.b, s.a_row, s.b_row);
  const F8Plan p = f8_plan(s.M, s.N, s.K, fast);
  s.kb = (s.K + 127) / 128;
  s.splits = p.splits, s.per = p.per;
  s.part = p.splits > 1 ? static_cast<float*>(ws) : nullptr;
  if (p.rows_tiles) {
    const dim3 grid((s.N + 15) / 16);
    if (p.rows_tiles == 1) f8_rows_kernel<E, 1, ROWS><<<grid, 512, 0, st>>>(s);
    else if (p.rows_tiles == 2) f8_rows_kernel<E, 2, ROWS><<<grid, 512, 0, st>>>(s);
    else f8_rows_kernel<E, 4, ROWS><<<grid, 512, 0, st>>>(s);
    return hipGetLastError();
  }
  const int B = p.big ? 256 : 128;
  s.tm = (s.M + B - 1) / B, s.tn = (s.N + B - 1) / B;
  const unsigned grid = static_cast<unsigned>(static_cast<long long>(s.tm) * s.tn * s.splits);
  if (p.big && fast) f8_tile_kernel<E, 256, 256, 2, 4, ROWS, true><<<grid, 512, 0, st>>>(s);
  else if (p.big) f8_tile_kernel<E, 256, 256, 2, 4, ROWS, false><<<grid, 512, 0, st>>>(s);
  else if (fast) f8_tile_kernel<E, 128, 128, 2, 2, ROWS, true><<<grid, 256, 0, st>>>(s);
  else f8_tile_kernel<E, 128, 128, 2, 2, ROWS, false><<<grid, 256, 0, st>>>(s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !s.part) return e;
  const long long all = static_cast<long long>(s.M) * s.N;
  f8_join_kernel<E><<<static_cast<unsigned>((all + 255) / 256), 256, 0, st>>>(s);
  return hipGetLastError();
}

hipError_t launch_f8_gemm(const F8GemmArgs& s, int rows, bool bf16, void* ws, hipStream_t st) {
  if (rows == 1) return bf16 ? f8_gemm_e<bf16_t, 1>(s, ws, st) : f8_gemm_e<float, 1>(s, ws, st);
  return bf16 ? f8_gemm_e<bf16_t, kF8Block>(s, ws, st) : f8_gemm_e<float, kF8Block>(s, ws, st);
}

}  // namespace kata
