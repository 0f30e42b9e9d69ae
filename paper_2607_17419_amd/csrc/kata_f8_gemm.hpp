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

namespace kata {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 f8_mfma(const i32x8& a, const i32x8& b) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 0, 0, 0);  // unscaled
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
  F8Operand() = default;
  __device__ __forceinline__ explicit F8Operand(const i32x8& codes) : v(codes) {}
};
template <>
struct F8Operand<true> {
  f16x8 v[4];
  F8Operand() = default;
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

// The products of TN operands with one.
template <int TN>
__device__ __forceinline__ void f8_row(const F8Operand<false> (&b)[TN], const F8Operand<false>& a,
                                       f32x4 (&p)[TN]) {
#pragma unroll
  for (int j = 0; j < TN; ++j) p[j] = f8_mfma(b[j].v, a.v);
}
template <int TN>
__device__ __forceinline__ void f8_row(const F8Operand<true> (&b)[TN], const F8Operand<true>& a,
                                       f32x4 (&p)[TN]) {
#pragma unroll
  for (int j = 0; j < TN; ++j) p[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int j = 0; j < TN; ++j)
      p[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[j].v[k], a.v[k], p[j], 0, 0, 0);
}
// The order of instructions that the scheduler is to keep for a row: its LDS reads, then
// matrix instructions with the vector work of the row before spread between them.
template <bool F16, int TN, int VALU>
__device__ __forceinline__ void f8_order(bool both) {
  __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
  if (both) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
      for (int k = 0; k < (F16 ? 4 : 1); ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, F16 ? (VALU + 4) / 4 : VALU, 0);
      }
    }
  } else {
    __builtin_amdgcn_sched_group_barrier(0x008, F16 ? 4 * TN : TN, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// 16 codes of a row of K from k on, zeros past its end.  VEC: aligned rows, whose chunk that K
// ends in is read whole, but of the tensor's last row, where its end may be the memory's.
template <bool VEC>
__device__ __forceinline__ uint4 f8_chunk(const uint8_t* row, int k, int K, bool last_row) {
  uint32_t w[4] = {0, 0, 0, 0};
  const int n = K - k;  // codes that are there
  if (VEC && (n >= 16 || (n > 0 && !last_row))) {
    const uint4 v = *reinterpret_cast<const uint4*>(row + k);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    if (n < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int there = n - 4 * i;
        w[i] = there >= 4 ? w[i] : there <= 0 ? 0u : w[i] & ((1u << (8 * there)) - 1u);
      }
    }
  } else if (n > 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) w[i >> 2] |= static_cast<uint32_t>(row[k + i]) << (8 * (i & 3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ i32x8 f8_operand(uint4 lo, uint4 hi) {
  struct Two { uint4 a, b; };
  return __builtin_bit_cast(i32x8, Two{lo, hi});
}

// Whether a scale's product with one of the other operand may leave fp32's normal range: two that
// are not far are between 2^-124 and 2^126.  0 and the quantisers' least scale, whose blocks hold no
// value above 2^-117, are not: such a block's part of a result is off by up to 2^-125.  A far scale
// counts as 0 in the kernels' loops; blocks that have one are gone through once more behind them,
// for the results that they left out, in fp64.  (Both ways in one loop spill.)  Without far scales
// that costs a look at four scales and a barrier, 0 to 0.3 us; 8192^3 with a far scale in every
// block 2640 us.
constexpr uint32_t kF8Least = 0x00800000, kF8Low = 0x20800000, kF8High = 0x5F000000;  // 2^-126, 2^-62, 2^63
__device__ __forceinline__ bool f8_far(float scale) {
  const uint32_t m = __float_as_uint(scale) & 0x7FFFFFFFu;
  return m - kF8Low > kF8High - kF8Low && (m & ~kF8Least) != 0;
}
__device__ __forceinline__ float f8_far_sum(float p, float sa, float sb, float acc) {
  return f8_far(sa) || f8_far(sb) ? static_cast<float>(static_cast<double>(p) * sa * sb + acc) : acc;
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
// A workgroup forms BM x BN of c over blocks of K one after the other: the next block's rows
// are copied to LDS (global_load_lds) while this one's are multiplied.  A staged row is its 128
// codes; its 16-byte chunk c lies at chunk c ^ ((row >> 1) & 7), so that the 16 rows of a
// fragment read meet no bank conflict.  The scales of all rows of four blocks at a time go
// through registers to LDS a group ahead.

__device__ __forceinline__ int f8_swz(int row) { return (row >> 1) & 7; }

// One 16-byte chunk a lane from base + offset to LDS at lds + 16 lane, counted by vmcnt.  In
// inline assembly because the compiler would drive every copy in flight home before each LDS
// read; the kernel waits with wait_vmcnt, before which it uses no vector load's result.
__device__ __forceinline__ void f8_copy16(const uint8_t* base, uint32_t offset, void* lds) {
  typedef __attribute__((address_space(3))) void lds_void;
  const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(offset), "s"(base), "s"(at)
               : "memory", "m0");
}

// Fragment of 16 rows: lane l holds chunks l / 16 and l / 16 + 4 of row l % 16 (a and b alike,
// so which k they are does not matter).  So read, 16 bytes a lane take four cycles a wave;
// as chunks 2 (l / 16) and the next, eight (measured by themselves).
__device__ __forceinline__ i32x8 f8_fragment(const char* tile, int row0) {
  const int lane = threadIdx.x & 63, r = row0 + (lane & 15), at = (lane >> 4) ^ f8_swz(r);
  const char* row = tile + r * 128;
  return f8_operand(*reinterpret_cast<const uint4*>(row + 16 * at),
                    *reinterpret_cast<const uint4*>(row + 16 * (at ^ 4)));
}

// Tiles in an order in which those that run on one XCD at a time share rows of a and of b:
// each XCD (launch index mod 8) takes a run of tiles, eight rows of tiles by column.
__device__ __forceinline__ void f8_place(const F8GemmArgs& s, int& split, int& tm, int& tn) {
  const int all = s.tm * s.tn * s.splits, xcd = blockIdx.x & 7, q = all >> 3, r = all & 7;
  int id = xcd * q + min(xcd, r) + (blockIdx.x >> 3);
  const int tiles = s.tm * s.tn;
  split = id / tiles;
  id -= split * tiles;
  const int band = id / (8 * s.tn), rows = min(8, s.tm - 8 * band);
  id -= band * 8 * s.tn;
  tn = id / rows;
  tm = 8 * band + (id - tn * rows);
}

template <int V>
struct F8Int {
  static constexpr int value = V;
};

// 8192 x 8192 x 8192 to bf16: 480-540 us on different cards, 2.0-2.3 PFLOP/s (a library product with one
// scale for all 2.71, with a scale per row 2.34); the matrix units are busy 53% of the cycles at
// 1.9 GHz.  Without the copies 427 us, without the scaled sums 355 (timing copies): the sums
// are half of the matrix time on the vector units and overlap it in part only.  Tried and not
// kept: tiles of 32 x 32 (v_mfma_f32_32x32x64: 513 us, spills), a block's first fragments read
// during the block before (spills; in tiles of 128 x 128 634 for 589), touching the lines of the
// block after the next for the L2 (578 for 540), wave priorities (nothing).
// WM x WN waves.  ROWS: rows of a block of b.  FAST: aligned rows.
template <typename E, int BM, int BN, int WM, int WN, int ROWS, bool FAST>
__global__ __launch_bounds__(64 * WM * WN, 2) void f8_tile_kernel(F8GemmArgs s) {
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int STAGE = (BM + BN) * 128, COPIES = (BM + BN) / 8 / WAVES, ROWS_ALL = BM + BN;
  constexpr bool F16 = sizeof(E) == 4;
  static_assert(ROWS_ALL <= 64 * WAVES && (BM / 8) % WAVES == 0 && (BN / 8) % WAVES == 0, "");
  __shared__ __align__(16) char lds[2 * STAGE];
  __shared__ __align__(16) float scales[2][4][ROWS_ALL];
  __shared__ int any_far;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int split, tm, tn;
  f8_place(s, split, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN, wm = wave % WM, wn = wave / WM;
  const int first = split * s.per, last = min(first + s.per, s.kb);
  const int whole = s.K / 128;  // blocks without a tail

  // copy j of a wave: rows 8 (j WAVES + wave) .. of a's tile, then of b's, one chunk a lane
  const int crow = wave * 8 + (lane >> 3);
  const uint32_t cchunk = 16 * ((lane & 7) ^ f8_swz(crow));  // (the same for all j)
  static_assert(8 * WAVES % 16 == 0, "");
  const auto copy = [&](int crow, int j, int kb, char* to) {
    constexpr int A = BM / 8 / WAVES;
    const bool is_a = j < A;
    const uint8_t* base = (is_a ? s.a + m0 * s.a_row : s.b + n0 * s.b_row) + kb * 128LL;
    const int r = min(crow + (is_a ? j : j - A) * 8 * WAVES, (is_a ? s.M - m0 : s.N - n0) - 1);
    const uint32_t ld = static_cast<uint32_t>(is_a ? s.a_row : s.b_row);  // (24 bits: f8_fast)
    f8_copy16(base, __umul24(r, ld) + cchunk, to + (j * WAVES + wave) * 1024);
  };
  const auto stage_slow = [&](int kb, char* to) {  // by registers: any alignment, any K
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      constexpr int A = BM / 8 / WAVES;
      const bool is_a = j < A;
      const int r = crow + (is_a ? j : j - A) * 8 * WAVES, end = is_a ? s.M - m0 : s.N - n0;
      const int at = min(r, end - 1);
      const uint8_t* row = is_a ? s.a + (m0 + at) * s.a_row : s.b + (n0 + at) * s.b_row;
      const uint4 v = f8_chunk<FAST>(row, kb * 128 + static_cast<int>(cchunk), s.K, at == end - 1);
      *reinterpret_cast<uint4*>(to + (j * WAVES + wave) * 1024 + lane * 16) = v;
    }
  };
  // a thread's row of scales (past the end of c: of its last row or column)
  const bool row_a = threadIdx.x < BM;
  const int sr = row_a ? min(m0 + static_cast<int>(threadIdx.x), s.M - 1)
                       : min(n0 + static_cast<int>(threadIdx.x) - BM, s.N - 1);
  const float* srow = row_a ? s.sa + static_cast<size_t>(sr) * s.kb
                            : s.sb + static_cast<size_t>(sr / ROWS) * s.kb;
  float four[4];
  const auto fetch = [&](int kb) {
#pragma unroll
    for (int k = 0; k < 4; ++k) four[k] = srow[min(kb + k, s.kb - 1)];
  };
  unsigned long long far = 0;
  const auto put = [&](int group) {
    // hardly ever more than this one look at four of them (as words: a negative one is looked at, too)
    uint32_t most = 0, least = ~0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      most = max(most, __float_as_uint(four[k]));
      least = min(least, __float_as_uint(four[k]));
    }
    if (__any(most > kF8High || least < kF8Low)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool one = f8_far(four[k]);
        far |= __ballot(one);
        if (one) four[k] = 0.f;
      }
    }
    if (threadIdx.x < ROWS_ALL) {
#pragma unroll
      for (int k = 0; k < 4; ++k) scales[group & 1][k][threadIdx.x] = four[k];
    }
  };

  f32x4 acc[TM][TN] = {};
  if (FAST && first < whole) {
#pragma unroll
    for (int j = 0; j < COPIES; ++j) copy(crow, j, first, lds);
  } else {
    stage_slow(first, lds);
  }
  if (threadIdx.x == 0) any_far = 0;
  fetch(first);
  put(0);
  const auto block = [&](int kb, auto with_copies) {
    constexpr bool COPY = decltype(with_copies)::value;
    const int step = kb - first;
    const char* now = lds + (step & 1) * STAGE;
    wait_vmcnt<0>();
    if ((step & 3) == 0 && step) put(step >> 2);
    lds_barrier();
    // the next block's copies are issued between the first rows of products; a tail here
    char* next = lds + ((step + 1) & 1) * STAGE;
    if (!COPY && kb + 1 < last) stage_slow(kb + 1, next);
    if ((step & 3) == 0) fetch(kb + 4);
    int row = crow;
    if (COPY) asm volatile("" : "+v"(row));  // so that the copies' offsets are formed here, not kept
    // fragments in the order in which they are needed
    i32x8 raw = f8_fragment(now, wm * TM * 16);
    F8Operand<F16> fb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = F8Operand<F16>(f8_fragment(now + BM * 128, (wn * TN + j) * 16));
    const float* sc = scales[(step >> 2) & 1][step & 3];
    const float* sca = sc + wm * TM * 16 + (lane & 15);
    float sa[2], sb[TN][ROWS == 1 ? 4 : 1];
    sa[0] = sca[0];
    if constexpr (ROWS == 1) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const float4 v = *reinterpret_cast<const float4*>(sc + BM + (wn * TN + j) * 16 + 4 * (lane >> 4));
        sb[j][0] = v.x, sb[j][1] = v.y, sb[j][2] = v.z, sb[j][3] = v.w;
      }
    } else {
      sb[0][0] = sc[BM + wn * TN * 16];
    }
    // the products of one row of fragments while those of the row before are scaled and added
    // and the next row's fragment is on its way
    f32x4 p[2][TN];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i <= TM; ++i) {
      if (COPY && i < TM / 2) {
#pragma unroll
        for (int k = 0; k < 2 * COPIES / TM; ++k) copy(row, i * 2 * COPIES / TM + k, kb + 1, next);
      }
      if (i < TM) {
        const F8Operand<F16> fa(raw);
        if (i + 1 < TM) raw = f8_fragment(now, (wm * TM + i + 1) * 16);
        f8_row<TN>(fb, fa, p[i & 1]);
      }
      if (i > 0) {
        const float si = ROWS == 1 ? sa[(i - 1) & 1] : sa[(i - 1) & 1] * sb[0][0];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[i - 1][j][e] = fmaf(p[(i - 1) & 1][j][e],
                                    ROWS == 1 ? si * sb[j][ROWS == 1 ? e : 0] : si, acc[i - 1][j][e]);
      }
      if (i + 1 < TM) sa[(i + 1) & 1] = sca[(i + 1) * 16];
      f8_order<F16, TN, (ROWS == 1 ? 8 : 4)>(i > 0 && i < TM);
    }
  };
  int kb = first;
  if constexpr (FAST) {
    for (; kb + 1 < min(last, whole); ++kb) block(kb, F8Int<1>());
  }
  for (; kb < last; ++kb) block(kb, F8Int<0>());
  if (far) any_far = 1;
  __syncthreads();
  if (any_far) {
    float* sc = scales[0][0];
    for (kb = first; kb < last; ++kb) {
      const float one = srow[kb];
      if (!__syncthreads_or(f8_far(one))) continue;
      __syncthreads();  // the block before has been read
      stage_slow(kb, lds);
      if (threadIdx.x < ROWS_ALL) sc[threadIdx.x] = one;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const F8Operand<F16> fa(f8_fragment(lds, (wm * TM + i) * 16));
        const float sa = sc[(wm * TM + i) * 16 + (lane & 15)];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const F8Operand<F16> fb(f8_fragment(lds + BM * 128, (wn * TN + j) * 16));
          const f32x4 p = f8_block(fb, fa);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[i][j][e] = f8_far_sum(
                p[e], sa, sc[BM + wn * TN * 16 + (ROWS == 1 ? j * 16 + 4 * (lane >> 4) + e : 0)], acc[i][j][e]);
          __builtin_amdgcn_sched_barrier(0);
        }
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

// The sum of the splits' parts, in order, V neighbouring values a thread.
template <typename E, int V>
__global__ __launch_bounds__(256) void f8_join_kernel(F8GemmArgs s) {
  const long long id = (blockIdx.x * 256LL + threadIdx.x) * V, all = static_cast<long long>(s.M) * s.N;
  if (id >= all) return;
  const float* part = s.part + id;
  float v[V] = {};
#pragma unroll 8
  for (int k = 0; k < s.splits; ++k) {
    float t[V];
    load_vec<V>(part + k * all, t);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += t[e];
  }
  const long long m = id / s.N;
  store_vec<V>(static_cast<E*>(s.c) + m * s.c_row + (id - m * s.N), v);
}

// ---- few rows of a --------------------------------------------------------------
// A workgroup forms 16 columns of c of all rows (16 MT of them); its eight waves take every
// eighth block of K, both operands straight from memory to registers, and are joined in LDS.
// 8 rows, 8192 x 4096: 10.3 us, b at 3.3 TB/s (one launch's loads are all on their way at once, so
// latency counts as much as the rate).
template <typename E, int MT, int ROWS>
__global__ __launch_bounds__(512) void f8_rows_kernel(F8GemmArgs s) {
  constexpr bool F16 = sizeof(E) == 4;
  constexpr int U = MT <= 2 ? 4 : 2;  // blocks on their way at once
  __shared__ float red[8][MT][64][4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16, whole = s.K / 128;
  const int nr = min(n0 + r, s.N - 1);
  const uint8_t* brow = s.b + nr * s.b_row;
  f32x4 acc[MT] = {};
  int far = 0;
  const auto ordinary = [&](float scale) {
    const bool one = f8_far(scale);
    far = one ? 1 : far;
    return one ? 0.f : scale;
  };
  // N blocks from kb on, every eighth; TAIL: the one that K ends in
  const auto blocks = [&](int kb, auto count, auto tail) {
    constexpr int N = decltype(count)::value;
    constexpr bool TAIL = decltype(tail)::value;
    uint4 fb[N][2], fa[N][MT][2];
    float sa[N][MT], sb[N][ROWS == 1 ? 4 : 1];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int at = kb + 8 * u, k = at * 128 + g * 32;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (TAIL) fb[u][h] = f8_chunk<true>(brow, k + 16 * h, s.K, nr == s.N - 1);
        else fb[u][h] = *reinterpret_cast<const uint4*>(brow + k + 16 * h);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int m = min(i * 16 + r, s.M - 1);
        const uint8_t* arow = s.a + m * s.a_row;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if constexpr (TAIL) fa[u][i][h] = f8_chunk<true>(arow, k + 16 * h, s.K, m == s.M - 1);
          else fa[u][i][h] = *reinterpret_cast<const uint4*>(arow + k + 16 * h);
        }
        sa[u][i] = s.sa[static_cast<size_t>(m) * s.kb + at];
      }
      if constexpr (ROWS == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sb[u][e] = s.sb[static_cast<size_t>(min(n0 + 4 * g + e, s.N - 1)) * s.kb + at];
      } else {
        sb[u][0] = s.sb[static_cast<size_t>(n0 / kF8Block) * s.kb + at];
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
#pragma unroll
      for (int e = 0; e < (ROWS == 1 ? 4 : 1); ++e) sb[u][e] = ordinary(sb[u][e]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const f32x4 p = f8_block(F8Operand<F16>(f8_operand(fb[u][0], fb[u][1])),
                                 F8Operand<F16>(f8_operand(fa[u][i][0], fa[u][i][1])));
        const float si = ordinary(sa[u][i]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][e] = fmaf(p[e], si * sb[u][ROWS == 1 ? e : 0], acc[i][e]);
      }
    }
  };
  int kb = wave;
  for (; kb + 8 * (U - 1) < whole; kb += 8 * U) blocks(kb, F8Int<U>(), F8Int<0>());
  for (; kb < whole; kb += 8) blocks(kb, F8Int<1>(), F8Int<0>());
  if (kb < s.kb) blocks(kb, F8Int<1>(), F8Int<1>());
  if (__any(far)) {
    for (kb = wave; kb < s.kb; kb += 8) {
      const int k = kb * 128 + g * 32;
      const F8Operand<F16> fb(f8_operand(f8_chunk<true>(brow, k, s.K, nr == s.N - 1),
                                         f8_chunk<true>(brow, k + 16, s.K, nr == s.N - 1)));
      float sb[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) sb[e] = s.sb[static_cast<size_t>(min(n0 + 4 * g + e, s.N - 1) / ROWS) * s.kb + kb];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int m = min(i * 16 + r, s.M - 1);
        const uint8_t* arow = s.a + m * s.a_row;
        const F8Operand<F16> fa(f8_operand(f8_chunk<true>(arow, k, s.K, m == s.M - 1),
                                           f8_chunk<true>(arow, k + 16, s.K, m == s.M - 1)));
        const f32x4 p = f8_block(fb, fa);
        const float sa = s.sa[static_cast<size_t>(m) * s.kb + kb];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = f8_far_sum(p[e], sa, sb[e], acc[i][e]);
        __builtin_amdgcn_sched_barrier(0);
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

// Tiles of 256 x 256 where there is one for each of the 256 CUs (4096 x 4096 x 4096 in bf16: 74 us
// for 88 in tiles of 128 x 128; 2048 x 2048 x 2048: 34 for 17; in fp32 their operands in f16 do
// not fit the registers).  Else tiles of 128 x 128, and K in as many splits as the model of
// the time says: a block of K takes a workgroup 0.8 us (fp32: 1.3) while it has a CU for itself
// and 0.7 (1.05) of that for each that share one; the parts' sum costs a launch, 3 us, and its
// bytes at 4 TB/s.  256 x 4096 x 4096: 1, 2, 4, 14 splits 25, 22, 22, 29 us; 1152 x 1024 x 32768 in
// fp32: 1, 2, 7, 14 splits 314, 170, 113, 133 us.
inline F8Plan f8_plan(int M, int N, int K, bool fast, bool f16) {
  const int kb = (K + 127) / 128;
  F8Plan p = {0, 0, 1, kb};
  if (fast && M <= 64) {
    p.rows_tiles = (M + 15) / 16;
    return p;
  }
  const long long big = ((M + 255LL) / 256) * ((N + 255LL) / 256);
  p.big = !f16 && big >= 256;
  const long long tiles = ((M + 127LL) / 128) * ((N + 127LL) / 128);
  if (p.big || tiles >= 256) return p;
  double best = 0.0;
  for (int n = 1; n <= 32 && n <= kb; ++n) {
    const int per = (kb + n - 1) / n, splits = (kb + per - 1) / per;
    if (splits != n) continue;
    const double share = (f16 ? 1.05 : 0.7) * static_cast<double>((tiles * n + 255) / 256);
    double us = per * (f16 ? 1.3 : 0.8) * (share > 1.0 ? share : 1.0);
    if (n > 1) us += 3.0 + 8e-6 / 4 * static_cast<double>(M) * N * n;
    if (n == 1 || us < best) best = us, p.splits = n, p.per = per;
  }
  return p;
}

// Rows of whole aligned chunks, 256 of them within 32 bits of an offset, the next one not before
// the end of a row's last chunk (which is read whole but of the last row).
inline bool f8_fast(const void* a, const void* b, long long a_row, long long b_row) {
  const auto fits = [](long long row) { return row % 16 == 0 && row >= 16 && row < (1 << 23); };
  return fits(a_row) && fits(b_row) && ptr_aligned({a, b}, 16);
}

// For any alignment: the splits do not depend on it.
size_t f8_gemm_workspace_bytes(int M, int N, int K) {
  long long splits = 1;
  for (int k = 0; k < 4; ++k) {
    const F8Plan p = f8_plan(M, N, K, k & 1, k & 2);
    if (p.splits > splits) splits = p.splits;
  }
  return splits == 1 ? 256
                     : (static_cast<size_t>(splits) * M * N * sizeof(float) + 255) &
                           ~static_cast<size_t>(255);
}

template <typename E, int ROWS>
hipError_t f8_gemm_e(F8GemmArgs s, void* ws, hipStream_t st) {
  if (s.M == 1) s.a_row = 16;  // one row: its stride is not used
  if (s.N == 1) s.b_row = 16;
  const bool fast = f8_fast(s.a, s.b, s.a_row, s.b_row);
  const F8Plan p = f8_plan(s.M, s.N, s.K, fast, sizeof(E) == 4);
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
  if (p.big) {
    if constexpr (sizeof(E) == 2) {
      if (fast) f8_tile_kernel<E, 256, 256, 2, 4, ROWS, true><<<grid, 512, 0, st>>>(s);
      else f8_tile_kernel<E, 256, 256, 2, 4, ROWS, false><<<grid, 512, 0, st>>>(s);
    }
  } else if (fast) f8_tile_kernel<E, 128, 128, 2, 2, ROWS, true><<<grid, 256, 0, st>>>(s);
  else f8_tile_kernel<E, 128, 128, 2, 2, ROWS, false><<<grid, 256, 0, st>>>(s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !s.part) return e;
  const long long all = static_cast<long long>(s.M) * s.N;
  const bool four = s.N % 4 == 0 && s.c_row % 4 == 0 && ptr_aligned({s.c}, 4 * sizeof(E));
  const unsigned blocks = static_cast<unsigned>((all / (four ? 4 : 1) + 255) / 256);
  if (four) f8_join_kernel<E, 4><<<blocks, 256, 0, st>>>(s);
  else f8_join_kernel<E, 1><<<blocks, 256, 0, st>>>(s);
  return hipGetLastError();
}

hipError_t launch_f8_gemm(const F8GemmArgs& s, int rows, bool bf16, void* ws, hipStream_t st) {
  if (rows == 1) return bf16 ? f8_gemm_e<bf16_t, 1>(s, ws, st) : f8_gemm_e<float, 1>(s, ws, st);
  return bf16 ? f8_gemm_e<bf16_t, kF8Block>(s, ws, st) : f8_gemm_e<float, kF8Block>(s, ws, st);
}

}  // namespace kata
