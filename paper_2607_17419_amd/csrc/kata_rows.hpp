// kata_rows.hpp -- what the mixer operators (kata_conv.hpp, kata_qknorm.hpp,
// kata_ssm.hpp) share: short vectors of elements as fp32, and the sum of
// per-workgroup partial sums.
#pragma once

#include <initializer_list>

#include "kata_internal.hpp"

namespace kata {

// Whether all addresses (or null) are multiples of a power of two.
inline bool ptr_aligned(std::initializer_list<const void*> p, int bytes) {
  for (const void* q : p)
    if (reinterpret_cast<uintptr_t>(q) & static_cast<uintptr_t>(bytes - 1)) return false;
  return true;
}

// V consecutive elements as fp32; the address is aligned to V elements.
template <int V>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(p + i);
      v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[i];
  }
}

template <int V>
__device__ __forceinline__ void load_vec(const bf16_t* p, float (&v)[V]) {
  if constexpr (V == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16lo_f32(w[i]), v[2 * i + 1] = bf16hi_f32(w[i]);
  } else if constexpr (V == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = bf16lo_f32(u.x), v[1] = bf16hi_f32(u.x), v[2] = bf16lo_f32(u.y), v[3] = bf16hi_f32(u.y);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(p[i]);
  }
}

__device__ __forceinline__ void store_f32(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_f32(bf16_t* p, float x) {
  p->bits = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

// The same elements back, each rounded once to its type.
template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4)
      *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v[i];
  }
}

template <int V>
__device__ __forceinline__ void store_vec(bf16_t* p, const float (&v)[V]) {
  if constexpr (V == 8) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                   pack_bf16x2(v[6], v[7]));
  } else if constexpr (V == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) store_f32(p + i, v[i]);
  }
}

// Logistic function from the hardware's exp2 and reciprocal (each within 1 ulp; the
// product x log2 e adds |x| 2^-24 to the exponential's relative error, which counts only
// where the result is near 0 or 1 and x (1 - sigmoid) small).  1 + inf gives 0.
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * x));
}

// V elements as they stand in memory, loaded some time before they are used.
template <typename E, int V>
struct RawVec {
  E e[V];
};
template <typename E, int V>
__device__ __forceinline__ RawVec<E, V> load_raw(const E* p) {
  RawVec<E, V> r;
  if constexpr (V * sizeof(E) == 16) r = __builtin_bit_cast(RawVec<E, V>, *reinterpret_cast<const uint4*>(p));
  else if constexpr (V * sizeof(E) == 8) r = __builtin_bit_cast(RawVec<E, V>, *reinterpret_cast<const uint2*>(p));
  else
#pragma unroll
    for (int i = 0; i < V; ++i) r.e[i] = p[i];
  return r;
}
template <typename E, int V>
__device__ __forceinline__ void raw_f32(const RawVec<E, V>& r, float (&v)[V]) {
  if constexpr (sizeof(E) == 2 && V % 2 == 0) {
    struct Words { uint32_t w[V / 2]; };
    const Words u = __builtin_bit_cast(Words, r);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) v[2 * i] = bf16lo_f32(u.w[i]), v[2 * i + 1] = bf16hi_f32(u.w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(r.e[i]);
  }
}

// Sum over groups of LANES (a power of two) neighbouring lanes, in every lane; within
// rows of 16 lanes by DPP moves.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ float sum_group(float x) {
  if constexpr (LANES >= 2) x += dpp_move<0xB1>(x);    // lane ^ 1
  if constexpr (LANES >= 4) x += dpp_move<0x4E>(x);    // lane ^ 2
  if constexpr (LANES >= 8) x += dpp_move<0x141>(x);   // 7 - lane of 8
  if constexpr (LANES >= 16) x += dpp_move<0x140>(x);  // 15 - lane of 16
  if constexpr (LANES >= 32) x += __shfl_xor(x, 16);
  if constexpr (LANES >= 64) x += __shfl_xor(x, 32);
  return x;
}

// Sums of per-workgroup partial sums: part[n][cols], fp32 or fp64, is summed over n
// in fp64 in a fixed order, so that results do not depend on the order in which
// workgroups ran; column c goes to out[0], out[1] or out[2] with their widths
// one after the other (a null one is dropped).
struct SumOutputs {
  float* out[3];
  int width[3];
};
constexpr int kSumCols = 16, kSumRows = 16;  // a workgroup: 16 columns, 16 shares of n each

template <typename Part>
__global__ __launch_bounds__(kSumCols* kSumRows) void sum_partials(const Part* part, int n,
                                                                   int cols, SumOutputs o) {
  __shared__ double s[kSumRows][kSumCols];
  const int x = threadIdx.x % kSumCols, y = threadIdx.x / kSumCols;
  int c = blockIdx.x * kSumCols + x;
  double acc = 0.0;
  if (c < cols) {
#pragma unroll 8
    for (int i = y; i < n; i += kSumRows) acc += part[static_cast<size_t>(i) * cols + c];
  }
  s[y][x] = acc;
  __syncthreads();
  if (y != 0 || c >= cols) return;
#pragma unroll
  for (int i = 1; i < kSumRows; ++i) acc += s[i][x];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (c < o.width[k]) {
      if (o.out[k]) o.out[k][c] = static_cast<float>(acc);
      return;
    }
    c -= o.width[k];
  }
}

template <typename Part>
hipError_t launch_sum_partials(const Part* part, int n, int cols, const SumOutputs& o,
                               hipStream_t st) {
  sum_partials<<<(cols + kSumCols - 1) / kSumCols, kSumCols * kSumRows, 0, st>>>(part, n, cols, o);
  return hipGetLastError();
}

}  // namespace kata
