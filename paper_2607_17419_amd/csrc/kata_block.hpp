// kata_block.hpp -- launch interface between the host side of kata_block_api.hpp and the
// kernels of kata_block.hip.
#pragma once

#include "kata_internal.hpp"

namespace kata {

constexpr int kF8Block = 128;  // columns (and rows) of a scale

// Strides are in elements between rows; rows are contiguous.
struct AddNormArgs {
  int M, D;
  long long x_row, res_row, sum_row, y_row, q_row;  // backward: s, dy, dsum, dx
  float eps;
};
hipError_t launch_add_norm(const void* x, const void* res, const float* w, void* sum, void* y,
                           void* q, float* scale, const AddNormArgs& s, bool bf16, hipStream_t st);
size_t add_norm_bwd_workspace_bytes(int M, int D);
hipError_t launch_add_norm_bwd(const void* sum, const float* w, const void* dy, const void* dsum,
                               void* dx, float* dw, void* ws, const AddNormArgs& s, bool bf16,
                               bool dy_bf16, hipStream_t st);

struct F8QuantArgs {
  int M, K;
  long long x_row, q_row, qt_row;
  int kt;  // tiles along the columns
};
hipError_t launch_f8_quant(const void* x, void* q, float* scale, void* qt, float* scale_t, int rows,
                           F8QuantArgs s, bool bf16, hipStream_t st);

struct F8GemmArgs {
  const uint8_t *a, *b;
  const float *sa, *sb;
  void* c;
  float* part;  // [splits][M][N], or null: c itself
  long long a_row, b_row, c_row;
  int M, N, K, kb;  // kb: blocks of K
  int tm, tn;       // tiles
  int splits, per;  // blocks of a split
};
size_t f8_gemm_workspace_bytes(int M, int N, int K);
hipError_t launch_f8_gemm(const F8GemmArgs& s, int rows, bool bf16, void* ws, hipStream_t st);

constexpr int kRecurSpan = 64;   // tokens of a state kept for the gradients
constexpr int kRecurCols = 128;  // channels of a workgroup
struct RecurArgs {
  const void *x, *r, *i, *dy;
  const float *lam, *rb, *ib, *h_in, *dh_out;
  const int* lengths;
  void *y, *dx, *dr, *di;
  float *h_out, *dh_in;
  float* starts;    // [B][ceil(T / kRecurSpan)][D]: the state before each span (gradients: read)
  float* part;      // [B * spans][3 D]: sums for dlam, drb, dib
  unsigned* ticket;  // the chain: see kata_recur.hpp
  uint64_t* words;
  const float* slopes;  // [D]: c softplus(lam), or null
  int B, T, D, spans, tiles, cols;
  long long xb, xt, rb_, rt, ib_, it, yb, yt;  // y, or dy in the backward
  long long dxb, dxt, drb, drt, dib, dit;
  float c;
};
size_t recur_workspace_bytes(int B, int T, int D, bool backward);
hipError_t launch_recur_fwd(const RecurArgs& s, void* ws, bool bf16, hipStream_t st);
hipError_t launch_recur_bwd(const RecurArgs& s, float* dlam, float* drb, float* dib, void* ws, bool bf16,
                            hipStream_t st);
hipError_t launch_recur_step(float* h, const RecurArgs& s, bool bf16, hipStream_t st);

}  // namespace kata
