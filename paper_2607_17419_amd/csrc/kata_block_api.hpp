// kata_block_api.hpp -- host side of the residual norm, the e4m3 quantiser and product, and the
// gated linear recurrence of kata.h: argument checks and launches.  Included by kata_api.hip
// after kata_mixer_api.hpp, whose helpers it uses.
#include "kata_block.hpp"

namespace {

constexpr int kMaxRows = 1 << 30;
constexpr int kMaxNormWidth = 1 << 15;

bool row_ok(long long rows, long long stride, long long inner, bool output) {
  return layout_ok({{rows, stride}}, inner, output);
}

// ---- residual norm ------------------------------------------------------------------

kata_status_t add_norm_check(int M, int D, float eps, int dtype) {
  if (M < 1 || D < 1 || !type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return KATA_ERR_INVALID_ARG;
  if (!product_ok(M, D, 1, 1)) return KATA_ERR_INVALID_ARG;
  if (D > kMaxNormWidth || M > kMaxThreads / (D > 8192 ? 1024 : 256)) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

// ---- e4m3 ---------------------------------------------------------------------------

kata_status_t f8_quant_check(int M, int K, int rows, int dtype) {
  if (M < 1 || K < 1 || !type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (rows != 1 && rows != kata::kF8Block) return KATA_ERR_INVALID_ARG;
  if (!product_ok(M, K, 1, 1)) return KATA_ERR_INVALID_ARG;
  if (M > kMaxRows || K > kMaxRows) return KATA_ERR_UNSUPPORTED;
  const long long tiles = ((M + 127LL) / 128) * ((K + 127LL) / 128);
  return tiles > kMaxThreads / 256 ? KATA_ERR_UNSUPPORTED : KATA_OK;
}

kata_status_t f8_gemm_check(int M, int N, int K, int b_rows, int dtype) {
  if (M < 1 || N < 1 || K < 1 || !type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (b_rows != 1 && b_rows != kata::kF8Block) return KATA_ERR_INVALID_ARG;
  if (!product_ok(M, K, 1, 1) || !product_ok(N, K, 1, 1) || !product_ok(M, N, 1, 1))
    return KATA_ERR_INVALID_ARG;
  if (M > kMaxRows || N > kMaxRows || K > kMaxRows) return KATA_ERR_UNSUPPORTED;
  const long long tiles = ((M + 127LL) / 128) * ((N + 127LL) / 128);
  if (tiles > kMaxThreads / 512 || (N + 15LL) / 16 > kMaxThreads / 512) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

// ---- gated linear recurrence ------------------------------------------------------------

kata_status_t recur_check(int B, int T, int D, float c, int dtype) {
  if (B < 1 || T < 1 || D < 1 || !type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (!(c > 0.f) || !std::isfinite(c)) return KATA_ERR_INVALID_ARG;
  if (!product_ok(B, T, D, 1)) return KATA_ERR_INVALID_ARG;
  if (T > kMaxTokens || D > (1 << 20)) return KATA_ERR_UNSUPPORTED;
  const long long spans = (T + kata::kRecurSpan - 1LL) / kata::kRecurSpan;
  const long long tiles = (D + kata::kRecurCols - 1LL) / kata::kRecurCols;
  if (B * spans > kMaxThreads / 512 / tiles) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

kata_recur_strides_t recur_contiguous(int T, int D) {
  const long long t = D, b = static_cast<long long>(T) * D;
  return {b, t, b, t, b, t, b, t, b, t, b, t, b, t};
}

// The inputs that all directions take; false: something is wrong with them.
bool recur_inputs(kata::RecurArgs& a, const void* x, const void* r, const void* i, const float* lam,
                  const float* rb, const float* ib, int B, int T, int D,
                  const kata_recur_strides_t& s, float c, int dtype) {
  for (const void* p : {x, r, i})
    if (!p || !elem_aligned(p, dtype)) return false;
  if (!lam || !aligned_to(lam, 4) || !aligned_to(rb, 4) || !aligned_to(ib, 4)) return false;
  if (!layout_ok({{B, s.x_batch}, {T, s.x_token}}, D, false)) return false;
  if (!layout_ok({{B, s.r_batch}, {T, s.r_token}}, D, false)) return false;
  if (!layout_ok({{B, s.i_batch}, {T, s.i_token}}, D, false)) return false;
  a = {};
  a.x = x, a.r = r, a.i = i, a.lam = lam, a.rb = rb, a.ib = ib;
  a.B = B, a.T = T, a.D = D, a.c = c;
  a.xb = s.x_batch, a.xt = s.x_token, a.rb_ = s.r_batch, a.rt = s.r_token;
  a.ib_ = s.i_batch, a.it = s.i_token, a.yb = s.y_batch, a.yt = s.y_token;
  return true;
}

}  // namespace

extern "C" {

kata_status_t kata_add_norm_fwd(const void* x, const void* res, const float* w, void* sum, void* y,
                                void* q, float* scale, int M, int D, long long x_row,
                                long long res_row, long long sum_row, long long y_row,
                                long long q_row, float eps, kata_dtype_t dtype,
                                hipStream_t stream) {
  const kata_status_t c = add_norm_check(M, D, eps, raw(dtype));
  if (c != KATA_OK) return c;
  if (!x || (res != nullptr) != (sum != nullptr) || (q != nullptr) != (scale != nullptr) || (!y && !q))
    return KATA_ERR_INVALID_ARG;
  for (const void* p : {x, res, static_cast<const void*>(sum), static_cast<const void*>(y)})
    if (!elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  if (!aligned_to(w, 4) || !aligned_to(scale, 4)) return KATA_ERR_INVALID_ARG;
  if (!row_ok(M, x_row, D, false) || (res && !row_ok(M, res_row, D, false)) ||
      (sum && !row_ok(M, sum_row, D, true)) || (y && !row_ok(M, y_row, D, true)) ||
      (q && !row_ok(M, q_row, D, true)))
    return KATA_ERR_INVALID_ARG;
  // sum may stand in res's place, row by row
  const bool in_place = sum && sum == res && sum_row == res_row;
  if (!apart({y, q, scale}, {x, res, w, sum}) || (!in_place && !apart({sum}, {x, res, w})) ||
      (in_place && (sum == x || sum == w)))
    return KATA_ERR_INVALID_ARG;
  const kata::AddNormArgs a = {M,     D, x_row, res ? res_row : 0, sum ? sum_row : 0, y ? y_row : 0,
                               q ? q_row : 0, eps};
  return from_hip(kata::launch_add_norm(x, res, w, sum, y, q, scale, a, dtype == KATA_BF16, stream));
}

size_t kata_add_norm_bwd_workspace_bytes(int M, int D, kata_dtype_t dtype) {
  if (add_norm_check(M, D, 0.f, raw(dtype)) != KATA_OK) return 0;
  return kata::add_norm_bwd_workspace_bytes(M, D);
}

kata_status_t kata_add_norm_bwd_ws(const void* sum, const float* w, const void* dy,
                                   const void* dsum, void* dx, float* dw, int M, int D,
                                   long long sum_row, long long dy_row, long long dsum_row,
                                   long long dx_row, float eps, kata_dtype_t dtype,
                                   kata_dtype_t dy_dtype, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  const kata_status_t c = add_norm_check(M, D, eps, raw(dtype));
  if (c != KATA_OK) return c;
  if (!type_ok(raw(dy_dtype))) return KATA_ERR_INVALID_ARG;
  if (dy_dtype == KATA_BF16 && dtype != KATA_BF16) return KATA_ERR_UNSUPPORTED;
  if (!sum || !dy || !dx) return KATA_ERR_INVALID_ARG;
  for (const void* p : {sum, dsum, static_cast<const void*>(dx)})
    if (!elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  if (!elem_aligned(dy, dy_dtype) || !aligned_to(w, 4) || !aligned_to(dw, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({dx, dw, workspace}, {sum, w, dy, dsum})) return KATA_ERR_INVALID_ARG;
  if (!row_ok(M, sum_row, D, false) || !row_ok(M, dy_row, D, false) ||
      (dsum && !row_ok(M, dsum_row, D, false)) || !row_ok(M, dx_row, D, true))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::add_norm_bwd_workspace_bytes(M, D)))
    return KATA_ERR_INVALID_ARG;
  const kata::AddNormArgs a = {M, D, sum_row, dy_row, dsum ? dsum_row : 0, dx_row, 0, eps};
  return from_hip(kata::launch_add_norm_bwd(sum, w, dy, dsum, dx, dw, workspace, a,
                                            dtype == KATA_BF16, dy_dtype == KATA_BF16, stream));
}

kata_status_t kata_f8_quant(const void* x, void* q, float* scale, void* qt, float* scale_t, int M,
                            int K, int rows, long long x_row, long long q_row, long long qt_row,
                            kata_dtype_t dtype, hipStream_t stream) {
  const kata_status_t c = f8_quant_check(M, K, rows, raw(dtype));
  if (c != KATA_OK) return c;
  if (!x || !elem_aligned(x, dtype) || (!q && !qt) || (q != nullptr) != (scale != nullptr) ||
      (qt != nullptr) != (scale_t != nullptr))
    return KATA_ERR_INVALID_ARG;
  if (!aligned_to(scale, 4) || !aligned_to(scale_t, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({q, scale, qt, scale_t}, {x})) return KATA_ERR_INVALID_ARG;
  if (!row_ok(M, x_row, K, false) || (q && !row_ok(M, q_row, K, true)) ||
      (qt && !row_ok(K, qt_row, M, true)))
    return KATA_ERR_INVALID_ARG;
  const kata::F8QuantArgs a = {M, K, x_row, q ? q_row : 0, qt ? qt_row : 0, 0};
  return from_hip(kata::launch_f8_quant(x, q, scale, qt, scale_t, rows, a, dtype == KATA_BF16, stream));
}

size_t kata_f8_gemm_workspace_bytes(int M, int N, int K) {
  if (f8_gemm_check(M, N, K, 1, KATA_BF16) != KATA_OK) return 0;
  return kata::f8_gemm_workspace_bytes(M, N, K);
}

kata_status_t kata_f8_gemm_ws(const void* a, const float* a_scale, const void* b,
                              const float* b_scale, void* c, int M, int N, int K, int b_rows,
                              long long a_row, long long b_row, long long c_row,
                              kata_dtype_t dtype, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  const kata_status_t st = f8_gemm_check(M, N, K, b_rows, raw(dtype));
  if (st != KATA_OK) return st;
  if (!a || !a_scale || !b || !b_scale || !c || !elem_aligned(c, dtype)) return KATA_ERR_INVALID_ARG;
  if (!aligned_to(a_scale, 4) || !aligned_to(b_scale, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({c, workspace}, {a, a_scale, b, b_scale})) return KATA_ERR_INVALID_ARG;
  if (!row_ok(M, a_row, K, false) || !row_ok(N, b_row, K, false) || !row_ok(M, c_row, N, true))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::f8_gemm_workspace_bytes(M, N, K)))
    return KATA_ERR_INVALID_ARG;
  kata::F8GemmArgs s = {};
  s.a = static_cast<const uint8_t*>(a), s.b = static_cast<const uint8_t*>(b);
  s.sa = a_scale, s.sb = b_scale, s.c = c;
  s.a_row = a_row, s.b_row = b_row, s.c_row = c_row, s.M = M, s.N = N, s.K = K;
  return from_hip(kata::launch_f8_gemm(s, b_rows, dtype == KATA_BF16, workspace, stream));
}

int kata_recur_spans(int T) {
  return T < 1 ? 0 : (T - 1) / kata::kRecurSpan + 1;
}

size_t kata_recur_workspace_bytes(int B, int T, int D, kata_dtype_t dtype, int backward) {
  if (recur_check(B, T, D, 1.f, raw(dtype)) != KATA_OK) return 0;
  return kata::recur_workspace_bytes(B, T, D, backward != 0);
}

kata_status_t kata_recur_fwd_ws(const void* x, const void* r, const void* i, const float* lam,
                                const float* r_bias, const float* i_bias, const float* h_in,
                                const int* lengths, void* y, float* h_out, float* starts, int B,
                                int T, int D, const kata_recur_strides_t* strides, float c,
                                kata_dtype_t dtype, void* workspace, size_t workspace_bytes,
                                hipStream_t stream) {
  const kata_status_t st = recur_check(B, T, D, c, raw(dtype));
  if (st != KATA_OK) return st;
  const kata_recur_strides_t s = strides ? *strides : recur_contiguous(T, D);
  kata::RecurArgs a;
  if (!y || !elem_aligned(y, dtype) ||
      !recur_inputs(a, x, r, i, lam, r_bias, i_bias, B, T, D, s, c, dtype))
    return KATA_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(h_in), static_cast<const void*>(lengths),
                        static_cast<const void*>(h_out), static_cast<const void*>(starts)})
    if (!aligned_to(p, 4)) return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, s.y_batch}, {T, s.y_token}}, D, true)) return KATA_ERR_INVALID_ARG;
  if (!apart({y, h_out, starts, workspace}, {x, r, i, lam, r_bias, i_bias, h_in, lengths}))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::recur_workspace_bytes(B, T, D, false)))
    return KATA_ERR_INVALID_ARG;
  a.y = y, a.h_in = h_in, a.h_out = h_out, a.lengths = lengths, a.starts = starts;
  return from_hip(kata::launch_recur_fwd(a, workspace, dtype == KATA_BF16, stream));
}

kata_status_t kata_recur_bwd_ws(const void* x, const void* r, const void* i, const float* lam,
                                const float* r_bias, const float* i_bias, const float* h_in,
                                const int* lengths, const float* starts, const void* dy,
                                const float* dh_out, void* dx, void* dr, void* di, float* dlam,
                                float* dr_bias, float* di_bias, float* dh_in, int B, int T, int D,
                                const kata_recur_strides_t* strides, float c, kata_dtype_t dtype,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const kata_status_t st = recur_check(B, T, D, c, raw(dtype));
  if (st != KATA_OK) return st;
  const kata_recur_strides_t s = strides ? *strides : recur_contiguous(T, D);
  kata::RecurArgs a;
  if (!recur_inputs(a, x, r, i, lam, r_bias, i_bias, B, T, D, s, c, dtype)) return KATA_ERR_INVALID_ARG;
  for (const void* p : {dy, static_cast<const void*>(dx), static_cast<const void*>(dr),
                        static_cast<const void*>(di)})
    if (!p || !elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(h_in), static_cast<const void*>(lengths),
                        static_cast<const void*>(starts), static_cast<const void*>(dh_out),
                        static_cast<const void*>(dlam), static_cast<const void*>(dr_bias),
                        static_cast<const void*>(di_bias), static_cast<const void*>(dh_in)})
    if (!aligned_to(p, 4)) return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, s.y_batch}, {T, s.y_token}}, D, false) ||
      !layout_ok({{B, s.dx_batch}, {T, s.dx_token}}, D, true) ||
      !layout_ok({{B, s.dr_batch}, {T, s.dr_token}}, D, true) ||
      !layout_ok({{B, s.di_batch}, {T, s.di_token}}, D, true))
    return KATA_ERR_INVALID_ARG;
  if (!apart({dx, dr, di, dlam, dr_bias, di_bias, dh_in, workspace},
             {x, r, i, lam, r_bias, i_bias, h_in, lengths, starts, dy, dh_out}))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::recur_workspace_bytes(B, T, D, true)))
    return KATA_ERR_INVALID_ARG;
  a.dy = dy, a.h_in = h_in, a.lengths = lengths, a.dh_out = dh_out, a.dh_in = dh_in;
  a.starts = const_cast<float*>(starts);  // read where they are given
  a.dx = dx, a.dr = dr, a.di = di;
  a.dxb = s.dx_batch, a.dxt = s.dx_token, a.drb = s.dr_batch, a.drt = s.dr_token;
  a.dib = s.di_batch, a.dit = s.di_token;
  return from_hip(
      kata::launch_recur_bwd(a, dlam, dr_bias, di_bias, workspace, dtype == KATA_BF16, stream));
}

kata_status_t kata_recur_step(float* h, const void* x, const void* r, const void* i,
                              const float* lam, const float* r_bias, const float* i_bias, void* y,
                              int B, int D, long long x_batch, long long r_batch,
                              long long i_batch, long long y_batch, float c, kata_dtype_t dtype,
                              hipStream_t stream) {
  const kata_status_t st = recur_check(B, 1, D, c, raw(dtype));
  if (st != KATA_OK) return st;
  kata_recur_strides_t s = {};
  s.x_batch = x_batch, s.r_batch = r_batch, s.i_batch = i_batch, s.y_batch = y_batch;
  kata::RecurArgs a;
  if (!h || !aligned_to(h, 4) || !y || !elem_aligned(y, dtype) ||
      !recur_inputs(a, x, r, i, lam, r_bias, i_bias, B, 1, D, s, c, dtype))
    return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, y_batch}}, D, true)) return KATA_ERR_INVALID_ARG;
  if (!apart({y, h}, {x, r, i, lam, r_bias, i_bias})) return KATA_ERR_INVALID_ARG;
  a.y = y;
  return from_hip(kata::launch_recur_step(h, a, dtype == KATA_BF16, stream));
}

}  // extern "C"
