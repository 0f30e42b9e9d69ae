// kata_mixer_api.hpp -- host side of the mixer operators of kata.h (short
// convolution, query-key norms with rotation, selective scan): argument checks
// and launches.  Included by kata_api.hip, whose helpers it uses.

namespace {

constexpr int kMaxTokens = 1 << 30;
constexpr long long kMaxThreads = (1LL << 32) - 512;  // of a launch, in whole workgroups

struct Dim {
  long long n, stride;
};

// Outer dimensions with their strides, over rows of `inner` elements: offsets
// within bounds, and for an output rows that do not overlap.
template <int K>
bool layout_ok(const Dim (&dims)[K], long long inner, bool output) {
  Dim d[K];
  long long extent = inner;
  for (int i = 0; i < K; ++i) {
    d[i] = dims[i];
    if (d[i].stride < 0 || d[i].stride > kMaxElems) return false;
    if (d[i].n > 1) {
      if (d[i].stride > kMaxElems / (d[i].n - 1)) return false;
      extent += d[i].stride * (d[i].n - 1);
    }
  }
  if (extent > kMaxElems) return false;
  if (!output) return true;
  for (int i = 1; i < K; ++i)  // by stride
    for (int j = i; j > 0 && d[j].stride < d[j - 1].stride; --j) {
      const Dim t = d[j];
      d[j] = d[j - 1];
      d[j - 1] = t;
    }
  extent = inner;
  for (int i = 0; i < K; ++i) {
    if (d[i].n < 2) continue;
    if (d[i].stride < extent) return false;
    extent += d[i].stride * (d[i].n - 1);
  }
  return true;
}

// An enumerator as the number that the caller passed, whatever it is.
template <typename Enum>
int raw(const Enum& e) {
  static_assert(sizeof(Enum) == sizeof(int), "C enumerations are ints here");
  int v;
  std::memcpy(&v, &e, sizeof(v));
  return v;
}
bool type_ok(int dtype) { return dtype == KATA_F32 || dtype == KATA_BF16; }

bool aligned_to(const void* p, unsigned bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1u)) == 0;
}
bool elem_aligned(const void* p, int dtype) { return aligned_to(p, dtype == KATA_BF16 ? 2 : 4); }
// Whether no output stands where an input or another output begins.
bool apart(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* const* o = outs.begin(); o != outs.end(); ++o) {
    if (!*o) continue;
    for (const void* in : ins)
      if (in == *o) return false;
    for (const void* const* other = outs.begin(); other != o; ++other)
      if (*other == *o) return false;
  }
  return true;
}
bool ws_ok(const void* ws, size_t have, size_t need) {
  return ws && aligned_to(ws, 256) && have >= need;
}

// ---- short convolution ------------------------------------------------------------

kata_status_t conv_check(int B, int T, int D, int W, int act, int dtype) {
  if (B < 1 || T < 1 || D < 1 || W < 1) return KATA_ERR_INVALID_ARG;
  if (!type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (act != KATA_CONV_NONE && act != KATA_CONV_SILU) return KATA_ERR_INVALID_ARG;
  if (!product_ok(B, T, D, 1)) return KATA_ERR_INVALID_ARG;
  if (W < 2 || W > 4 || D > (1 << 20) || T > kMaxTokens) return KATA_ERR_UNSUPPORTED;
  // a thread per channel and 16 tokens at the most (runs of four: of few threads)
  if (static_cast<long long>(B) * ((T + 15) / 16) > kMaxThreads / D) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

// ---- norms and rotation -----------------------------------------------------------

kata_status_t norm_check(int B, int T, int Hq, int Hk, int d, int r, int norm, float eps, int pairs,
                         int dtype) {
  if (B < 1 || T < 1 || Hq < 1 || Hk < 0 || d < 1 || r < 0 || r > d || r % 2)
    return KATA_ERR_INVALID_ARG;
  if (!type_ok(dtype)) return KATA_ERR_INVALID_ARG;
  if (norm != KATA_NORM_NONE && norm != KATA_NORM_RMS && norm != KATA_NORM_L2)
    return KATA_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return KATA_ERR_INVALID_ARG;
  if (pairs != 0 && pairs != 1) return KATA_ERR_INVALID_ARG;
  if (static_cast<long long>(Hq) + Hk > kGridYZ || d > 256 || T > kMaxTokens)
    return KATA_ERR_UNSUPPORTED;
  if (!product_ok(B, T, Hq + Hk, d)) return KATA_ERR_INVALID_ARG;
  if (static_cast<long long>(B) * T > kMaxThreads / kata::norm_lanes(d)) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

// The inputs that both directions take.
bool norm_inputs_ok(const void* q, const void* k, const float* wq, const float* wk, const int* pos,
                    const double* freq, int B, int T, int Hq, int Hk, int d, int r,
                    const long long (&s)[6], int dtype) {
  if (!q || !elem_aligned(q, dtype) || (Hk > 0) != (k != nullptr) || (wk && !k)) return false;
  if (k && !elem_aligned(k, dtype)) return false;
  if (!aligned_to(wq, 4) || !aligned_to(wk, 4) || !aligned_to(pos, 4)) return false;
  if ((r > 0) != (freq != nullptr) || !aligned_to(freq, 8)) return false;
  if (!layout_ok({{B, s[0]}, {T, s[1]}, {Hq, s[2]}}, d, false)) return false;
  return !k || layout_ok({{B, s[3]}, {T, s[4]}, {Hk, s[5]}}, d, false);
}

kata::NormArgs norm_args(int B, int T, int Hq, int Hk, int d, int r, const long long (&s)[6],
                         int norm, float eps, int pairs) {
  kata::NormArgs n = {};
  n.side[0] = {s[0], s[1], s[2], Hq};
  if (Hk > 0) n.side[1] = {s[3], s[4], s[5], Hk};
  n.B = B, n.T = T, n.d = d, n.r = r, n.norm = norm, n.pairs = pairs, n.eps = eps;
  return n;
}

// ---- selective scan ---------------------------------------------------------------

kata_status_t ssm_check(int B, int T, int H, int G, int N, int P, int softplus, int dtype,
                        bool backward) {
  if (B < 1 || T < 1 || H < 1 || G < 1 || N < 1 || P < 1 || H % G) return KATA_ERR_INVALID_ARG;
  if (!type_ok(dtype) || (softplus != 0 && softplus != 1)) return KATA_ERR_INVALID_ARG;
  if (!product_ok(B, T, H, N > P ? N : P)) return KATA_ERR_INVALID_ARG;
  if (N > 128 || P > 256 || static_cast<long long>(B) * H > kGridYZ || T > kMaxTokens)
    return KATA_ERR_UNSUPPORTED;
  // per chunk of 32 tokens or more: a wave per head, and in the backward up to eight per group
  const long long chunks = static_cast<long long>(B) * (T / (dtype == KATA_BF16 ? 64 : 32) + 1);
  if (chunks > kMaxThreads / ((H + 3) / 4 * 256)) return KATA_ERR_UNSUPPORTED;
  if (backward && chunks > kMaxThreads / (G * 512LL)) return KATA_ERR_UNSUPPORTED;
  return KATA_OK;
}

kata_ssm_strides_t ssm_contiguous(int T, int H, int G, int N, int P) {
  const long long t = T, h = H, g = G, n = N, p = P;
  return {t * h * p, h * p, p, t * h,     h,     1, t * g * n, g * n,
          n,         t * g * n, g * n, n, t * h * p, h * p, p};
}

// y: the output, or null; dy: the backward's input, or null.
bool ssm_tensors(kata::SsmArgs& a, const void* x, const void* dt, const float* A, const void* Bm,
                 const void* Cm, const float* D, const float* bias, const void* dy, void* y, int B,
                 int T, int H, int G, int N, int P, const kata_ssm_strides_t* strides, int softplus,
                 int dtype) {
  for (const void* p : {x, dt, Bm, Cm})
    if (!p || !elem_aligned(p, dtype)) return false;
  if (!A || !aligned_to(A, 4) || !aligned_to(D, 4) || !aligned_to(bias, 4)) return false;
  if ((!y && !dy) || !elem_aligned(y, dtype) || !elem_aligned(dy, dtype)) return false;
  const kata_ssm_strides_t s = strides ? *strides : ssm_contiguous(T, H, G, N, P);
  if (!layout_ok({{B, s.x_batch}, {T, s.x_token}, {H, s.x_head}}, P, false)) return false;
  if (!layout_ok({{B, s.dt_batch}, {T, s.dt_token}, {H, s.dt_head}}, 1, false)) return false;
  if (!layout_ok({{B, s.b_batch}, {T, s.b_token}, {G, s.b_group}}, N, false)) return false;
  if (!layout_ok({{B, s.c_batch}, {T, s.c_token}, {G, s.c_group}}, N, false)) return false;
  if (!layout_ok({{B, s.y_batch}, {T, s.y_token}, {H, s.y_head}}, P, y != nullptr)) return false;
  const int piece = dtype == KATA_BF16 ? 8 : 4;
  const auto pieces = [piece](const void* p, int cols, long long u, long long v, long long w) {
    return aligned_to(p, 16) && cols % piece == 0 && u % piece == 0 && v % piece == 0 &&
           w % piece == 0 && v <= 1 << 21 && v >= cols;  // (also of one token: its rows end there)
  };
  a = {};
  a.x = x, a.dt = dt, a.A = A, a.Bm = Bm, a.Cm = Cm, a.D = D, a.bias = bias, a.dy = dy, a.y = y;
  a.B = B, a.T = T, a.H = H, a.G = G, a.N = N, a.P = P, a.softplus = softplus;
  a.xb = s.x_batch, a.xt = s.x_token, a.xh = s.x_head;
  a.db = s.dt_batch, a.dt_t = s.dt_token, a.dh = s.dt_head;
  a.bb = s.b_batch, a.bt = s.b_token, a.bg = s.b_group;
  a.cb = s.c_batch, a.ct = s.c_token, a.cg = s.c_group;
  a.yb = s.y_batch, a.yt = s.y_token, a.yh = s.y_head;
  a.vec = pieces(x, P, a.xb, a.xt, a.xh) && pieces(Bm, N, a.bb, a.bt, a.bg) &&
          pieces(Cm, N, a.cb, a.ct, a.cg) && pieces(y ? y : dy, P, a.yb, a.yt, a.yh);
  return true;
}

}  // namespace

extern "C" {

kata_status_t kata_conv_fwd(const void* x, const float* w, const float* bias, const void* state_in,
                            const int* lengths, void* y, void* state_out, int B, int T, int D,
                            int W, long long x_batch, long long x_token, long long y_batch,
                            long long y_token, kata_conv_act_t act, kata_dtype_t dtype,
                            hipStream_t stream) {
  if (!x || !w || !y) return KATA_ERR_INVALID_ARG;
  const kata_status_t c = conv_check(B, T, D, W, raw(act), raw(dtype));
  if (c != KATA_OK) return c;
  for (const void* p : {x, state_in, static_cast<const void*>(y), static_cast<const void*>(state_out)})
    if (!elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  if (!aligned_to(w, 4) || !aligned_to(bias, 4) || !aligned_to(lengths, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({y, state_out}, {x, w, bias, state_in, lengths})) return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, x_batch}, {T, x_token}}, D, false) ||
      !layout_ok({{B, y_batch}, {T, y_token}}, D, true))
    return KATA_ERR_INVALID_ARG;
  const kata::ConvShape s = {B, T, D, act == KATA_CONV_SILU, x_batch, x_token, y_batch, y_token, 0, 0};
  return from_hip(kata::launch_conv_fwd(x, w, bias, state_in, lengths, y, state_out, s, W,
                                        dtype == KATA_BF16, stream));
}

kata_status_t kata_conv_step(void* state, const void* x, const float* w, const float* bias, void* y,
                             int B, int D, int W, long long x_batch, long long y_batch,
                             kata_conv_act_t act, kata_dtype_t dtype, hipStream_t stream) {
  if (!state || !x || !w || !y) return KATA_ERR_INVALID_ARG;
  const kata_status_t c = conv_check(B, 1, D, W, raw(act), raw(dtype));
  if (c != KATA_OK) return c;
  for (const void* p : {x, static_cast<const void*>(state), static_cast<const void*>(y)})
    if (!elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  if (!aligned_to(w, 4) || !aligned_to(bias, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({y, state}, {x, w, bias})) return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, x_batch}}, D, false) || !layout_ok({{B, y_batch}}, D, true))
    return KATA_ERR_INVALID_ARG;
  const kata::ConvShape s = {B, 1, D, act == KATA_CONV_SILU, x_batch, 0, y_batch, 0, 0, 0};
  return from_hip(kata::launch_conv_step(state, x, w, bias, y, s, W, dtype == KATA_BF16, stream));
}

size_t kata_conv_bwd_workspace_bytes(int B, int T, int D, int W, kata_dtype_t dtype) {
  if (conv_check(B, T, D, W, KATA_CONV_NONE, raw(dtype)) != KATA_OK) return 0;
  return kata::conv_bwd_workspace_bytes(B, T, D, W);
}

kata_status_t kata_conv_bwd_ws(const void* x, const float* w, const float* bias, const void* dy,
                               void* dx, float* dw, float* dbias, int B, int T, int D, int W,
                               long long x_batch, long long x_token, long long dy_batch,
                               long long dy_token, long long dx_batch, long long dx_token,
                               kata_conv_act_t act, kata_dtype_t dtype, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
  if (!x || !w || !dy || !dx) return KATA_ERR_INVALID_ARG;
  const kata_status_t c = conv_check(B, T, D, W, raw(act), raw(dtype));
  if (c != KATA_OK) return c;
  for (const void* p : {x, dy, static_cast<const void*>(dx)})
    if (!elem_aligned(p, dtype)) return KATA_ERR_INVALID_ARG;
  for (const float* p : {w, bias, static_cast<const float*>(dw), static_cast<const float*>(dbias)})
    if (!aligned_to(p, 4)) return KATA_ERR_INVALID_ARG;
  if (!apart({dx, dw, dbias, workspace}, {x, w, bias, dy})) return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, x_batch}, {T, x_token}}, D, false) ||
      !layout_ok({{B, dy_batch}, {T, dy_token}}, D, false) ||
      !layout_ok({{B, dx_batch}, {T, dx_token}}, D, true))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::conv_bwd_workspace_bytes(B, T, D, W)))
    return KATA_ERR_INVALID_ARG;
  const kata::ConvShape s = {B,        T,        D,        act == KATA_CONV_SILU, x_batch,
                             x_token,  dx_batch, dx_token, dy_batch,              dy_token};
  return from_hip(kata::launch_conv_bwd(x, w, bias, dy, dx, dw, dbias, workspace, s, W,
                                        dtype == KATA_BF16, stream));
}

kata_status_t kata_qk_norm_fwd(const void* q, const void* k, const float* wq, const float* wk,
                               const int* pos, const double* freq, void* yq, void* yk, int B, int T,
                               int Hq, int Hk, int d, int r, long long q_batch, long long q_token,
                               long long q_head, long long k_batch, long long k_token,
                               long long k_head, kata_norm_t norm, float eps, int pairs,
                               kata_dtype_t dtype, hipStream_t stream) {
  const kata_status_t c = norm_check(B, T, Hq, Hk, d, r, raw(norm), eps, pairs, raw(dtype));
  if (c != KATA_OK) return c;
  const long long s[6] = {q_batch, q_token, q_head, k_batch, k_token, k_head};
  if (!norm_inputs_ok(q, k, wq, wk, pos, freq, B, T, Hq, Hk, d, r, s, dtype))
    return KATA_ERR_INVALID_ARG;
  if (!yq || !elem_aligned(yq, dtype) || (Hk > 0) != (yk != nullptr)) return KATA_ERR_INVALID_ARG;
  if (yk && !elem_aligned(yk, dtype)) return KATA_ERR_INVALID_ARG;
  if (!apart({yq, yk}, {q, k, wq, wk, pos, freq})) return KATA_ERR_INVALID_ARG;
  return from_hip(kata::launch_qk_norm_fwd(q, k, wq, wk, pos, freq, yq, yk,
                                           norm_args(B, T, Hq, Hk, d, r, s, norm, eps, pairs),
                                           dtype == KATA_BF16, stream));
}

size_t kata_qk_norm_bwd_workspace_bytes(int B, int T, int Hq, int Hk, int d, kata_dtype_t dtype) {
  if (norm_check(B, T, Hq, Hk, d, 0, KATA_NORM_NONE, 0.f, 0, raw(dtype)) != KATA_OK) return 0;
  return kata::norm_bwd_workspace_bytes(B, T, Hq + Hk, d);
}

kata_status_t kata_qk_norm_bwd_ws(
    const void* q, const void* k, const float* wq, const float* wk, const int* pos,
    const double* freq, const void* dq, const void* dk, void* dxq, void* dxk, float* dwq,
    float* dwk, int B, int T, int Hq, int Hk, int d, int r, long long q_batch, long long q_token,
    long long q_head, long long k_batch, long long k_token, long long k_head, long long dxq_batch,
    long long dxq_token, long long dxq_head, long long dxk_batch, long long dxk_token,
    long long dxk_head, kata_norm_t norm, float eps, int pairs, kata_dtype_t dtype,
    kata_dtype_t dy_dtype, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const kata_status_t c = norm_check(B, T, Hq, Hk, d, r, raw(norm), eps, pairs, raw(dtype));
  if (c != KATA_OK) return c;
  if (!type_ok(raw(dy_dtype))) return KATA_ERR_INVALID_ARG;
  if (dy_dtype == KATA_BF16 && dtype != KATA_BF16) return KATA_ERR_UNSUPPORTED;
  const long long s[6] = {q_batch, q_token, q_head, k_batch, k_token, k_head};
  if (!norm_inputs_ok(q, k, wq, wk, pos, freq, B, T, Hq, Hk, d, r, s, dtype))
    return KATA_ERR_INVALID_ARG;
  const bool keys = Hk > 0;
  if (!dq || !elem_aligned(dq, dy_dtype) || keys != (dk != nullptr) || !elem_aligned(dk, dy_dtype))
    return KATA_ERR_INVALID_ARG;
  if (!dxq || !elem_aligned(dxq, dtype) || keys != (dxk != nullptr) || !elem_aligned(dxk, dtype))
    return KATA_ERR_INVALID_ARG;
  if (!aligned_to(dwq, 4) || !aligned_to(dwk, 4) || (dwk && !keys)) return KATA_ERR_INVALID_ARG;
  if (!apart({dxq, dxk, dwq, dwk, workspace}, {q, k, wq, wk, pos, freq, dq, dk}))
    return KATA_ERR_INVALID_ARG;
  if (!layout_ok({{B, dxq_batch}, {T, dxq_token}, {Hq, dxq_head}}, d, true)) return KATA_ERR_INVALID_ARG;
  if (keys && !layout_ok({{B, dxk_batch}, {T, dxk_token}, {Hk, dxk_head}}, d, true))
    return KATA_ERR_INVALID_ARG;
  if (!ws_ok(workspace, workspace_bytes, kata::norm_bwd_workspace_bytes(B, T, Hq + Hk, d)))
    return KATA_ERR_INVALID_ARG;
  const kata::NormSide oq = {dxq_batch, dxq_token, dxq_head, Hq};
  kata::NormSide ok = {};
  if (keys) ok = {dxk_batch, dxk_token, dxk_head, Hk};
  return from_hip(kata::launch_qk_norm_bwd(q, k, wq, wk, pos, freq, dq, dk, dxq, dxk, dwq, dwk,
                                           workspace,
                                           norm_args(B, T, Hq, Hk, d, r, s, norm, eps, pairs), oq,
                                           ok, dtype == KATA_BF16, dy_dtype == KATA_BF16, stream));
}

size_t kata_ssm_workspace_bytes(int B, int T, int H, int G, int N, int P, kata_dtype_t dtype,
                                int backward) {
  if (ssm_check(B, T, H, G, N, P, 1, raw(dtype), backward != 0) != KATA_OK) return 0;
  return kata::ssm_workspace_bytes(B, T, H, G, N, P, dtype == KATA_BF16, backward != 0);
}

kata_status_t kata_ssm_fwd_ws(const void* x, const void* dt, const float* A, const void* Bm,
                              const void* Cm, const float* D, const float* dt_bias,
                              const float* S_in, const int* lengths, void* y, float* S_out, int B,
                              int T, int H, int G, int N, int P, const kata_ssm_strides_t* strides,
                              int softplus, kata_dtype_t dtype, void* workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  const kata_status_t c = ssm_check(B, T, H, G, N, P, softplus, raw(dtype), false);
  if (c != KATA_OK) return c;
  kata::SsmArgs a;
  if (!y || !ssm_tensors(a, x, dt, A, Bm, Cm, D, dt_bias, nullptr, y, B, T, H, G, N, P, strides,
                         softplus, dtype))
    return KATA_ERR_INVALID_ARG;
  if (!apart({y, S_out, workspace}, {x, dt, A, Bm, Cm, D, dt_bias, S_in, lengths}))
    return KATA_ERR_INVALID_ARG;
  if (!aligned16(S_in) || !aligned16(S_out) || !aligned_to(lengths, 4)) return KATA_ERR_INVALID_ARG;
  const bool bf16 = dtype == KATA_BF16;
  if (!ws_ok(workspace, workspace_bytes,
             kata::ssm_workspace_bytes(B, T, H, G, N, P, bf16, false)))
    return KATA_ERR_INVALID_ARG;
  a.S_in = S_in, a.S_out = S_out, a.lengths = lengths;
  return from_hip(kata::launch_ssm_fwd(a, workspace, bf16, stream));
}

kata_status_t kata_ssm_bwd_ws(const void* x, const void* dt, const float* A, const void* Bm,
                              const void* Cm, const float* D, const float* dt_bias, const void* dy,
                              void* dx, void* ddt, float* dA, void* dBm, void* dCm, float* dD,
                              float* dt_dbias, int B, int T, int H, int G, int N, int P,
                              const kata_ssm_strides_t* strides, int softplus, kata_dtype_t dtype,
                              void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const kata_status_t c = ssm_check(B, T, H, G, N, P, softplus, raw(dtype), true);
  if (c != KATA_OK) return c;
  kata::SsmArgs a;
  if (!dy || !ssm_tensors(a, x, dt, A, Bm, Cm, D, dt_bias, dy, nullptr, B, T, H, G, N, P, strides,
                          softplus, dtype))
    return KATA_ERR_INVALID_ARG;
  for (const void* out : {static_cast<const void*>(dx), static_cast<const void*>(ddt),
                          static_cast<const void*>(dBm), static_cast<const void*>(dCm)}) {
    if (!out || !elem_aligned(out, dtype)) return KATA_ERR_INVALID_ARG;
  }
  if (!apart({dx, ddt, dA, dBm, dCm, dD, dt_dbias, workspace}, {x, dt, A, Bm, Cm, D, dt_bias, dy}))
    return KATA_ERR_INVALID_ARG;
  if (!aligned_to(dA, 4) || !aligned_to(dD, 4) || !aligned_to(dt_dbias, 4))
    return KATA_ERR_INVALID_ARG;
  const bool bf16 = dtype == KATA_BF16;
  a.vec = a.vec && aligned16(dx) && aligned16(dBm) && aligned16(dCm);
  if (!ws_ok(workspace, workspace_bytes, kata::ssm_workspace_bytes(B, T, H, G, N, P, bf16, true)))
    return KATA_ERR_INVALID_ARG;
  return from_hip(kata::launch_ssm_bwd(a, dx, ddt, dA, dBm, dCm, dD, dt_dbias, workspace, bf16,
                                       stream));
}

kata_status_t kata_ssm_step(float* S, const void* x, const void* dt, const float* A, const void* Bm,
                            const void* Cm, const float* D, const float* dt_bias, void* y, int B,
                            int H, int G, int N, int P, const kata_ssm_strides_t* strides,
                            int softplus, kata_dtype_t dtype, hipStream_t stream) {
  const kata_status_t c = ssm_check(B, 1, H, G, N, P, softplus, raw(dtype), false);
  if (c != KATA_OK) return c;
  kata::SsmArgs a;
  kata_ssm_strides_t s = strides ? *strides : ssm_contiguous(1, H, G, N, P);
  s.x_token = s.dt_token = s.b_token = s.c_token = s.y_token = 0;  // not the caller's: may be anything
  if (!S || !aligned16(S) || !y ||
      !ssm_tensors(a, x, dt, A, Bm, Cm, D, dt_bias, nullptr, y, B, 1, H, G, N, P, &s, softplus, dtype))
    return KATA_ERR_INVALID_ARG;
  if (!apart({y, S}, {x, dt, A, Bm, Cm, D, dt_bias})) return KATA_ERR_INVALID_ARG;
  return from_hip(kata::launch_ssm_step(S, a, dtype == KATA_BF16, stream));
}

}  // extern "C"
