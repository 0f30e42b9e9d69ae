/*
 * kata.h -- C ABI of libkata: causal KATA-M1 attention (rank-one PSD feature
 * map), and its block-diagonal KATA-Mg variant, on AMD Instinct MI355X (gfx950).
 *
 * The operation.  For every head, with query q_t, key k_t in R^d and value v_t
 * in R^dv, the feature map is the rank-one PSD lift phi(x) = vec(x x^T)
 * (section "Rank-one packing into the PSD cone"), whose inner product is
 * <phi(q), phi(k)> = (q . k)^2.  Normalised causal linear attention
 * (eq. linatt) with this map gives
 *
 *     o_t = sum_{i<=t} (q_t . k_i)^2 v_i  /  sum_{i<=t} (q_t . k_i)^2 ,
 *
 * a convex combination of the values (output-gate proposition).  A row whose
 * denominator is 0 (q_t orthogonal to every k_i, i <= t, e.g. q_t = 0) is
 * defined as all zeros; the paper leaves it undefined.
 *
 * Conventions shared by every entry point:
 *  - Tensors are contiguous, row-major, device-resident (HBM), 16-byte aligned:
 *      q, k : [B][H][T][d]     v : [B][H][T][dv]     out : [B][H][T][dv] fp32.
 *    q, k, v are fp32 or bf16 (kata_dtype_t); out, S and z are always fp32.
 *  - The caller owns every buffer.  `out` must not alias an input.
 *  - Every call validates its arguments on the host before touching the GPU;
 *    on an error nothing is launched and nothing is written.
 *  - Calls only enqueue work on `stream` and return; they never synchronise.
 *    A device fault surfaces at the caller's next synchronisation.
 *  - The calls that take a caller workspace (the _ws and _timed variants),
 *    kata_fwd_chunked_noalloc, kata_prefill_state and kata_decode_step
 *    enqueue kernel launches only (and the _timed variants event records), so
 *    a caller may capture them into a HIP graph and replay it; the variants
 *    without a workspace argument allocate theirs stream-ordered
 *    (hipMallocAsync / hipFreeAsync) on `stream`.
 *  - The library keeps no global mutable state (except the scratch array of
 *    kata_fwd_chunked_noalloc, see there); calls from several threads are
 *    safe.  NaN and Inf in inputs propagate; inputs are not normalised.
 *  - Packed state layout (decode and prefill): the n = d(d+1)/2 features of
 *    the pair (a, b), a <= b, in row-major upper-triangle order,
 *        f(a, b) = a*d - a*(a-1)/2 + (b - a),
 *    S : [B][H][n][dv] holds sum_i k_a k_b v_i (unscaled), z : [B][H][n]
 *    holds sum_i k_a k_b.
 */
#ifndef KATA_H
#define KATA_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>

#ifndef KATA_API
#define KATA_API __attribute__((visibility("default")))
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  KATA_OK = 0,
  KATA_ERR_INVALID_ARG = 1, /* null pointer, size < 1, or a size product overflows */
  KATA_ERR_UNSUPPORTED = 2, /* valid arguments outside what is implemented */
  KATA_ERR_HIP = 3          /* a HIP launch or allocation failed */
} kata_status_t;

typedef enum { KATA_F32 = 0, KATA_BF16 = 1 } kata_dtype_t;

/*
 * Causal KATA-M1 forward in the exact O(T) chunked-state form (eq. chunk-SZ,
 * eq. chunk-out and the chunkwise algorithm of the appendix; the three-stage
 * state / associative-scan / output pipeline of the tree-scan section).
 * The final chunk is zero-padded on chip and the output is truncated to T rows.
 *   q, k, v, out : see the conventions above.
 *   B, H, T >= 1.  d in 1..64.  dv >= 1.  C >= 1 is the chunk size.
 *   Fast path (bf16 MFMA): dtype = KATA_BF16, d in {32, 64}, dv = 64,
 *   C a multiple of 32 up to 1024.  Every other shape with d <= 64, dv <= 256
 *   and C <= 128 runs on the fp32 path (with g = 1 in the quadratic form where
 *   that is faster: kata_fwd_form); anything else is KATA_ERR_UNSUPPORTED.
 *   Workspace (kata_fwd_workspace_bytes) is allocated stream-ordered with
 *   hipMallocAsync on `stream` and released with hipFreeAsync.
 */
KATA_API kata_status_t kata_fwd_chunked(const void* q, const void* k, const void* v, float* out,
                               int B, int H, int T, int d, int dv, int C,
                               kata_dtype_t dtype, hipStream_t stream);

/*
 * kata_fwd_chunked for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, default span and results as kata_fwd_chunked; it calls no
 * hipMalloc / hipFree or allocating library routine.  Its workspace is a
 * library-owned device array of kata_noalloc_scratch_bytes() bytes (256 MiB),
 * one per GPU, held by every GPU the library runs on until the process ends;
 * the first call on a device looks up that device's copy (the stream's device;
 * the current device for the null stream).
 *   Returns KATA_ERR_UNSUPPORTED when the workspace kata_fwd_chunked would
 *   allocate (kata_fwd_workspace_bytes at the default span) exceeds the array,
 *   e.g. B*H*T above about 650k head-tokens at d = dv = 64 on the bf16 path.
 *   Every call on one GPU shares that GPU's array and leaves its contents
 *   behind: calls that overlap on one GPU (different streams, or host
 *   threads) race and give undefined results.  No kernel reads scratch that
 *   the same call has not written, so nothing is cleared between calls.
 */
KATA_API kata_status_t kata_fwd_chunked_noalloc(const void* q, const void* k, const void* v,
                                                float* out, int B, int H, int T, int d, int dv,
                                                int C, kata_dtype_t dtype, hipStream_t stream);

/* Size in bytes of the per-device scratch array of kata_fwd_chunked_noalloc. */
KATA_API size_t kata_noalloc_scratch_bytes(void);

/*
 * The same forward with caller-provided workspace and an explicit span.
 *   span_chunks : number of chunks folded into one stored state (the state
 *                 written to HBM covers span_chunks*C tokens; the chunks inside
 *                 a span are combined on chip).  0 selects the default
 *                 (kata_fwd_default_span; on the fast path, sequences short
 *                 enough for it to be the faster form are evaluated
 *                 quadratically, with no stored state: kata_fwd_form).  1 is the
 *                 per-chunk form.  Results do not depend on it beyond rounding.
 *   workspace   : device buffer of at least kata_fwd_workspace_bytes(...)
 *                 bytes, 256-byte aligned, owned by the caller, contents
 *                 ignored on entry and undefined on exit.  Two calls in flight
 *                 at once must not share it.
 */
KATA_API kata_status_t kata_fwd_chunked_ws(const void* q, const void* k, const void* v, float* out,
                                  int B, int H, int T, int d, int dv, int C,
                                  kata_dtype_t dtype, int span_chunks, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream);

/*
 * kata_fwd_chunked_ws plus stage timing, for profiling: stage_events[0..3]
 * (caller-created HIP events, all non-null) are recorded on `stream` before the
 * state kernel and after each of the three stages (chunk or span state,
 * associative scan, output; the first two are empty in the quadratic form).
 * Nothing synchronises; the caller reads the elapsed times with
 * hipEventElapsedTime once the stream has reached them.
 */
KATA_API kata_status_t kata_fwd_chunked_timed(const void* q, const void* k, const void* v,
                                              float* out, int B, int H, int T, int d, int dv,
                                              int C, kata_dtype_t dtype, int span_chunks,
                                              void* workspace, size_t workspace_bytes,
                                              hipEvent_t* stage_events, hipStream_t stream);

/*
 * kata_fwd_chunked_ws for a training step: it also writes each row's
 * denominator D_t = sum_{i<=t} (q_t . k_i)^2 (the normaliser of eq. linatt,
 * fp32 as the forward computed it) to den, fp32 [B][H][T], caller-owned,
 * 16-byte aligned, for kata_bwd_chunked_ex, which then need not form it again
 * from the prefix states.  Supported on the bf16 MFMA path (the shapes of
 * kata_fwd_chunked_ws with dtype KATA_BF16, d in {32, 64}, dv = 64, C a
 * multiple of 32); other valid arguments give KATA_ERR_UNSUPPORTED.  den null:
 * KATA_ERR_INVALID_ARG.
 */
KATA_API kata_status_t kata_fwd_chunked_train_ws(const void* q, const void* k, const void* v,
                                                 float* out, float* den, int B, int H, int T,
                                                 int d, int dv, int C, kata_dtype_t dtype,
                                                 int span_chunks, void* workspace,
                                                 size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes kata_fwd_chunked_ws needs for these arguments (0 when the
 * arguments are invalid or unsupported). */
KATA_API size_t kata_fwd_workspace_bytes(int B, int H, int T, int d, int dv, int C,
                                kata_dtype_t dtype, int span_chunks);

/* The span (in chunks) that span_chunks = 0 selects for these arguments where
 * kata_fwd_form(..., 0) is KATA_FWD_STATES; it also sizes the workspace where it
 * is not. */
KATA_API int kata_fwd_default_span(int B, int H, int T, int d, int dv, int C, kata_dtype_t dtype);

/* The form in which a forward of these arguments runs (g = 1: kata_fwd_chunked*,
 * whose entry points without a span leave it 0; else kata_mg_fwd_chunked*): span or
 * chunk states, or the quadratic form.  -1 where the arguments are invalid or
 * unsupported. */
enum { KATA_FWD_STATES = 0, KATA_FWD_QUADRATIC = 1 };
KATA_API int kata_fwd_form(int B, int H, int T, int d, int dv, int C, int g, kata_dtype_t dtype,
                           int span_chunks);

/*
 * The same causal KATA-M1 forward in the quadratic (flash-style) form: the
 * O(T^2) definition above evaluated in 32x32 query-key blocks on chip
 * (squared scores, causal mask, P V and the row sums), never forming a
 * feature state (section "Synthetic induction and hardware microbenchmarks",
 * paragraph "Kernel latency and throughput ratios": the quadratic operating
 * point, preferable to the O(T) form at short T).  Same outputs as
 * kata_fwd_chunked up to rounding.
 *   Supported: dtype = KATA_BF16, d in {32, 64}, dv = 64 (bf16 MFMA);
 *   other valid arguments give KATA_ERR_UNSUPPORTED.  B*H <= 65535.
 *   workspace : device buffer of at least kata_fwd_quadratic_workspace_bytes(...)
 *               bytes, 256-byte aligned, caller-owned (checked, but unused since
 *               no copy of V is made any more).
 * kata_fwd_quadratic allocates that workspace stream-ordered (hipMallocAsync /
 * hipFreeAsync on `stream`).
 */
KATA_API kata_status_t kata_fwd_quadratic(const void* q, const void* k, const void* v, float* out,
                                          int B, int H, int T, int d, int dv,
                                          kata_dtype_t dtype, hipStream_t stream);
KATA_API kata_status_t kata_fwd_quadratic_ws(const void* q, const void* k, const void* v,
                                             float* out, int B, int H, int T, int d, int dv,
                                             kata_dtype_t dtype, void* workspace,
                                             size_t workspace_bytes, hipStream_t stream);
/* Workspace bytes kata_fwd_quadratic_ws needs (0 when the arguments are
 * invalid or unsupported). */
KATA_API size_t kata_fwd_quadratic_workspace_bytes(int B, int H, int T, int d, int dv,
                                                   kata_dtype_t dtype);

/*
 * State after T tokens by the additive recurrence of eq. linatt:
 *   S = sum_{t<T} phi(k_t) v_t^T,  z = sum_{t<T} phi(k_t)   (packed layout above).
 * Overwrites S : [B][H][n][dv] and z : [B][H][n] (fp32).  Products k_a k_b and
 * the sums are formed in fp32.  Bridges a prefill to kata_decode_step.
 *   k, v : [B][H][T][d], [B][H][T][dv];  d in 1..64, dv in 1..256.
 */
KATA_API kata_status_t kata_prefill_state(const void* k, const void* v, float* S, float* z,
                                 int B, int H, int T, int d, int dv,
                                 kata_dtype_t dtype, hipStream_t stream);

/*
 * One recurrent decode step for all B*H heads (eq. linatt's recurrence and its
 * normalised readout, using the updated state so the current token counts, as
 * in the forward):
 *   S <- S + phi(k) v^T,  z <- z + phi(k),  out = phi(q)^T S / phi(q)^T z.
 *   S : [B][H][n][dv] fp32 and z : [B][H][n] fp32, updated in place (packed
 *       layout above; caller-owned, so a failed step can be retried from the
 *       caller's copy).
 *   q, k : [B][H][d], v : [B][H][dv] in `dtype`;  out : [B][H][dv] fp32.
 *   d in 1..64, dv in 1..256.  State arithmetic is fp32.
 */
KATA_API kata_status_t kata_decode_step(float* S, float* z, const void* q, const void* k,
                               const void* v, float* out, int B, int H, int d, int dv,
                               kata_dtype_t dtype, hipStream_t stream);

/*
 * KATA-Mg, the block-diagonal PSD feature (section "From rank-one rays to
 * low-rank PSD packing").  Each query and key is split into g blocks of
 * m = d/g consecutive coordinates, u = (u_1, ..., u_g), and the feature keeps
 * one rank-one factor per block, psi(u) = (u_1 u_1^T, ..., u_g u_g^T), so
 *
 *     o_t = sum_{i<=t} w_ti v_i / sum_{i<=t} w_ti,   w_ti = sum_a (q_{t,a} . k_{i,a})^2 .
 *
 * g = 1 is KATA-M1 (the calls above).  g >= 1 must divide d, else
 * KATA_ERR_INVALID_ARG.  Packed state layout (prefill, decode): n = g*m(m+1)/2
 * features; block a's pair (i, j), i <= j < m, at a*m(m+1)/2 + f_m(i, j)
 * (the M1 order over m coordinates); S : [B][H][n][dv], z : [B][H][n].
 * Forward fast path (bf16 MFMA): dtype = KATA_BF16, dv = 64, C a multiple of
 * 32 up to 1024 and (d, g) in {(64, 1), (64, 2), (32, 1)}; other shapes with
 * d <= 64, dv <= 256 and C <= 128 run on the fp32 path.  The quadratic form
 * exists on the fast path only.  Arguments, workspace ownership, errors and
 * asynchrony otherwise as for the M1 call of the same name.
 */
KATA_API kata_status_t kata_mg_fwd_chunked(const void* q, const void* k, const void* v,
                                           float* out, int B, int H, int T, int d, int dv, int C,
                                           int g, kata_dtype_t dtype, hipStream_t stream);
KATA_API kata_status_t kata_mg_fwd_chunked_ws(const void* q, const void* k, const void* v,
                                              float* out, int B, int H, int T, int d, int dv,
                                              int C, int g, kata_dtype_t dtype, int span_chunks,
                                              void* workspace, size_t workspace_bytes,
                                              hipStream_t stream);
KATA_API kata_status_t kata_mg_fwd_chunked_timed(const void* q, const void* k, const void* v,
                                                 float* out, int B, int H, int T, int d, int dv,
                                                 int C, int g, kata_dtype_t dtype,
                                                 int span_chunks, void* workspace,
                                                 size_t workspace_bytes,
                                                 hipEvent_t* stage_events, hipStream_t stream);
KATA_API size_t kata_mg_fwd_workspace_bytes(int B, int H, int T, int d, int dv, int C, int g,
                                            kata_dtype_t dtype, int span_chunks);
KATA_API kata_status_t kata_mg_fwd_quadratic_ws(const void* q, const void* k, const void* v,
                                                float* out, int B, int H, int T, int d, int dv,
                                                int g, kata_dtype_t dtype, void* workspace,
                                                size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_mg_fwd_quadratic_workspace_bytes(int B, int H, int T, int d, int dv, int g,
                                                      kata_dtype_t dtype);
KATA_API kata_status_t kata_mg_prefill_state(const void* k, const void* v, float* S, float* z,
                                             int B, int H, int T, int d, int dv, int g,
                                             kata_dtype_t dtype, hipStream_t stream);
KATA_API kata_status_t kata_mg_decode_step(float* S, float* z, const void* q, const void* k,
                                           const void* v, float* out, int B, int H, int d, int dv,
                                           int g, kata_dtype_t dtype, hipStream_t stream);

/*
 * Causal linear attention with a linear (n_psi ~ d) feature map: the orthant
 * maps and the Lorentz lift of section "Classical feature maps", the n_psi = d
 * Lorentz variant of the appendix KATA-Lorentz model, and the plain feature
 * psi(x) = x of the associative-scan measurements (appendix "Associative-scan
 * kernel", table of small-batch associative-scan throughput).  With
 * w_ti = <psi(q_t), psi(k_i)>:
 *     normalize = 1:  o_t = sum_{i<=t} w_ti v_i / sum_{i<=t} w_ti   (eq. linatt),
 *                     and o_t = 0 when the denominator is not positive;
 *     normalize = 0:  o_t = sum_{i<=t} w_ti v_i  (unnormalised; the usual
 *                     choice for KATA_LIN_IDENTITY, whose weights carry a sign).
 * Computed in the three-stage chunk-state / associative-scan / chunk-output
 * form (paragraph "Three-kernel pipeline" of that appendix).
 *   feature : a kata_lin_feature_t; eps (>= 0, finite) is used by
 *             KATA_LIN_RELU only.  n_psi = kata_lin_dim(d, feature).
 *   Fast path (bf16 MFMA): dtype = KATA_BF16, d = dv = 64, every feature, C a
 *   multiple of 64 up to 1024 (KATA_LIN_LORENTZ's extra coordinate ||x|| is
 *   carried as a rank-one fp32 term beside the d x d MFMA state).  Every
 *   other shape with d <= 64, dv <= 256 and C <= 128 runs on the fp32 path;
 *   anything else is KATA_ERR_UNSUPPORTED.
 *   span_chunks, workspace, stage_events: as for kata_fwd_chunked_ws and
 *   kata_fwd_chunked_timed (records of span_chunks * C tokens on the fast
 *   path; one per chunk on the fp32 path).  Tensors, ownership, errors and
 *   asynchrony as in the conventions at the top of this file.
 */
typedef enum {
  KATA_LIN_IDENTITY = 0,  /* psi(x) = x                                  n_psi = d     */
  KATA_LIN_RELU = 1,      /* psi(x) = ReLU(x) + eps                      n_psi = d     */
  KATA_LIN_ELU = 2,       /* psi(x) = ELU(x) + 1                         n_psi = d     */
  KATA_LIN_LORENTZ = 3,   /* psi(x) = (x, ||x||_2)                       n_psi = d + 1 */
  KATA_LIN_LORENTZ_S = 4  /* psi(x) = (y, ||y||_2 (1 + s^2)), y = x_1..x_{d-1},
                             s = x_d                                     n_psi = d     */
} kata_lin_feature_t;

/* n_psi of a feature at width d (0 when d < 1 or the feature is unknown). */
KATA_API int kata_lin_dim(int d, kata_lin_feature_t feature);
KATA_API kata_status_t kata_lin_fwd_chunked(const void* q, const void* k, const void* v,
                                            float* out, int B, int H, int T, int d, int dv,
                                            int C, kata_lin_feature_t feature, float eps,
                                            int normalize, kata_dtype_t dtype,
                                            hipStream_t stream);
KATA_API kata_status_t kata_lin_fwd_chunked_ws(const void* q, const void* k, const void* v,
                                               float* out, int B, int H, int T, int d, int dv,
                                               int C, kata_lin_feature_t feature, float eps,
                                               int normalize, kata_dtype_t dtype,
                                               int span_chunks, void* workspace,
                                               size_t workspace_bytes, hipStream_t stream);
KATA_API kata_status_t kata_lin_fwd_chunked_timed(const void* q, const void* k, const void* v,
                                                  float* out, int B, int H, int T, int d, int dv,
                                                  int C, kata_lin_feature_t feature, float eps,
                                                  int normalize, kata_dtype_t dtype,
                                                  int span_chunks, void* workspace,
                                                  size_t workspace_bytes,
                                                  hipEvent_t* stage_events, hipStream_t stream);
/* Workspace bytes for these arguments (0 when invalid or unsupported). */
KATA_API size_t kata_lin_fwd_workspace_bytes(int B, int H, int T, int d, int dv, int C,
                                             kata_lin_feature_t feature, kata_dtype_t dtype,
                                             int span_chunks);
/* The span (in chunks) that span_chunks = 0 selects (0 when invalid or unsupported). */
KATA_API int kata_lin_default_span(int B, int H, int T, int d, int dv, int C,
                                   kata_lin_feature_t feature, kata_dtype_t dtype);

/*
 * Backward of the causal KATA-Mg forward (g = 1: KATA-M1) in the O(T)
 * chunked form: the chunked backward of the appendix's chunkwise algorithm (a
 * reverse scan over chunks carrying the state cotangent, forward quantities
 * recomputed from chunk-boundary states, the feature-map VJP
 * dx = (dPsi + dPsi^T) x closing the chain).  For output cotangents
 * dout = dL/do it returns
 *     dq = dL/dq, dk = dL/dk, dv_out = dL/dv,
 * with a_t = dout_t / D_t, b_t = -<dout_t, o_t> / D_t, dL/dw_ti = <a_t, v_i> + b_t
 * (i <= t), w_ti = sum_blk (q_t,blk . k_i,blk)^2.  A row with D_t = 0 (whose
 * readout is the constant 0) passes no gradient.
 *   q, k, v : the forward's inputs (dtype), out : its fp32 output
 *             [B][H][T][dv] (kata_fwd_chunked or kata_mg_fwd_chunked), dout :
 *             fp32 [B][H][T][dv]; dq, dk : fp32 [B][H][T][d], dv_out : fp32
 *             [B][H][T][dv], overwritten, none aliasing an input.
 *   Supported: d <= 64, dv <= 256, C <= 64, g | d, fp32 or bf16 inputs.  Else
 *   KATA_ERR_UNSUPPORTED (shape) or KATA_ERR_INVALID_ARG.
 *   Arithmetic: fp32 throughout, except for bf16 inputs with d = dv = C = 64
 *   and g = 1, where the chunk states, the scanned state records (S rounded to
 *   bf16, z fp32, fp32 sums) and the gradient products run on the bf16 matrix
 *   cores with fp32 accumulation, a_t and b_t entering as bf16 hi + lo pairs;
 *   that path's gradients are within 2e-2 (per-head relative l2) of the exact
 *   ones, about 2e-3 on the test workloads.  Up to T = 4096 (8192 from eight
 *   heads B x H on) those shapes take the quadratic form instead, pair tiles on
 *   the same matrix cores with no chunk states (a_t as a bf16 pair, b_t fp32),
 *   and so do the fp32-arithmetic shapes with g = 1 and dv <= 64 where that is
 *   faster, in fp32, at most up to T = 4096 (8192 where d and dv are 16, 32 or 64):
 *   kata_bwd_form.
 *   workspace : >= kata_bwd_workspace_bytes(...) bytes, 256-byte aligned,
 *   caller-owned, contents undefined on exit; kata_bwd_chunked allocates it
 *   stream-ordered.  stage_events : 7 caller-created events, recorded before
 *   the first launch and after each of the six (forward states, prefix scan,
 *   per-token coefficients, backward states, suffix scan, gradients); where
 *   kata_bwd_form() is KATA_BWD_FUSED_STATES each state launch also writes the
 *   scanned records and the two scan intervals are empty; KATA_BWD_QUADRATIC
 *   leaves all four state and scan intervals empty.
 */
KATA_API kata_status_t kata_bwd_chunked(const void* q, const void* k, const void* v,
                                        const float* out, const float* dout, float* dq,
                                        float* dk, float* dv_out, int B, int H, int T, int d,
                                        int dv, int C, int g, kata_dtype_t dtype,
                                        hipStream_t stream);
KATA_API kata_status_t kata_bwd_chunked_ws(const void* q, const void* k, const void* v,
                                           const float* out, const float* dout, float* dq,
                                           float* dk, float* dv_out, int B, int H, int T, int d,
                                           int dv, int C, int g, kata_dtype_t dtype,
                                           void* workspace, size_t workspace_bytes,
                                           hipStream_t stream);
KATA_API kata_status_t kata_bwd_chunked_timed(const void* q, const void* k, const void* v,
                                              const float* out, const float* dout, float* dq,
                                              float* dk, float* dv_out, int B, int H, int T,
                                              int d, int dv, int C, int g, kata_dtype_t dtype,
                                              void* workspace, size_t workspace_bytes,
                                              hipEvent_t* stage_events, hipStream_t stream);
/*
 * kata_bwd_chunked_ws with two optional arguments: den, null or the
 * denominators D_t that kata_fwd_chunked_train_ws wrote for this forward
 * (fp32 [B][H][T], 16-byte aligned), from which the per-token coefficients
 * a_t, b_t are formed directly instead of from the prefix states (same values
 * up to rounding); stage_events, null or 7 events as for
 * kata_bwd_chunked_timed (all non-null).  Any supported backward shape.
 */
KATA_API kata_status_t kata_bwd_chunked_ex(const void* q, const void* k, const void* v,
                                           const float* out, const float* dout, const float* den,
                                           float* dq, float* dk, float* dv_out, int B, int H,
                                           int T, int d, int dv, int C, int g,
                                           kata_dtype_t dtype, void* workspace,
                                           size_t workspace_bytes, hipEvent_t* stage_events,
                                           hipStream_t stream);
KATA_API size_t kata_bwd_workspace_bytes(int B, int H, int T, int d, int dv, int C, int g,
                                         kata_dtype_t dtype);
/* The form in which kata_bwd_chunked* of these arguments runs: chunk states with a
 * state launch and a scan launch for each record stream, chunk states with both in
 * one launch, or the quadratic form.  -1 where the arguments are invalid or
 * unsupported. */
enum { KATA_BWD_STATES = 0, KATA_BWD_FUSED_STATES = 1, KATA_BWD_QUADRATIC = 2 };
KATA_API int kata_bwd_form(int B, int H, int T, int d, int dv, int C, int g, kata_dtype_t dtype);
/* The form of the chunk-state backward for this shape (whether or not its T
 * takes the quadratic form, which kata_bwd_form tells): 1 when it computes the prefix and suffix records
 * with the state and the scan in one launch each (bf16 inputs at
 * d = dv = C = 64, g = 1, from 16 heads B x H on), 0 when it runs a state launch
 * and a scan launch for each, -1 for an unsupported shape. */
KATA_API int kata_bwd_fused_scan(int B, int H, int T, int d, int dv, int C, int g,
                                 kata_dtype_t dtype);

/*
 * Operators around a recurrent mixer: the short convolution over a projection's
 * channels, the norms of query and key heads with their position rotation, and
 * the selective state space scan.  Conventions that differ from the ones above:
 *  - Activations are token-major, as a projection writes them, and may be views
 *    of a wider tensor: each has element strides (>= 0) over its outer
 *    dimensions, the innermost dimension being contiguous.  Their base addresses
 *    need the alignment of one element only; rows of aligned 16-byte pieces
 *    are read and written as such.  The rows of an output must not overlap.
 *  - Inputs, outputs and gradients of activations are fp32 or bf16 (dtype), each
 *    output rounded once; parameters, their gradients and states are fp32 unless
 *    stated, 4-byte aligned and contiguous.  Sums are held in fp32 or fp64.
 *  - lengths (nullable): int32 [B] on the device, the tokens of each sequence of
 *    a padded batch (clamped to 0..T).  Rows past a sequence's end are neither
 *    read nor written; a returned state is the one after its last token (of
 *    no tokens: the given state, or zeros).
 *  - No output may alias or overlap an input, except the states that a step
 *    updates in place, or another output; equal base addresses are
 *    KATA_ERR_INVALID_ARG.
 *  - Non-finite inputs reach no output of an earlier token, another sequence or
 *    (where heads are separate) another head; in gradients they may reach
 *    every output of their sequence, and the parameters'.
 *  - Every call enqueues kernel launches only and can be captured into a HIP
 *    graph; results do not depend on the order in which workgroups run.
 *    T <= 2^30; larger T and launches of 2^32 threads or more are
 *    KATA_ERR_UNSUPPORTED.
 */

/*
 * Causal depthwise convolution of W taps (2, 3 or 4; else KATA_ERR_UNSUPPORTED) over
 * D <= 2^20 channels:
 *     pre[t] = bias + sum_{j<W} w[j] x[t - (W-1) + j],   y = act(pre).
 *   x, y : [B][T][D], strides x_batch, x_token, y_batch, y_token;  w : [D][W];
 *   bias : [D], nullable.
 *   state_in  (nullable: zeros) : [B][W-1][D] in dtype, the rows before x[0],
 *   state_out (nullable) : the last W-1 rows, for kata_conv_step or a next call.
 */
typedef enum { KATA_CONV_NONE = 0, KATA_CONV_SILU = 1 } kata_conv_act_t;
KATA_API kata_status_t kata_conv_fwd(const void* x, const float* w, const float* bias,
                                     const void* state_in, const int* lengths, void* y,
                                     void* state_out, int B, int T, int D, int W,
                                     long long x_batch, long long x_token, long long y_batch,
                                     long long y_token, kata_conv_act_t act, kata_dtype_t dtype,
                                     hipStream_t stream);
/* One token of every sequence: x, y [B][D] (strides x_batch, y_batch); the rows of
 * state [B][W-1][D] move up by one. */
KATA_API kata_status_t kata_conv_step(void* state, const void* x, const float* w,
                                      const float* bias, void* y, int B, int D, int W,
                                      long long x_batch, long long y_batch, kata_conv_act_t act,
                                      kata_dtype_t dtype, hipStream_t stream);
/* Gradients of kata_conv_fwd without state and lengths: dx [B][T][D] (strides), dw [D][W],
 * dbias [D] (either nullable) from dy [B][T][D] (strides).  workspace: at least
 * kata_conv_bwd_workspace_bytes(...) bytes (0: invalid or unsupported arguments),
 * 256-byte aligned, contents undefined on exit. */
KATA_API kata_status_t kata_conv_bwd_ws(const void* x, const float* w, const float* bias,
                                        const void* dy, void* dx, float* dw, float* dbias, int B,
                                        int T, int D, int W, long long x_batch, long long x_token,
                                        long long dy_batch, long long dy_token,
                                        long long dx_batch, long long dx_token,
                                        kata_conv_act_t act, kata_dtype_t dtype, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_conv_bwd_workspace_bytes(int B, int T, int D, int W, kata_dtype_t dtype);

/*
 * Norms of query and key heads with the position rotation in the same pass, from a
 * projection's rows to the head-major tensors of the attention calls above (at T = 1:
 * of the decode step), which take as many key heads as query heads.  For every head row x of
 * width d:
 *     hat = x / sqrt(mean(x^2) + eps)  (KATA_NORM_RMS; KATA_NORM_L2: the sum for the mean;
 *           KATA_NORM_NONE: x),        y = R (w hat),
 * R turning pair i < r/2 of the first r coordinates by the angle pos * freq[i]:
 * coordinates (i, i + r/2), or with pairs = 1 (2i, 2i+1).
 *   q : [B][T][Hq][d], k : [B][T][Hk][d] with strides (batch, token, head); k, wk and the
 *   key outputs are null where Hk = 0.  wq, wk : [d], nullable (ones).
 *   pos : int32 [B][T], nullable (0..T-1);  freq : fp64 [r/2], null where r = 0 (angles are
 *   formed in fp64, off by 2^-52 of themselves: 5e-10 rad at a position of 2^21, 5e-7 at 2^31).
 *   yq : [B][Hq][T][d], yk : [B][Hk][T][d], contiguous, in dtype.
 *   d <= 256 (else KATA_ERR_UNSUPPORTED), r even, 0 <= r <= d, eps >= 0 and finite;
 *   Hq + Hk <= 65535.  Squares are summed in fp32: a row's sum and its mean + eps (L2: sum + eps)
 *   have to lie between 2^-126 and 2^128, so a row of zeros needs an eps of 2^-126 or more.
 */
typedef enum { KATA_NORM_NONE = 0, KATA_NORM_RMS = 1, KATA_NORM_L2 = 2 } kata_norm_t;
KATA_API kata_status_t kata_qk_norm_fwd(const void* q, const void* k, const float* wq,
                                        const float* wk, const int* pos, const double* freq,
                                        void* yq, void* yk, int B, int T, int Hq, int Hk, int d,
                                        int r, long long q_batch, long long q_token,
                                        long long q_head, long long k_batch, long long k_token,
                                        long long k_head, kata_norm_t norm, float eps, int pairs,
                                        kata_dtype_t dtype, hipStream_t stream);
/* Its gradients: dq, dk of the outputs, head-major as yq and yk, in dy_dtype (fp32 as the
 * attention's gradients, or dtype); dxq [B][T][Hq][d] and dxk [B][T][Hk][d] in dtype, with
 * strides of their own; dwq, dwk [d], nullable.  workspace as for kata_conv_bwd_ws. */
KATA_API kata_status_t kata_qk_norm_bwd_ws(
    const void* q, const void* k, const float* wq, const float* wk, const int* pos,
    const double* freq, const void* dq, const void* dk, void* dxq, void* dxk, float* dwq,
    float* dwk, int B, int T, int Hq, int Hk, int d, int r, long long q_batch, long long q_token,
    long long q_head, long long k_batch, long long k_token, long long k_head, long long dxq_batch,
    long long dxq_token, long long dxq_head, long long dxk_batch, long long dxk_token,
    long long dxk_head, kata_norm_t norm, float eps, int pairs, kata_dtype_t dtype,
    kata_dtype_t dy_dtype, void* workspace, size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_qk_norm_bwd_workspace_bytes(int B, int T, int Hq, int Hk, int d,
                                                 kata_dtype_t dtype);

/*
 * Selective state space scan, per head with a state S [N][P]:
 *     step_t = softplus(dt_t + bias)   (softplus = 0: dt_t + bias),
 *     S_t = exp(step_t A) S_{t-1} + step_t B_t x_t^T,    y_t = C_t^T S_t + D x_t.
 *   x, y : [B][T][H][P];  dt : [B][T][H];  Bm, Cm : [B][T][G][N], a group's rows shared by its
 *   H / G heads (G divides H, else KATA_ERR_INVALID_ARG); all in dtype, with strides.
 *   A : [H] (negative for a decaying state), D, dt_bias : [H], nullable.
 *   S_in (nullable: zeros), S_out (nullable) : fp32 [B][H][N][P], 16-byte aligned.
 *   N <= 128, P <= 256, B*H <= 65535, else KATA_ERR_UNSUPPORTED.
 *   Computed in chunks of 64 (fp32: 32) tokens on the matrix cores; long sequences of few
 *   heads are split into spans whose states are joined.  bf16: products accumulate in fp32,
 *   the weights of a chunk's pairs and the state that y reads are rounded to bf16 once, D x is
 *   added in fp32, the state itself keeps 2^-17 of every term (all of fp32's bits where S_out is
 *   asked for: y of the two calls may differ in a last rounding).
 *   A positive A or a negative step grows the state as the formula says, until it overflows.
 *   With softplus a dt of -inf, or of the type's lowest value, is a step of 0: its token leaves
 *   the state as it is.
 *   strides : element strides over batch, token and head (group); null: contiguous.
 *   workspace : at least kata_ssm_workspace_bytes(..., backward) bytes (0: invalid or
 *   unsupported arguments), 256-byte aligned, contents undefined on exit.
 */
typedef struct {
  long long x_batch, x_token, x_head;
  long long dt_batch, dt_token, dt_head;
  long long b_batch, b_token, b_group;
  long long c_batch, c_token, c_group;
  long long y_batch, y_token, y_head; /* y, or dy in the backward */
} kata_ssm_strides_t;
KATA_API kata_status_t kata_ssm_fwd_ws(const void* x, const void* dt, const float* A,
                                       const void* Bm, const void* Cm, const float* D,
                                       const float* dt_bias, const float* S_in,
                                       const int* lengths, void* y, float* S_out, int B, int T,
                                       int H, int G, int N, int P,
                                       const kata_ssm_strides_t* strides, int softplus,
                                       kata_dtype_t dtype, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
/* Gradients of kata_ssm_fwd_ws from a zero state, without lengths: dx, ddt, dBm, dCm in
 * dtype, contiguous and shaped as x, dt, Bm, Cm (those of a group summed over its heads);
 * dA, dD, dt_dbias [H], each nullable.  bf16: the pair weights that dx, dBm and dCm are formed from,
 * and the state's gradient that dBm reads, are rounded to bf16 once; ddt and the parameters'
 * gradients keep fp32's bits throughout, their sums over tokens are fp64. */
KATA_API kata_status_t kata_ssm_bwd_ws(const void* x, const void* dt, const float* A,
                                       const void* Bm, const void* Cm, const float* D,
                                       const float* dt_bias, const void* dy, void* dx, void* ddt,
                                       float* dA, void* dBm, void* dCm, float* dD,
                                       float* dt_dbias, int B, int T, int H, int G, int N, int P,
                                       const kata_ssm_strides_t* strides, int softplus,
                                       kata_dtype_t dtype, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_ssm_workspace_bytes(int B, int T, int H, int G, int N, int P,
                                         kata_dtype_t dtype, int backward);
/* One token: x, y [B][H][P], dt [B][H], Bm, Cm [B][G][N] (the token strides are not read);
 * S [B][H][N][P], 16-byte aligned, updated in place. */
KATA_API kata_status_t kata_ssm_step(float* S, const void* x, const void* dt, const float* A,
                                     const void* Bm, const void* Cm, const float* D,
                                     const float* dt_bias, void* y, int B, int H, int G, int N,
                                     int P, const kata_ssm_strides_t* strides, int softplus,
                                     kata_dtype_t dtype, hipStream_t stream);

/*
 * Operators of a mixer's layer in 8 bits: the residual's addition and its norm, the quantiser,
 * the projections' product, and a recurrent mixer with a decay per channel.  The conventions of
 * the operators above hold, with these additions:
 *  - Activations without a batch are rows [M][..] with one row stride (elements).
 *  - 8 bits: e4m3 codes (1 sign, 4 exponent, 3 mantissa bits; largest 448, no infinity), one
 *    byte each, with an fp32 scale for each block of 128 columns of a row, or of 128 x 128:
 *    a code stands for its value times its block's scale.  Scales are contiguous,
 *    [rows][ceil(columns / 128)] or [ceil(rows / 128)][ceil(columns / 128)], the last blocks
 *    being those that are left.  Quantising:
 *        scale = max(max |x| / 448, 2^-126),  code = x / scale to nearest, ties to even
 *    (of bf16 inputs to kata_f8_quant: x (1 / scale) in fp32, to nearest).
 *    A NaN becomes a NaN code and leaves the scale to the block's other values; an infinity
 *    makes its block's scale infinite and its own code NaN.
 *  - Rows of codes may begin anywhere; products of rows that begin at multiples of 16 bytes
 *    are several times faster.
 */

/*
 * Root-mean-square norm with the residual's addition:
 *     s = x + res (rounded to dtype; without res: x),   y = s w / sqrt(mean(s^2) + eps).
 *   x, res, sum, y : [M][D] in dtype;  w : [D], nullable (ones).
 *   res, sum : both or neither; sum receives s, and may be res itself with its row stride.
 *   y, or q and scale (y in 8 bits, quantised before it is rounded, blocks of one row), or all three.
 *   D <= 32768, else KATA_ERR_UNSUPPORTED.  Squares are summed in fp64;
 *   mean + eps has to lie between 2^-250 and 2^250.
 */
KATA_API kata_status_t kata_add_norm_fwd(const void* x, const void* res, const float* w, void* sum,
                                         void* y, void* q, float* scale, int M, int D,
                                         long long x_row, long long res_row, long long sum_row,
                                         long long y_row, long long q_row, float eps,
                                         kata_dtype_t dtype, hipStream_t stream);
/* Its gradients from sum (s; x without res) and dy, the gradient of y before it is quantised, in
 * dy_dtype (fp32, or dtype): dx [M][D], the gradient of x and of res alike, to which dsum (nullable:
 * none), the gradient that reaches s by the residual's own way, is added; dw [D], nullable.
 * A row's sums are formed in fp32 here, in fp64 where they leave its range.  workspace as for kata_conv_bwd_ws. */
KATA_API kata_status_t kata_add_norm_bwd_ws(const void* sum, const float* w, const void* dy,
                                            const void* dsum, void* dx, float* dw, int M, int D,
                                            long long sum_row, long long dy_row,
                                            long long dsum_row, long long dx_row, float eps,
                                            kata_dtype_t dtype, kata_dtype_t dy_dtype,
                                            void* workspace, size_t workspace_bytes,
                                            hipStream_t stream);
KATA_API size_t kata_add_norm_bwd_workspace_bytes(int M, int D, kata_dtype_t dtype);

/*
 * x [M][K] (dtype, a row stride) in 8 bits: q [M][K] with scale, qt [K][M] (the transpose,
 * quantised by itself) with scale_t, or both.  rows = 1: blocks of one row (of x for q, of its
 * transpose for qt); rows = 128: blocks of 128 x 128, q and qt holding the same codes.
 * The operands of a product y = x w^T and of its gradients:
 *     y = (x rows) (w 128 x 128)^T,  dx = (dy rows) (wt 128 x 128)^T,
 *     dw = (dyt rows) (xt rows)^T.
 */
KATA_API kata_status_t kata_f8_quant(const void* x, void* q, float* scale, void* qt,
                                     float* scale_t, int M, int K, int rows, long long x_row,
                                     long long q_row, long long qt_row, kata_dtype_t dtype,
                                     hipStream_t stream);

/*
 * Product of 8-bit operands:  c[m][n] = sum_k a[m][k] b[n][k], each code times its scale.
 *   a : codes [M][K] with a_scale [M][ceil(K/128)];  b : codes [N][K] with b_scale of blocks of
 *   b_rows = 128 or 1 rows;  c : [M][N] in dtype (rounded once); row strides.
 *   A block's products are summed by the matrix cores, the scaled blocks in fp32.  For c in fp32 the
 *   products are exact and their sums fp32's.  For c in bf16 eight products of neighbouring k are cut,
 *   towards zero, to 2^-13 of the power of two below the largest of them before they are added: 1.3e-5 of
 *   a result of ordinary operands, at most 7 x 2^-13 of the sum of those largest.  Where results
 *   cancel so far that this counts, ask for fp32.
 *   Scales may have any finite value (blocks of one above 2^63 or below 2^-62 take up to six times as long;
 *   a part whose scale is the least one, 2^-126, may be off by 2^-125).  A non-finite scale or a NaN
 *   code reaches its rows of c.
 *   workspace : at least kata_f8_gemm_workspace_bytes(...) bytes (0: invalid or unsupported
 *   arguments), 256-byte aligned, contents undefined on exit.
 */
KATA_API kata_status_t kata_f8_gemm_ws(const void* a, const float* a_scale, const void* b,
                                       const float* b_scale, void* c, int M, int N, int K,
                                       int b_rows, long long a_row, long long b_row,
                                       long long c_row, kata_dtype_t dtype, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_f8_gemm_workspace_bytes(int M, int N, int K);

/*
 * Gated linear recurrence, per channel:
 *     rate_t = c softplus(lam) sigmoid(r_t + r_bias),   a_t = exp(-rate_t),
 *     h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t + i_bias) x_t,   y_t = h_t.
 *   x, r, i, y : [B][T][D] in dtype, with strides;  lam, r_bias, i_bias (both nullable) : [D].
 *   h_in (nullable: zeros), h_out (nullable) : fp32 [B][D].  c > 0 and finite; D <= 2^20.
 *   starts (nullable) : fp32 [B][kata_recur_spans(T)][D], the state before each span of tokens,
 *   for the gradients (undefined for spans past a sequence's end).
 *   strides : element strides over batch and token; null: contiguous (all [B][T][D]).
 *   workspace : at least kata_recur_workspace_bytes(..., backward) bytes (0: invalid or
 *   unsupported arguments), 256-byte aligned, contents undefined on exit.
 *   Once a state is not finite, later ones are not either, but may be NaN for infinity.
 */
typedef struct {
  long long x_batch, x_token, r_batch, r_token, i_batch, i_token;
  long long y_batch, y_token; /* y, or dy in the backward */
  long long dx_batch, dx_token, dr_batch, dr_token, di_batch, di_token; /* backward only */
} kata_recur_strides_t;
KATA_API kata_status_t kata_recur_fwd_ws(const void* x, const void* r, const void* i,
                                         const float* lam, const float* r_bias,
                                         const float* i_bias, const float* h_in,
                                         const int* lengths, void* y, float* h_out, float* starts,
                                         int B, int T, int D, const kata_recur_strides_t* strides,
                                         float c, kata_dtype_t dtype, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream);
/* Gradients of kata_recur_fwd_ws from dy [B][T][D] and dh_out [B][D] (nullable: zeros), the
 * gradient of its h_out: dx, dr, di [B][T][D] in dtype; dlam, dr_bias, di_bias [D] and dh_in [B][D]
 * in fp32, each nullable.  h_in and lengths as in the forward; starts: what it returned, or null
 * (formed again, at the cost of a pass over the inputs; with starts, h_in is not read).  Where a
 * rate is 0, so that a = 1, the gradients by the rate are taken as 0. */
KATA_API kata_status_t kata_recur_bwd_ws(
    const void* x, const void* r, const void* i, const float* lam, const float* r_bias,
    const float* i_bias, const float* h_in, const int* lengths, const float* starts,
    const void* dy, const float* dh_out, void* dx, void* dr, void* di, float* dlam, float* dr_bias,
    float* di_bias, float* dh_in, int B, int T, int D, const kata_recur_strides_t* strides,
    float c, kata_dtype_t dtype, void* workspace, size_t workspace_bytes, hipStream_t stream);
KATA_API size_t kata_recur_workspace_bytes(int B, int T, int D, kata_dtype_t dtype, int backward);
/* Spans of T tokens (0: T < 1). */
KATA_API int kata_recur_spans(int T);
/* One token: x, r, i, y [B][D]; h fp32 [B][D], updated in place. */
KATA_API kata_status_t kata_recur_step(float* h, const void* x, const void* r, const void* i,
                                       const float* lam, const float* r_bias, const float* i_bias,
                                       void* y, int B, int D, long long x_batch, long long r_batch,
                                       long long i_batch, long long y_batch, float c,
                                       kata_dtype_t dtype, hipStream_t stream);

/* Static, human-readable name of a status code. */
KATA_API const char* kata_status_string(kata_status_t s);

/* ABI version of this header (major*100 + minor). */
KATA_API int kata_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* KATA_H */
