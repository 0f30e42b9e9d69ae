"""libkata: causal KATA-M1 attention (rank-one PSD feature map) on MI355X.

Thin Python binding over the C ABI in include/kata.h.  It only marshals torch
device tensors (pointers, sizes, the current HIP stream) into the library;
every step of the computation runs in the library's HIP kernels.  There is no
fallback: if libkata.so is missing or fails to load, every call raises.

    import paper_2607_17419_amd as kata
    out = kata.fwd_chunked(q, k, v, C=64)           # q, k: [B,H,T,d]; v: [B,H,T,dv]
    S, z = kata.prefill_state(k, v)                 # packed state after T tokens
    o = kata.decode_step(S, z, q1, k1, v1)          # one token per head, in place

Around a recurrent mixer, on token-major rows (views of a projection's output):

    u = kata.conv_fwd(x, w, bias)                   # short causal convolution, [B,T,D]
    q, k = kata.qk_norm_fwd(q, k, wq, wk, freq)     # norms and rotation, to [B,H,T,d]
    y = kata.ssm_fwd(x, dt, A, Bm, Cm, D, bias)     # selective scan, [B,T,H,P]
    y = kata.recur_fwd(x, r, i, lam)                # gated linear recurrence, [B,T,D]

and of its layer in 8 bits (e4m3 with a scale for each block of 128):

    w8, ws = kata.f8_quant(w, rows=128)             # a weight's 128 x 128 blocks
    a8, as_, s = kata.add_norm_f8_fwd(x, g, res)    # residual and norm, to the product's operand
    c = kata.f8_gemm(a8, as_, w8, ws)               # [..,N]
"""
from __future__ import annotations

import ctypes
import functools
import os

__all__ = [
    "KataError", "lib", "fwd_chunked", "fwd_chunked_timed", "fwd_chunked_alloc", "workspace_bytes",
    "default_span", "prefill_state", "decode_step", "packed_dim", "LIB_PATH",
    "conv_fwd", "conv_step", "conv_bwd", "qk_norm_fwd", "qk_norm_bwd", "rope_frequencies",
    "ssm_fwd", "ssm_step", "ssm_bwd",
    "add_norm_fwd", "add_norm_f8_fwd", "add_norm_bwd", "f8_quant", "f8_gemm",
    "recur_fwd", "recur_fwd_train", "recur_bwd", "recur_step",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkata.so")

KATA_OK, KATA_ERR_INVALID_ARG, KATA_ERR_UNSUPPORTED, KATA_ERR_HIP = 0, 1, 2, 3
KATA_F32, KATA_BF16 = 0, 1

# every symbol include/kata.h declares
EXPORTED = (
    "kata_fwd_chunked", "kata_fwd_chunked_ws", "kata_fwd_chunked_timed", "kata_fwd_workspace_bytes",
    "kata_fwd_chunked_train_ws", "kata_bwd_chunked_ex",
    "kata_fwd_default_span", "kata_fwd_form", "kata_fwd_quadratic", "kata_fwd_quadratic_ws",
    "kata_fwd_quadratic_workspace_bytes", "kata_prefill_state", "kata_decode_step",
    "kata_mg_fwd_chunked", "kata_mg_fwd_chunked_ws", "kata_mg_fwd_chunked_timed",
    "kata_mg_fwd_workspace_bytes", "kata_mg_fwd_quadratic_ws",
    "kata_mg_fwd_quadratic_workspace_bytes", "kata_mg_prefill_state", "kata_mg_decode_step",
    "kata_lin_dim", "kata_lin_fwd_chunked", "kata_lin_fwd_chunked_ws",
    "kata_lin_fwd_chunked_timed", "kata_lin_fwd_workspace_bytes", "kata_lin_default_span",
    "kata_bwd_chunked", "kata_bwd_chunked_ws", "kata_bwd_chunked_timed",
    "kata_bwd_workspace_bytes", "kata_bwd_fused_scan", "kata_bwd_form",
    "kata_fwd_chunked_noalloc", "kata_noalloc_scratch_bytes",
    "kata_status_string", "kata_abi_version",
    "kata_conv_fwd", "kata_conv_step", "kata_conv_bwd_ws", "kata_conv_bwd_workspace_bytes",
    "kata_qk_norm_fwd", "kata_qk_norm_bwd_ws", "kata_qk_norm_bwd_workspace_bytes",
    "kata_ssm_fwd_ws", "kata_ssm_bwd_ws", "kata_ssm_workspace_bytes", "kata_ssm_step",
    "kata_add_norm_fwd", "kata_add_norm_bwd_ws", "kata_add_norm_bwd_workspace_bytes",
    "kata_f8_quant", "kata_f8_gemm_ws", "kata_f8_gemm_workspace_bytes",
    "kata_recur_fwd_ws", "kata_recur_bwd_ws", "kata_recur_workspace_bytes", "kata_recur_spans",
    "kata_recur_step",
)

# what kata_fwd_form and kata_bwd_form return (-1: unsupported)
FWD_STATES, FWD_QUADRATIC = 0, 1
BWD_STATES, BWD_FUSED_STATES, BWD_QUADRATIC = 0, 1, 2

# kata_lin_feature_t
LIN_IDENTITY, LIN_RELU, LIN_ELU, LIN_LORENTZ, LIN_LORENTZ_S = 0, 1, 2, 3, 4

# kata_conv_act_t, kata_norm_t
CONV_NONE, CONV_SILU = 0, 1
NORM_NONE, NORM_RMS, NORM_L2 = 0, 1, 2


class KataError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {_status_name(status)} ({status})")


_lib = None


def lib():
    """The loaded libkata (ctypes.CDLL); raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libkata.so not found at {LIB_PATH}; run "
                          "`python -m paper_2607_17419_amd.build` first")
    L = ctypes.CDLL(LIB_PATH)
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.kata_fwd_chunked.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    L.kata_fwd_chunked.restype = i
    L.kata_fwd_chunked_noalloc.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    L.kata_fwd_chunked_noalloc.restype = i
    L.kata_noalloc_scratch_bytes.argtypes = []
    L.kata_noalloc_scratch_bytes.restype = sz
    L.kata_fwd_chunked_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp, sz, vp]
    L.kata_fwd_chunked_ws.restype = i
    L.kata_fwd_chunked_timed.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp, sz, vp, vp]
    L.kata_fwd_chunked_timed.restype = i
    L.kata_fwd_chunked_train_ws.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp, sz, vp]
    L.kata_fwd_chunked_train_ws.restype = i
    L.kata_fwd_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.kata_fwd_workspace_bytes.restype = sz
    L.kata_fwd_default_span.argtypes = [i, i, i, i, i, i, i]
    L.kata_fwd_default_span.restype = i
    L.kata_fwd_form.argtypes = [i, i, i, i, i, i, i, i, i]
    L.kata_fwd_form.restype = i
    L.kata_prefill_state.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, vp]
    L.kata_prefill_state.restype = i
    L.kata_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    L.kata_decode_step.restype = i
    L.kata_fwd_quadratic.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, vp]
    L.kata_fwd_quadratic.restype = i
    L.kata_fwd_quadratic_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, vp, sz, vp]
    L.kata_fwd_quadratic_ws.restype = i
    L.kata_fwd_quadratic_workspace_bytes.argtypes = [i, i, i, i, i, i]
    L.kata_fwd_quadratic_workspace_bytes.restype = sz
    L.kata_mg_fwd_chunked.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp]
    L.kata_mg_fwd_chunked.restype = i
    L.kata_mg_fwd_chunked_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, i, vp, sz, vp]
    L.kata_mg_fwd_chunked_ws.restype = i
    L.kata_mg_fwd_chunked_timed.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, i, vp, sz,
                                            vp, vp]
    L.kata_mg_fwd_chunked_timed.restype = i
    L.kata_mg_fwd_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i]
    L.kata_mg_fwd_workspace_bytes.restype = sz
    L.kata_mg_fwd_quadratic_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, vp, sz, vp]
    L.kata_mg_fwd_quadratic_ws.restype = i
    L.kata_mg_fwd_quadratic_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    L.kata_mg_fwd_quadratic_workspace_bytes.restype = sz
    L.kata_mg_prefill_state.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, vp]
    L.kata_mg_prefill_state.restype = i
    L.kata_mg_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, vp]
    L.kata_mg_decode_step.restype = i
    f = ctypes.c_float
    L.kata_lin_dim.argtypes = [i, i]
    L.kata_lin_dim.restype = i
    L.kata_lin_fwd_chunked.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, i, vp]
    L.kata_lin_fwd_chunked.restype = i
    L.kata_lin_fwd_chunked_ws.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, i, i, vp,
                                          sz, vp]
    L.kata_lin_fwd_chunked_ws.restype = i
    L.kata_lin_fwd_chunked_timed.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, i, i, vp,
                                             sz, vp, vp]
    L.kata_lin_fwd_chunked_timed.restype = i
    L.kata_lin_fwd_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i]
    L.kata_lin_fwd_workspace_bytes.restype = sz
    L.kata_lin_default_span.argtypes = [i, i, i, i, i, i, i, i]
    L.kata_lin_default_span.restype = i
    L.kata_bwd_chunked.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i, vp]
    L.kata_bwd_chunked.restype = i
    L.kata_bwd_chunked_ws.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i,
                                      vp, sz, vp]
    L.kata_bwd_chunked_ws.restype = i
    L.kata_bwd_chunked_timed.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i,
                                         vp, sz, vp, vp]
    L.kata_bwd_chunked_timed.restype = i
    L.kata_bwd_chunked_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, i,
                                      vp, sz, vp, vp]
    L.kata_bwd_chunked_ex.restype = i
    L.kata_bwd_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.kata_bwd_workspace_bytes.restype = sz
    L.kata_bwd_fused_scan.argtypes = [i, i, i, i, i, i, i, i]
    L.kata_bwd_fused_scan.restype = i
    L.kata_bwd_form.argtypes = [i, i, i, i, i, i, i, i]
    L.kata_bwd_form.restype = i
    ll = ctypes.c_longlong
    L.kata_conv_fwd.argtypes = [vp] * 7 + [i] * 4 + [ll] * 4 + [i, i, vp]
    L.kata_conv_step.argtypes = [vp] * 5 + [i] * 3 + [ll] * 2 + [i, i, vp]
    L.kata_conv_bwd_ws.argtypes = [vp] * 7 + [i] * 4 + [ll] * 6 + [i, i, vp, sz, vp]
    L.kata_conv_bwd_workspace_bytes.argtypes = [i] * 5
    L.kata_qk_norm_fwd.argtypes = [vp] * 8 + [i] * 6 + [ll] * 6 + [i, f, i, i, vp]
    L.kata_qk_norm_bwd_ws.argtypes = ([vp] * 12 + [i] * 6 + [ll] * 12
                                      + [i, f, i, i, i, vp, sz, vp])
    L.kata_qk_norm_bwd_workspace_bytes.argtypes = [i] * 6
    L.kata_ssm_fwd_ws.argtypes = [vp] * 11 + [i] * 6 + [vp, i, i, vp, sz, vp]
    L.kata_ssm_bwd_ws.argtypes = [vp] * 15 + [i] * 6 + [vp, i, i, vp, sz, vp]
    L.kata_ssm_workspace_bytes.argtypes = [i] * 8
    L.kata_ssm_step.argtypes = [vp] * 9 + [i] * 5 + [vp, i, i, vp]
    L.kata_add_norm_fwd.argtypes = [vp] * 7 + [i] * 2 + [ll] * 5 + [f, i, vp]
    L.kata_add_norm_bwd_ws.argtypes = [vp] * 6 + [i] * 2 + [ll] * 4 + [f, i, i, vp, sz, vp]
    L.kata_add_norm_bwd_workspace_bytes.argtypes = [i] * 3
    L.kata_f8_quant.argtypes = [vp] * 5 + [i] * 3 + [ll] * 3 + [i, vp]
    L.kata_f8_gemm_ws.argtypes = [vp] * 5 + [i] * 4 + [ll] * 3 + [i, vp, sz, vp]
    L.kata_f8_gemm_workspace_bytes.argtypes = [i] * 3
    L.kata_recur_fwd_ws.argtypes = [vp] * 11 + [i] * 3 + [vp, f, i, vp, sz, vp]
    L.kata_recur_bwd_ws.argtypes = [vp] * 18 + [i] * 3 + [vp, f, i, vp, sz, vp]
    L.kata_recur_workspace_bytes.argtypes = [i] * 5
    L.kata_recur_spans.argtypes = [i]
    L.kata_recur_step.argtypes = [vp] * 8 + [i] * 2 + [ll] * 4 + [f, i, vp]
    for name in ("kata_conv_fwd", "kata_conv_step", "kata_conv_bwd_ws", "kata_qk_norm_fwd",
                 "kata_qk_norm_bwd_ws", "kata_ssm_fwd_ws", "kata_ssm_bwd_ws", "kata_ssm_step",
                 "kata_add_norm_fwd", "kata_add_norm_bwd_ws", "kata_f8_quant", "kata_f8_gemm_ws",
                 "kata_recur_fwd_ws", "kata_recur_bwd_ws", "kata_recur_spans", "kata_recur_step"):
        getattr(L, name).restype = i
    for name in ("kata_conv_bwd_workspace_bytes", "kata_qk_norm_bwd_workspace_bytes",
                 "kata_ssm_workspace_bytes", "kata_add_norm_bwd_workspace_bytes",
                 "kata_f8_gemm_workspace_bytes", "kata_recur_workspace_bytes"):
        getattr(L, name).restype = sz
    L.kata_status_string.argtypes = [i]
    L.kata_status_string.restype = ctypes.c_char_p
    L.kata_abi_version.argtypes = []
    L.kata_abi_version.restype = i
    _lib = L
    return L


def _status_name(s: int) -> str:
    try:
        return lib().kata_status_string(s).decode()
    except Exception:  # library not loadable: still report the number
        return f"status {s}"


def _check(status: int, what: str):
    if status != KATA_OK:
        raise KataError(status, what)


def packed_dim(d: int) -> int:
    return d * (d + 1) // 2


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return KATA_F32
    if t.dtype == torch.bfloat16:
        return KATA_BF16
    raise TypeError(f"q/k/v must be float32 or bfloat16, got {t.dtype}")


def _dev(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()  # the argtypes make it a void pointer


def _stream(stream, device):
    """The HIP stream handle to launch on.  The handle of the current stream is
    asked for as such: 0.1 us, where making a torch Stream object to read it
    from takes 2 us, a seventh of the smallest forward."""
    import torch
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream


def _qkv_shapes(q, k, v):
    qs, vs = q.shape, v.shape
    if len(qs) != 4 or k.shape != qs or len(vs) != 4 or vs[:3] != qs[:3]:
        raise ValueError(f"expected q,k [B,H,T,d] and v [B,H,T,dv]; got {tuple(qs)}, "
                         f"{tuple(k.shape)}, {tuple(vs)}")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k and v must share one dtype")
    B, H, T, d = qs
    return B, H, T, d, vs[3]


def workspace_bytes(B, H, T, d, dv, C, dtype_code, span_chunks=0) -> int:
    return int(lib().kata_fwd_workspace_bytes(B, H, T, d, dv, C, dtype_code, span_chunks))


def default_span(B, H, T, d, dv, C, dtype_code) -> int:
    return int(lib().kata_fwd_default_span(B, H, T, d, dv, C, dtype_code))


def fwd_form(B, H, T, d, dv, C, g, dtype_code, span_chunks=0) -> int:
    """FWD_STATES, FWD_QUADRATIC, or -1 (kata_fwd_form)."""
    return int(lib().kata_fwd_form(B, H, T, d, dv, C, g, dtype_code, span_chunks))


def fwd_chunked(q, k, v, C: int, span_chunks: int = 0, out=None, workspace=None, stream=None):
    """Causal KATA-M1 forward via kata_fwd_chunked_ws; returns out [B,H,T,dv] fp32.

    The workspace is a torch uint8 device tensor (allocated here if not given).
    """
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = workspace_bytes(B, H, T, d, dv, C, code, span_chunks)
    if nbytes == 0:
        # let the library report why
        _check(lib().kata_fwd_chunked_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                         _dev(out, "out"), B, H, T, d, dv, C, code,
                                         span_chunks, ctypes.c_void_p(0), 0,
                                         _stream(stream, q.device)), "kata_fwd_chunked_ws")
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    _check(lib().kata_fwd_chunked_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                     B, H, T, d, dv, C, code, span_chunks,
                                     _dev(workspace, "workspace"), workspace.numel(),
                                     _stream(stream, q.device)), "kata_fwd_chunked_ws")
    return out


def fwd_chunked_timed(q, k, v, C: int, events, span_chunks: int = 0, out=None, workspace=None,
                      stream=None):
    """fwd_chunked that also records 4 caller-created HIP events (a ctypes array
    of 4 void pointers) around the three stages on the launch stream."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = workspace_bytes(B, H, T, d, dv, C, code, span_chunks)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=q.device)
    _check(lib().kata_fwd_chunked_timed(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                        _dev(out, "out"), B, H, T, d, dv, C, code, span_chunks,
                                        _dev(workspace, "workspace"), workspace.numel(),
                                        events, _stream(stream, q.device)),
           "kata_fwd_chunked_timed")
    return out


def fwd_chunked_train(q, k, v, C: int, span_chunks: int = 0, out=None, den=None, workspace=None,
                      stream=None):
    """Forward via kata_fwd_chunked_train_ws, which also writes the row
    denominators D_t for the backward; returns (out [B,H,T,dv], den [B,H,T])
    fp32."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    if den is None:
        den = torch.empty((B, H, T), dtype=torch.float32, device=q.device)
    nbytes = workspace_bytes(B, H, T, d, dv, C, code, span_chunks)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    _check(lib().kata_fwd_chunked_train_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                           _dev(out, "out"), _dev(den, "den"), B, H, T, d, dv, C,
                                           code, span_chunks, _dev(workspace, "workspace"),
                                           workspace.numel(), _stream(stream, q.device)),
           "kata_fwd_chunked_train_ws")
    return out, den


def fwd_chunked_alloc(q, k, v, C: int, out=None, stream=None):
    """Causal forward via kata_fwd_chunked (library allocates its workspace
    stream-ordered); returns out [B,H,T,dv] fp32."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_fwd_chunked(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                  B, H, T, d, dv, C, code, _stream(stream, q.device)),
           "kata_fwd_chunked")
    return out


def noalloc_scratch_bytes() -> int:
    return int(lib().kata_noalloc_scratch_bytes())


def fwd_chunked_noalloc(q, k, v, C: int, out=None, stream=None):
    """Causal forward via kata_fwd_chunked_noalloc (workspace in the library's
    per-device scratch array, nothing allocated by the library); returns out
    [B,H,T,dv] fp32 (allocated here by torch if not given)."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_fwd_chunked_noalloc(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                          _dev(out, "out"), B, H, T, d, dv, C, code,
                                          _stream(stream, q.device)),
           "kata_fwd_chunked_noalloc")
    return out


def quadratic_workspace_bytes(B, H, T, d, dv, dtype_code) -> int:
    return int(lib().kata_fwd_quadratic_workspace_bytes(B, H, T, d, dv, dtype_code))


def fwd_quadratic(q, k, v, out=None, workspace=None, stream=None):
    """Causal KATA-M1 forward in the quadratic form via kata_fwd_quadratic_ws;
    returns out [B,H,T,dv] fp32.  The workspace (a torch uint8 device tensor)
    is allocated here if not given."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = quadratic_workspace_bytes(B, H, T, d, dv, code)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    _check(lib().kata_fwd_quadratic_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                       _dev(out, "out"), B, H, T, d, dv, code,
                                       _dev(workspace, "workspace"), workspace.numel(),
                                       _stream(stream, q.device)), "kata_fwd_quadratic_ws")
    return out


def fwd_quadratic_alloc(q, k, v, out=None, stream=None):
    """Quadratic forward via kata_fwd_quadratic (library allocates its
    workspace stream-ordered); returns out [B,H,T,dv] fp32."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_fwd_quadratic(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                    B, H, T, d, dv, code, _stream(stream, q.device)),
           "kata_fwd_quadratic")
    return out


def prefill_state(k, v, S=None, z=None, stream=None):
    """Packed state after all T tokens: S [B,H,n,dv], z [B,H,n] (fp32)."""
    import torch
    if k.dim() != 4 or v.dim() != 4 or v.shape[:3] != k.shape[:3] or k.dtype != v.dtype:
        raise ValueError("expected k [B,H,T,d] and v [B,H,T,dv] of one dtype")
    B, H, T, d = k.shape
    dv = v.shape[3]
    n = packed_dim(d)
    if S is None:
        S = torch.empty((B, H, n, dv), dtype=torch.float32, device=k.device)
    if z is None:
        z = torch.empty((B, H, n), dtype=torch.float32, device=k.device)
    _check(lib().kata_prefill_state(_dev(k, "k"), _dev(v, "v"), _dev(S, "S"), _dev(z, "z"),
                                    B, H, T, d, dv, _dtype_code(k), _stream(stream, k.device)),
           "kata_prefill_state")
    return S, z


def decode_step(S, z, q, k, v, out=None, stream=None):
    """One decode step (S, z updated in place); q, k [B,H,d], v [B,H,dv] -> out [B,H,dv]."""
    import torch
    if q.dim() != 3 or k.shape != q.shape or v.dim() != 3 or v.shape[:2] != q.shape[:2]:
        raise ValueError("expected q, k [B,H,d] and v [B,H,dv]")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k and v must share one dtype")
    B, H, d = q.shape
    dv = v.shape[2]
    if out is None:
        out = torch.empty((B, H, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_decode_step(_dev(S, "S"), _dev(z, "z"), _dev(q, "q"), _dev(k, "k"),
                                  _dev(v, "v"), _dev(out, "out"), B, H, d, dv, _dtype_code(q),
                                  _stream(stream, q.device)), "kata_decode_step")
    return out


# ---- KATA-Mg (g feature blocks of d/g coordinates; g = 1 is KATA-M1) ------------

def packed_dim_mg(d: int, g: int) -> int:
    m = d // g
    return g * (m * (m + 1) // 2)


def mg_workspace_bytes(B, H, T, d, dv, C, g, dtype_code, span_chunks=0) -> int:
    return int(lib().kata_mg_fwd_workspace_bytes(B, H, T, d, dv, C, g, dtype_code, span_chunks))


def mg_fwd_chunked(q, k, v, C: int, g: int, span_chunks: int = 0, out=None, workspace=None,
                   stream=None):
    """Causal KATA-Mg forward via kata_mg_fwd_chunked_ws; returns out [B,H,T,dv] fp32."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = mg_workspace_bytes(B, H, T, d, dv, C, g, code, span_chunks)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    _check(lib().kata_mg_fwd_chunked_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                        _dev(out, "out"), B, H, T, d, dv, C, g, code, span_chunks,
                                        _dev(workspace, "workspace"), workspace.numel(),
                                        _stream(stream, q.device)), "kata_mg_fwd_chunked_ws")
    return out


def mg_fwd_chunked_timed(q, k, v, C: int, g: int, events, span_chunks: int = 0, out=None,
                         workspace=None, stream=None):
    """mg_fwd_chunked that also records 4 caller-created HIP events around the
    three stages on the launch stream."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = mg_workspace_bytes(B, H, T, d, dv, C, g, code, span_chunks)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    _check(lib().kata_mg_fwd_chunked_timed(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                           _dev(out, "out"), B, H, T, d, dv, C, g, code,
                                           span_chunks, _dev(workspace, "workspace"),
                                           workspace.numel(), events, _stream(stream, q.device)),
           "kata_mg_fwd_chunked_timed")
    return out


def mg_fwd_chunked_alloc(q, k, v, C: int, g: int, out=None, stream=None):
    """KATA-Mg forward via kata_mg_fwd_chunked (stream-ordered library workspace)."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_mg_fwd_chunked(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                     B, H, T, d, dv, C, g, code, _stream(stream, q.device)),
           "kata_mg_fwd_chunked")
    return out


def mg_fwd_quadratic(q, k, v, g: int, out=None, workspace=None, stream=None):
    """KATA-Mg forward in the quadratic form via kata_mg_fwd_quadratic_ws."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = int(lib().kata_mg_fwd_quadratic_workspace_bytes(B, H, T, d, dv, g, code))
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    _check(lib().kata_mg_fwd_quadratic_ws(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"),
                                          _dev(out, "out"), B, H, T, d, dv, g, code,
                                          _dev(workspace, "workspace"), workspace.numel(),
                                          _stream(stream, q.device)), "kata_mg_fwd_quadratic_ws")
    return out


def mg_prefill_state(k, v, g: int, S=None, z=None, stream=None):
    """KATA-Mg packed state after all T tokens: S [B,H,n_g,dv], z [B,H,n_g] (fp32)."""
    import torch
    if k.dim() != 4 or v.dim() != 4 or v.shape[:3] != k.shape[:3] or k.dtype != v.dtype:
        raise ValueError("expected k [B,H,T,d] and v [B,H,T,dv] of one dtype")
    B, H, T, d = k.shape
    dv = v.shape[3]
    n = packed_dim_mg(d, g)
    if S is None:
        S = torch.empty((B, H, n, dv), dtype=torch.float32, device=k.device)
    if z is None:
        z = torch.empty((B, H, n), dtype=torch.float32, device=k.device)
    _check(lib().kata_mg_prefill_state(_dev(k, "k"), _dev(v, "v"), _dev(S, "S"), _dev(z, "z"),
                                       B, H, T, d, dv, g, _dtype_code(k),
                                       _stream(stream, k.device)), "kata_mg_prefill_state")
    return S, z


def mg_decode_step(S, z, q, k, v, g: int, out=None, stream=None):
    """One KATA-Mg decode step (S, z updated in place) -> out [B,H,dv]."""
    import torch
    if q.dim() != 3 or k.shape != q.shape or v.dim() != 3 or v.shape[:2] != q.shape[:2]:
        raise ValueError("expected q, k [B,H,d] and v [B,H,dv]")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k and v must share one dtype")
    B, H, d = q.shape
    dv = v.shape[2]
    if out is None:
        out = torch.empty((B, H, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_mg_decode_step(_dev(S, "S"), _dev(z, "z"), _dev(q, "q"), _dev(k, "k"),
                                     _dev(v, "v"), _dev(out, "out"), B, H, d, dv, g,
                                     _dtype_code(q), _stream(stream, q.device)),
           "kata_mg_decode_step")
    return out


# ---- linear features --------------------------------------------------------

def lin_dim(d: int, feature: int) -> int:
    return int(lib().kata_lin_dim(d, feature))


def lin_workspace_bytes(B, H, T, d, dv, C, feature, dtype_code, span_chunks=0) -> int:
    return int(lib().kata_lin_fwd_workspace_bytes(B, H, T, d, dv, C, feature, dtype_code,
                                                  span_chunks))


def lin_default_span(B, H, T, d, dv, C, feature, dtype_code) -> int:
    return int(lib().kata_lin_default_span(B, H, T, d, dv, C, feature, dtype_code))


def lin_fwd_chunked(q, k, v, C: int, feature: int, eps: float = 0.0, normalize: bool = True,
                    span_chunks: int = 0, out=None, workspace=None, stream=None, events=None):
    """Causal linear attention with a linear feature map via kata_lin_fwd_chunked_ws
    (or kata_lin_fwd_chunked_timed when `events`, a ctypes array of 4 HIP events,
    is given); returns out [B,H,T,dv] fp32."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    nbytes = lin_workspace_bytes(B, H, T, d, dv, C, feature, code, span_chunks)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    args = (_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"), B, H, T, d, dv, C,
            feature, float(eps), int(normalize), code, span_chunks, _dev(workspace, "workspace"),
            workspace.numel())
    if events is None:
        _check(lib().kata_lin_fwd_chunked_ws(*args, _stream(stream, q.device)),
               "kata_lin_fwd_chunked_ws")
    else:
        _check(lib().kata_lin_fwd_chunked_timed(*args, events, _stream(stream, q.device)),
               "kata_lin_fwd_chunked_timed")
    return out


def lin_fwd_chunked_alloc(q, k, v, C: int, feature: int, eps: float = 0.0,
                          normalize: bool = True, out=None, stream=None):
    """The same forward via kata_lin_fwd_chunked (stream-ordered library workspace)."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_lin_fwd_chunked(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                      B, H, T, d, dv, C, feature, float(eps), int(normalize),
                                      code, _stream(stream, q.device)), "kata_lin_fwd_chunked")
    return out


# ---- backward -----------------------------------------------------------------

def bwd_workspace_bytes(B, H, T, d, dv, C, g, dtype_code) -> int:
    return int(lib().kata_bwd_workspace_bytes(B, H, T, d, dv, C, g, dtype_code))


def bwd_fused_scan(B, H, T, d, dv, C, g, dtype_code) -> int:
    """1 when the chunk-state backward's state launches also scan
    (kata_bwd_fused_scan); bwd_form tells whether a call takes that form."""
    return int(lib().kata_bwd_fused_scan(B, H, T, d, dv, C, g, dtype_code))


def bwd_form(B, H, T, d, dv, C, g, dtype_code) -> int:
    """BWD_STATES, BWD_FUSED_STATES, BWD_QUADRATIC, or -1 (kata_bwd_form)."""
    return int(lib().kata_bwd_form(B, H, T, d, dv, C, g, dtype_code))


def bwd_chunked(q, k, v, out, dout, C: int, g: int = 1, workspace=None, stream=None,
                events=None, grads=None, den=None):
    """Gradients (dq, dk, dv) of the causal KATA-Mg forward (g = 1: M1) via
    kata_bwd_chunked_ws (or kata_bwd_chunked_timed when `events`, a ctypes
    array of 7 HIP events, is given; or kata_bwd_chunked_ex when `den`, the
    denominators from fwd_chunked_train, is given); fp32 tensors shaped like
    q, k, v."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    for name, t in (("out", out), ("dout", dout)):
        if t.dtype != torch.float32 or tuple(t.shape) != (B, H, T, dv):
            raise ValueError(f"{name} must be fp32 [B,H,T,dv]")
    if grads is None:
        grads = (torch.empty((B, H, T, d), dtype=torch.float32, device=q.device),
                 torch.empty((B, H, T, d), dtype=torch.float32, device=q.device),
                 torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device))
    dq, dk, dvv = grads
    nbytes = bwd_workspace_bytes(B, H, T, d, dv, C, g, code)
    if workspace is None or workspace.numel() < nbytes:
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=q.device)
    args = (_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"), _dev(dout, "dout"),
            _dev(dq, "dq"), _dev(dk, "dk"), _dev(dvv, "dv"), B, H, T, d, dv, C, g, code,
            _dev(workspace, "workspace"), workspace.numel())
    if den is not None:
        if den.dtype != torch.float32 or tuple(den.shape) != (B, H, T):
            raise ValueError("den must be fp32 [B,H,T]")
        args_ex = args[:5] + (_dev(den, "den"),) + args[5:]
        _check(lib().kata_bwd_chunked_ex(*args_ex, events if events is not None else None,
                                         _stream(stream, q.device)), "kata_bwd_chunked_ex")
    elif events is None:
        _check(lib().kata_bwd_chunked_ws(*args, _stream(stream, q.device)), "kata_bwd_chunked_ws")
    else:
        _check(lib().kata_bwd_chunked_timed(*args, events, _stream(stream, q.device)),
               "kata_bwd_chunked_timed")
    return dq, dk, dvv


def bwd_chunked_alloc(q, k, v, out, dout, C: int, g: int = 1, stream=None):
    """The same gradients via kata_bwd_chunked (stream-ordered library workspace)."""
    import torch
    B, H, T, d, dv = _qkv_shapes(q, k, v)
    code = _dtype_code(q)
    dq = torch.empty((B, H, T, d), dtype=torch.float32, device=q.device)
    dk = torch.empty((B, H, T, d), dtype=torch.float32, device=q.device)
    dvv = torch.empty((B, H, T, dv), dtype=torch.float32, device=q.device)
    _check(lib().kata_bwd_chunked(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"),
                                  _dev(dout, "dout"), _dev(dq, "dq"), _dev(dk, "dk"),
                                  _dev(dvv, "dv"), B, H, T, d, dv, C, g, code,
                                  _stream(stream, q.device)), "kata_bwd_chunked")
    return dq, dk, dvv


# ---- mixer operators ------------------------------------------------------------
# Activations are token-major and may be views with any strides over their outer
# dimensions; parameters and states are contiguous (fp32, a convolution's state in
# the activations' type).  Outputs are allocated where they are not given.

def _on_stream(call):
    """A call with stream=s runs as on s: the kernels there, and what torch
    allocates for them from s's memory.  The device of the first tensor is made the
    current one meanwhile, if it is not."""
    name = call.__code__.co_varnames[0]  # the first parameter's

    @functools.wraps(call)
    def run(*args, stream=None, **kw):
        import torch
        first = args[0] if args else kw.get(name)
        if first is None:
            raise TypeError(f"{call.__name__}() needs {name}")
        device = first.get_device()
        if device < 0:
            raise ValueError("expected device tensors")
        if stream is None:
            if device == torch._C._cuda_getDevice():
                return call(*args, **kw)
            with torch.cuda.device(first.device):
                return call(*args, **kw)
        if stream.device != first.device:
            raise ValueError(f"stream of {stream.device}, tensors of {first.device}")
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return run


_ANY = "any"  # strides over the innermost dimension too


def _tensor(t, name, device, shape, dtype, strided=False):
    """The address of a tensor of this shape (a tuple) and type on the device of this number.
    Few steps: of a single token's call these checks are half of the host's time."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        if t.shape != shape:
            raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        raise ValueError(f"{name} is on {t.device}, not on device {device}")
    if not t.is_contiguous():
        if not strided:
            raise ValueError(f"{name} must be contiguous")
        if strided is not _ANY and shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}'s innermost dimension must be contiguous")
    return t.data_ptr()


def _optional(t, name, device, shape, dtype, strided=False):
    return None if t is None else _tensor(t, name, device, shape, dtype, strided)


def _workspace(given, nbytes, like):
    import torch
    if given is None or given.numel() < nbytes:
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=like.device)
    _tensor(given, "workspace", like.get_device(), given.shape, torch.uint8)
    return given


def _dims(t, n, what):
    s = t.shape
    if len(s) != n:
        raise ValueError(f"expected {what}, got {tuple(s)}")
    return s


@_on_stream
def conv_fwd(x, w, bias=None, act: int = CONV_SILU, state=None, lengths=None, y=None,
             state_out=None, final_state: bool = False):
    """Causal depthwise convolution (kata_conv_fwd): x [B,T,D], w [D,W], bias [D]; returns y
    [B,T,D], or (y, state_out [B,W-1,D]) with final_state or a state_out.  state: the rows
    before x; lengths: int32 [B]."""
    import torch
    B, T, D = _dims(x, 3, "x [B,T,D]")
    W = _dims(w, 2, "w [D,W]")[1]
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    if y is None:
        y = torch.empty((B, T, D), dtype=x.dtype, device=x.device)
    if state_out is None and final_state:
        state_out = torch.empty((B, W - 1, D), dtype=x.dtype, device=x.device)
    rows = (B, W - 1, D)
    _check(lib().kata_conv_fwd(
        _tensor(x, "x", dev, (B, T, D), x.dtype, True), _tensor(w, "w", dev, (D, W), f32),
        _optional(bias, "bias", dev, (D,), f32), _optional(state, "state", dev, rows, x.dtype),
        _optional(lengths, "lengths", dev, (B,), torch.int32),
        _tensor(y, "y", dev, (B, T, D), x.dtype, True),
        _optional(state_out, "state_out", dev, rows, x.dtype), B, T, D, W, x.stride(0), x.stride(1),
        y.stride(0), y.stride(1), act, code, _stream(None, x.device)), "kata_conv_fwd")
    return y if state_out is None else (y, state_out)


@_on_stream
def conv_step(state, x, w, bias=None, act: int = CONV_SILU, y=None):
    """One token of every sequence (kata_conv_step): x [B,D] -> y [B,D]; state [B,W-1,D] is
    moved on in place."""
    import torch
    B, D = _dims(x, 2, "x [B,D]")
    W = _dims(w, 2, "w [D,W]")[1]
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    if y is None:
        y = torch.empty((B, D), dtype=x.dtype, device=x.device)
    _check(lib().kata_conv_step(
        _tensor(state, "state", dev, (B, W - 1, D), x.dtype),
        _tensor(x, "x", dev, (B, D), x.dtype, True), _tensor(w, "w", dev, (D, W), f32),
        _optional(bias, "bias", dev, (D,), f32), _tensor(y, "y", dev, (B, D), x.dtype, True), B, D, W,
        x.stride(0), y.stride(0), act, code, _stream(None, x.device)), "kata_conv_step")
    return y


@_on_stream
def conv_bwd(x, w, bias, dy, act: int = CONV_SILU, dx=None, workspace=None):
    """Gradients (dx, dw, dbias) of conv_fwd without state and lengths
    (kata_conv_bwd_ws); dbias is None where bias is."""
    import torch
    B, T, D = _dims(x, 3, "x [B,T,D]")
    W = _dims(w, 2, "w [D,W]")[1]
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    if dx is None:
        dx = torch.empty((B, T, D), dtype=x.dtype, device=x.device)
    dw = torch.empty((D, W), dtype=f32, device=x.device)
    db = None if bias is None else torch.empty((D,), dtype=f32, device=x.device)
    nbytes = int(lib().kata_conv_bwd_workspace_bytes(B, T, D, W, code))
    workspace = _workspace(workspace, nbytes, x)
    _check(lib().kata_conv_bwd_ws(
        _tensor(x, "x", dev, (B, T, D), x.dtype, True), _tensor(w, "w", dev, (D, W), f32),
        _optional(bias, "bias", dev, (D,), f32), _tensor(dy, "dy", dev, (B, T, D), x.dtype, True),
        _tensor(dx, "dx", dev, (B, T, D), x.dtype, True), dw.data_ptr(),
        None if db is None else db.data_ptr(), B, T, D, W, x.stride(0), x.stride(1), dy.stride(0),
        dy.stride(1), dx.stride(0), dx.stride(1), act, code, workspace.data_ptr(),
        workspace.numel(), _stream(None, x.device)), "kata_conv_bwd_ws")
    return dx, dw, db


def rope_frequencies(r: int, base: float = 10000.0, device="cuda"):
    """The fp64 frequencies base^(-2i/r), i < r/2, of a rotation of r coordinates."""
    import torch
    i = torch.arange(r // 2, dtype=torch.float64, device=device)
    return base ** (-2.0 * i / max(r, 1))


def _norm_sides(q, k, freq):
    B, T, Hq, d = _dims(q, 4, "q [B,T,Hq,d]")
    Hk = 0
    if k is not None:
        Hk = _dims(k, 4, "k [B,T,Hk,d]")[2]
    return B, T, Hq, Hk, d, 0 if freq is None else 2 * freq.shape[0]


def _strides3(t):
    return (0, 0, 0) if t is None else t.stride()[:3]


@_on_stream
def qk_norm_fwd(q, k=None, wq=None, wk=None, freq=None, pos=None, norm: int = NORM_RMS,
                eps: float = 1e-6, pairs: bool = False, yq=None, yk=None):
    """Norms of query and key heads with the position rotation (kata_qk_norm_fwd): q
    [B,T,Hq,d], k [B,T,Hk,d] (or None), weights [d], freq fp64 [r/2], pos int32 [B,T]
    (default 0..T-1); returns (yq [B,Hq,T,d], yk [B,Hk,T,d] or None)."""
    import torch
    B, T, Hq, Hk, d, r = _norm_sides(q, k, freq)
    code, f32, dev = _dtype_code(q), torch.float32, q.get_device()
    if yq is None:
        yq = torch.empty((B, Hq, T, d), dtype=q.dtype, device=q.device)
    if yk is None and k is not None:
        yk = torch.empty((B, Hk, T, d), dtype=q.dtype, device=q.device)
    _check(lib().kata_qk_norm_fwd(
        _tensor(q, "q", dev, (B, T, Hq, d), q.dtype, True),
        _optional(k, "k", dev, (B, T, Hk, d), q.dtype, True), _optional(wq, "wq", dev, (d,), f32),
        _optional(wk, "wk", dev, (d,), f32), _optional(pos, "pos", dev, (B, T), torch.int32),
        _optional(freq if r else None, "freq", dev, (r // 2,), torch.float64),
        _tensor(yq, "yq", dev, (B, Hq, T, d), q.dtype),
        _optional(yk, "yk", dev, (B, Hk, T, d), q.dtype), B, T, Hq, Hk, d, r, *_strides3(q),
        *_strides3(k), norm, eps, int(pairs), code, _stream(None, q.device)), "kata_qk_norm_fwd")
    return yq, yk


@_on_stream
def qk_norm_bwd(q, k=None, wq=None, wk=None, freq=None, dq=None, dk=None, pos=None,
                norm: int = NORM_RMS, eps: float = 1e-6, pairs: bool = False, dxq=None, dxk=None,
                workspace=None):
    """Gradients (dxq, dxk, dwq, dwk) of qk_norm_fwd from dq [B,Hq,T,d] and dk [B,Hk,T,d] (fp32
    or q's type), via kata_qk_norm_bwd_ws; None where the input is."""
    import torch
    B, T, Hq, Hk, d, r = _norm_sides(q, k, freq)
    if dq is None or (k is None) != (dk is None):
        raise ValueError("expected dq, and dk where there is k")
    code, f32, dev = _dtype_code(q), torch.float32, q.get_device()
    if dxq is None:
        dxq = torch.empty((B, T, Hq, d), dtype=q.dtype, device=q.device)
    if dxk is None and k is not None:
        dxk = torch.empty((B, T, Hk, d), dtype=q.dtype, device=q.device)
    dwq = None if wq is None else torch.empty((d,), dtype=f32, device=q.device)
    dwk = None if wk is None else torch.empty((d,), dtype=f32, device=q.device)
    nbytes = int(lib().kata_qk_norm_bwd_workspace_bytes(B, T, Hq, Hk, d, code))
    workspace = _workspace(workspace, nbytes, q)
    _check(lib().kata_qk_norm_bwd_ws(
        _tensor(q, "q", dev, (B, T, Hq, d), q.dtype, True),
        _optional(k, "k", dev, (B, T, Hk, d), q.dtype, True), _optional(wq, "wq", dev, (d,), f32),
        _optional(wk, "wk", dev, (d,), f32), _optional(pos, "pos", dev, (B, T), torch.int32),
        _optional(freq if r else None, "freq", dev, (r // 2,), torch.float64),
        _tensor(dq, "dq", dev, (B, Hq, T, d), dq.dtype),
        _optional(dk, "dk", dev, (B, Hk, T, d), dq.dtype),
        _tensor(dxq, "dxq", dev, (B, T, Hq, d), q.dtype, True),
        _optional(dxk, "dxk", dev, (B, T, Hk, d), q.dtype, True),
        None if dwq is None else dwq.data_ptr(), None if dwk is None else dwk.data_ptr(), B, T, Hq,
        Hk, d, r, *_strides3(q), *_strides3(k), *_strides3(dxq), *_strides3(dxk), norm, eps,
        int(pairs), code, _dtype_code(dq), workspace.data_ptr(), workspace.numel(),
        _stream(None, q.device)), "kata_qk_norm_bwd_ws")
    return dxq, dxk, dwq, dwk


_SsmStrides = ctypes.c_longlong * 15  # kata_ssm_strides_t


def _ssm_inputs(x, dt, A, Bm, Cm, D, dt_bias, tokens):
    """Sizes, and the addresses of the inputs in the order of the entry points; tokens: whether
    the activations have a token dimension."""
    import torch
    n = 4 if tokens else 3
    lead, (H, P) = x.shape[:-2], _dims(x, n, "x [B,T,H,P]" if tokens else "x [B,H,P]")[-2:]
    G, N = _dims(Bm, n, "Bm [B,T,G,N]" if tokens else "Bm [B,G,N]")[-2:]
    f32, dev = torch.float32, x.get_device()
    args = (_tensor(x, "x", dev, x.shape, x.dtype, True),
            _tensor(dt, "dt", dev, (*lead, H), x.dtype, _ANY),
            _tensor(A, "A", dev, (H,), f32), _tensor(Bm, "Bm", dev, (*lead, G, N), x.dtype, True),
            _tensor(Cm, "Cm", dev, (*lead, G, N), x.dtype, True), _optional(D, "D", dev, (H,), f32),
            _optional(dt_bias, "dt_bias", dev, (H,), f32))
    return lead[0], lead[1] if tokens else 1, H, G, N, P, args


def _ssm_strides(x, dt, Bm, Cm, y):
    if x.dim() == 3:  # one token
        (xb, xh, _), (tb, th), (bb, bg, _), (cb, cg, _), (yb, yh, _) = (
            x.stride(), dt.stride(), Bm.stride(), Cm.stride(), y.stride())
        s = (xb, 0, xh, tb, 0, th, bb, 0, bg, cb, 0, cg, yb, 0, yh)
    else:
        s = x.stride()[:3] + dt.stride() + Bm.stride()[:3] + Cm.stride()[:3] + y.stride()[:3]
    return _SsmStrides(*s)


def ssm_workspace_bytes(B, T, H, G, N, P, dtype_code, backward=False) -> int:
    return int(lib().kata_ssm_workspace_bytes(B, T, H, G, N, P, dtype_code, int(backward)))


@_on_stream
def ssm_fwd(x, dt, A, Bm, Cm, D=None, dt_bias=None, softplus: bool = True, state=None,
            lengths=None, y=None, state_out=None, final_state: bool = False, workspace=None):
    """Selective scan (kata_ssm_fwd_ws): x [B,T,H,P], dt [B,T,H], A [H], Bm and Cm [B,T,G,N], D
    and dt_bias [H]; returns y [B,T,H,P], or (y, state_out [B,H,N,P] fp32) with final_state
    or a state_out.  state: the one before the first token; lengths: int32 [B]."""
    import torch
    B, T, H, G, N, P, args = _ssm_inputs(x, dt, A, Bm, Cm, D, dt_bias, True)
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    if y is None:
        y = torch.empty((B, T, H, P), dtype=x.dtype, device=x.device)
    if state_out is None and final_state:
        state_out = torch.empty((B, H, N, P), dtype=f32, device=x.device)
    workspace = _workspace(workspace, ssm_workspace_bytes(B, T, H, G, N, P, code), x)
    _check(lib().kata_ssm_fwd_ws(
        *args, _optional(state, "state", dev, (B, H, N, P), f32),
        _optional(lengths, "lengths", dev, (B,), torch.int32),
        _tensor(y, "y", dev, (B, T, H, P), x.dtype, True),
        _optional(state_out, "state_out", dev, (B, H, N, P), f32), B, T, H, G, N, P,
        _ssm_strides(x, dt, Bm, Cm, y), int(softplus), code, workspace.data_ptr(),
        workspace.numel(), _stream(None, x.device)), "kata_ssm_fwd_ws")
    return y if state_out is None else (y, state_out)


@_on_stream
def ssm_step(S, x, dt, A, Bm, Cm, D=None, dt_bias=None, softplus: bool = True, y=None):
    """One token of every sequence (kata_ssm_step): x [B,H,P], dt [B,H], Bm and Cm [B,G,N] -> y
    [B,H,P]; S [B,H,N,P] fp32 is updated in place."""
    import torch
    B, _, H, G, N, P, args = _ssm_inputs(x, dt, A, Bm, Cm, D, dt_bias, False)
    code, dev = _dtype_code(x), x.get_device()
    if y is None:
        y = torch.empty((B, H, P), dtype=x.dtype, device=x.device)
    _check(lib().kata_ssm_step(
        _tensor(S, "S", dev, (B, H, N, P), torch.float32), *args,
        _tensor(y, "y", dev, (B, H, P), x.dtype, True), B, H, G, N, P,
        _ssm_strides(x, dt, Bm, Cm, y), int(softplus), code, _stream(None, x.device)),
        "kata_ssm_step")
    return y


@_on_stream
def ssm_bwd(x, dt, A, Bm, Cm, D, dt_bias, dy, softplus: bool = True, workspace=None):
    """Gradients (dx, ddt, dA, dBm, dCm, dD, dt_dbias) of ssm_fwd from a zero state without
    lengths (kata_ssm_bwd_ws); None where D or dt_bias is."""
    import torch
    B, T, H, G, N, P, args = _ssm_inputs(x, dt, A, Bm, Cm, D, dt_bias, True)
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    dx, ddt = (torch.empty(s, dtype=x.dtype, device=x.device) for s in ((B, T, H, P), (B, T, H)))
    dB, dC = (torch.empty((B, T, G, N), dtype=x.dtype, device=x.device) for _ in range(2))
    dA = torch.empty((H,), dtype=f32, device=x.device)
    dD = None if D is None else torch.empty((H,), dtype=f32, device=x.device)
    db = None if dt_bias is None else torch.empty((H,), dtype=f32, device=x.device)
    workspace = _workspace(workspace, ssm_workspace_bytes(B, T, H, G, N, P, code, True), x)
    _check(lib().kata_ssm_bwd_ws(
        *args, _tensor(dy, "dy", dev, (B, T, H, P), x.dtype, True), dx.data_ptr(), ddt.data_ptr(),
        dA.data_ptr(), dB.data_ptr(), dC.data_ptr(), None if dD is None else dD.data_ptr(),
        None if db is None else db.data_ptr(), B, T, H, G, N, P,
        _ssm_strides(x, dt, Bm, Cm, dy), int(softplus), code, workspace.data_ptr(),
        workspace.numel(), _stream(None, x.device)), "kata_ssm_bwd_ws")
    return dx, ddt, dA, dB, dC, dD, db


# ---- a layer in 8 bits ------------------------------------------------------------
# Rows [..,D] may have any leading dimensions that lie one after the other in memory (one row
# stride).  Codes are torch.float8_e4m3fn; those that are allocated here begin each row at a
# multiple of 16 bytes, as the product's fast forms ask for.

F8_BLOCK = 128  # columns (and rows) of a scale


def _rows(t, what):
    """Rows, width and row stride of t [..,D]."""
    s = t.shape
    n = len(s)
    if n == 2:
        return s[0], s[1], t.stride(0)
    if n < 2:
        raise ValueError(f"expected {what}, got {tuple(s)}")
    strides, rows, step = t.stride(), 1, None
    for k in range(n - 2, -1, -1):
        if s[k] == 1:
            continue
        if step is None:
            step = strides[k]
        elif strides[k] != step * rows:
            raise ValueError(f"{what}: leading dimensions {tuple(s[:-1])} are not rows of one stride")
        rows *= s[k]
    return rows, s[-1], s[-1] if step is None else step


def _row_of(t, name, device, shape, dtype):
    """The address and the row stride of a tensor of rows (None: none)."""
    if t is None:
        return None, 0
    if t.is_contiguous() and t.shape == shape and t.dtype is dtype and t.get_device() == device:
        return t.data_ptr(), shape[-1]
    return _tensor(t, name, device, shape, dtype, True), _rows(t, name)[2]


def _like(t):
    """An uninitialised contiguous tensor like t."""
    import torch
    if t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _codes(lead, n, device):
    import torch
    if n % 16 == 0:
        return torch.empty((*lead, n), dtype=torch.float8_e4m3fn, device=device)
    return torch.empty((*lead, (n + 15) // 16 * 16), dtype=torch.float8_e4m3fn, device=device)[..., :n]


def _f8_blocks(n):
    return (n + F8_BLOCK - 1) // F8_BLOCK


def _add_norm(x, w, res, eps, y, sum, q, scale):
    import torch
    M, D, x_row = _rows(x, "x [..,D]")
    code, f32, dev, shape, T = _dtype_code(x), torch.float32, x.get_device(), x.shape, x.dtype
    if res is None:
        if sum is not None:
            raise ValueError("sum without res is x itself")
    elif sum is None:
        sum = _like(x)
    res_at, res_row = _row_of(res, "res", dev, shape, T)
    sum_at, sum_row = _row_of(sum, "sum", dev, shape, T)
    y_at, y_row = _row_of(y, "y", dev, shape, T)
    q_at, q_row = _row_of(q, "q", dev, shape, torch.float8_e4m3fn)
    _check(lib().kata_add_norm_fwd(
        _tensor(x, "x", dev, shape, T, True), res_at, _optional(w, "w", dev, (D,), f32), sum_at, y_at,
        q_at, _optional(scale, "scale", dev, (*shape[:-1], _f8_blocks(D)), f32), M, D, x_row, res_row,
        sum_row, y_row, q_row, eps, code, _stream(None, x.device)), "kata_add_norm_fwd")
    return x if sum is None else sum


@_on_stream
def add_norm_fwd(x, w=None, res=None, eps: float = 1e-6, y=None, sum=None):
    """Root-mean-square norm of x + res (kata_add_norm_fwd): x, res [..,D], w [D] fp32; returns (y,
    sum), sum being x + res in x's type (x itself without res; it may be given as res)."""
    if y is None:
        y = _like(x)
    return y, _add_norm(x, w, res, eps, y, sum, None, None)


@_on_stream
def add_norm_f8_fwd(x, w=None, res=None, eps: float = 1e-6, q=None, scale=None, sum=None, y=None):
    """The same with its output in 8 bits: returns (q, scale, sum), scale fp32
    [..,ceil(D/128)].  y: where given, receives the output in x's type too."""
    import torch
    if x.dim() < 2:
        raise ValueError(f"expected x [..,D], got {tuple(x.shape)}")
    lead, D = x.shape[:-1], x.shape[-1]
    if q is None:
        q = _codes(lead, D, x.device)
    if scale is None:
        scale = torch.empty((*lead, _f8_blocks(D)), dtype=torch.float32, device=x.device)
    return q, scale, _add_norm(x, w, res, eps, y, sum, q, scale)


@_on_stream
def add_norm_bwd(sum, w, dy, dsum=None, eps: float = 1e-6, dx=None, workspace=None):
    """Gradients (dx, dw) of add_norm_fwd (kata_add_norm_bwd_ws) from its sum, dy [..,D] (fp32 or
    sum's type) and dsum, the gradient of sum itself; dx is that of x and of res.  dw is
    None where w is."""
    import torch
    M, D, row = _rows(sum, "sum [..,D]")
    code, f32, dev, shape, T = _dtype_code(sum), torch.float32, sum.get_device(), sum.shape, sum.dtype
    if dx is None:
        dx = _like(sum)
    dw = None if w is None else torch.empty((D,), dtype=f32, device=sum.device)
    workspace = _workspace(workspace, int(lib().kata_add_norm_bwd_workspace_bytes(M, D, code)), sum)
    dy_at, dy_row = _row_of(dy, "dy", dev, shape, dy.dtype)
    dsum_at, dsum_row = _row_of(dsum, "dsum", dev, shape, T)
    dx_at, dx_row = _row_of(dx, "dx", dev, shape, T)
    _check(lib().kata_add_norm_bwd_ws(
        _tensor(sum, "sum", dev, shape, T, True), _optional(w, "w", dev, (D,), f32), dy_at, dsum_at,
        dx_at, None if dw is None else dw.data_ptr(), M, D, row, dy_row, dsum_row, dx_row, eps, code,
        _dtype_code(dy), workspace.data_ptr(), workspace.numel(), _stream(None, sum.device)),
        "kata_add_norm_bwd_ws")
    return dx, dw


@_on_stream
def f8_quant(x, rows: int = 1, transposed: bool = False, q=None, scale=None, qt=None,
             scale_t=None):
    """x [..,K] in 8 bits (kata_f8_quant), blocks of rows (1 or 128) x 128: returns (q [..,K],
    scale), and with transposed (q, scale, qt [K,M], scale_t), M being x's rows.  The scale is
    fp32 [..,ceil(K/128)] for rows = 1, [ceil(M/128),ceil(K/128)] for rows = 128."""
    import torch
    M, K, x_row = _rows(x, "x [..,K]")
    code, f32, dev, f8 = _dtype_code(x), torch.float32, x.get_device(), torch.float8_e4m3fn
    if rows not in (1, F8_BLOCK):
        raise ValueError(f"rows must be 1 or {F8_BLOCK}, got {rows}")
    of = (*x.shape[:-1], _f8_blocks(K)) if rows == 1 else (_f8_blocks(M), _f8_blocks(K))
    of_t = (K if rows == 1 else _f8_blocks(K), _f8_blocks(M))
    if q is None:
        q = _codes(x.shape[:-1], K, x.device)
    if scale is None:
        scale = torch.empty(of, dtype=f32, device=x.device)
    if not transposed and (qt is not None or scale_t is not None):
        raise ValueError("qt and scale_t are for transposed")
    if transposed and qt is None:
        qt = _codes((K,), M, x.device)
    if transposed and scale_t is None:
        scale_t = torch.empty(of_t, dtype=f32, device=x.device)
    q_at, q_row = _row_of(q, "q", dev, x.shape, f8)
    _check(lib().kata_f8_quant(
        _tensor(x, "x", dev, x.shape, x.dtype, True), q_at, _tensor(scale, "scale", dev, of, f32), _optional(qt, "qt", dev, (K, M), f8, True),
        _optional(scale_t, "scale_t", dev, of_t, f32), M, K, rows, x_row, q_row,
        0 if qt is None else qt.stride(0), code, _stream(None, x.device)), "kata_f8_quant")
    return (q, scale, qt, scale_t) if transposed else (q, scale)


@_on_stream
def f8_gemm(a, a_scale, b, b_scale, out=None, dtype=None, workspace=None):
    """a b^T of 8-bit operands (kata_f8_gemm_ws): a [..,K] with a_scale [..,ceil(K/128)], b [N,K]
    with b_scale [ceil(N/128),ceil(K/128)] (128 x 128 blocks) or [N,ceil(K/128)] (blocks of a
    row); returns [..,N] in dtype: bf16 (the default), whose products keep 13 bits of the largest
    of eight, or fp32, whose products are exact."""
    import torch
    M, K, a_row = _rows(a, "a [..,K]")
    N, Kb = _dims(b, 2, "b [N,K]")
    f32, dev, f8, kb = torch.float32, a.get_device(), torch.float8_e4m3fn, _f8_blocks(K)
    if Kb != K:
        raise ValueError(f"a has {K} columns, b {Kb}")
    shape = (*a.shape[:-1], N)
    if out is None:
        out = torch.empty(shape, dtype=torch.bfloat16 if dtype is None else dtype, device=a.device)
    elif dtype is not None and out.dtype is not dtype:
        raise TypeError(f"out must be {dtype}, got {out.dtype}")
    code = _dtype_code(out)
    out_at, out_row = _row_of(out, "out", dev, shape, out.dtype)
    by_row = N > 1 and b_scale.shape == (N, kb)
    workspace = _workspace(workspace, int(lib().kata_f8_gemm_workspace_bytes(M, N, K)), a)
    _check(lib().kata_f8_gemm_ws(
        _tensor(a, "a", dev, a.shape, f8, True),
        _tensor(a_scale, "a_scale", dev, (*a.shape[:-1], kb), f32),
        _tensor(b, "b", dev, (N, K), f8, True),
        _tensor(b_scale, "b_scale", dev, (N, kb) if by_row else (_f8_blocks(N), kb), f32),
        out_at, M, N, K, 1 if by_row else F8_BLOCK, a_row, b.stride(0), out_row, code, workspace.data_ptr(), workspace.numel(),
        _stream(None, a.device)), "kata_f8_gemm_ws")
    return out


# ---- gated linear recurrence ----------------------------------------------------------

_RecurStrides = ctypes.c_longlong * 14  # kata_recur_strides_t


def _recur_inputs(x, r, i, lam, r_bias, i_bias):
    """The addresses of the inputs in the order of the entry points."""
    import torch
    f32, dev, D = torch.float32, x.get_device(), x.shape[-1]
    return (_tensor(x, "x", dev, x.shape, x.dtype, True), _tensor(r, "r", dev, x.shape, x.dtype, True),
            _tensor(i, "i", dev, x.shape, x.dtype, True), _tensor(lam, "lam", dev, (D,), f32),
            _optional(r_bias, "r_bias", dev, (D,), f32), _optional(i_bias, "i_bias", dev, (D,), f32))


def _recur_strides(*tensors):
    s = [v for t in tensors for v in t.stride()[:2]]
    return _RecurStrides(*s, *([0] * (14 - len(s))))


def recur_workspace_bytes(B, T, D, dtype_code, backward=False) -> int:
    return int(lib().kata_recur_workspace_bytes(B, T, D, dtype_code, int(backward)))


def _recur_fwd(x, r, i, lam, r_bias, i_bias, c, state, lengths, y, state_out, starts, workspace):
    import torch
    B, T, D = _dims(x, 3, "x [B,T,D]")
    code, f32, dev = _dtype_code(x), torch.float32, x.get_device()
    if y is None:
        y = torch.empty((B, T, D), dtype=x.dtype, device=x.device)
    workspace = _workspace(workspace, recur_workspace_bytes(B, T, D, code), x)
    _check(lib().kata_recur_fwd_ws(
        *_recur_inputs(x, r, i, lam, r_bias, i_bias), _optional(state, "state", dev, (B, D), f32),
        _optional(lengths, "lengths", dev, (B,), torch.int32),
        _tensor(y, "y", dev, (B, T, D), x.dtype, True),
        _optional(state_out, "state_out", dev, (B, D), f32), None if starts is None else starts.data_ptr(),
        B, T, D, _recur_strides(x, r, i, y), c, code, workspace.data_ptr(), workspace.numel(),
        _stream(None, x.device)), "kata_recur_fwd_ws")
    return y


@_on_stream
def recur_fwd(x, r, i, lam, r_bias=None, i_bias=None, c: float = 8.0, state=None, lengths=None,
              y=None, state_out=None, final_state: bool = False, workspace=None):
    """Gated linear recurrence (kata_recur_fwd_ws): x and the gates' r, i [B,T,D], lam, r_bias, i_bias
    [D] fp32; returns y [B,T,D], or (y, state_out [B,D] fp32) with final_state or a state_out.
    state: the one before the first token; lengths: int32 [B]."""
    import torch
    if state_out is None and final_state:
        B, _, D = _dims(x, 3, "x [B,T,D]")
        state_out = torch.empty((B, D), dtype=torch.float32, device=x.device)
    y = _recur_fwd(x, r, i, lam, r_bias, i_bias, c, state, lengths, y, state_out, None, workspace)
    return y if state_out is None else (y, state_out)


@_on_stream
def recur_fwd_train(x, r, i, lam, r_bias=None, i_bias=None, c: float = 8.0, state=None,
                    lengths=None, y=None, state_out=None, workspace=None):
    """recur_fwd that also returns what recur_bwd takes: (y, starts)."""
    import torch
    B, T, D = _dims(x, 3, "x [B,T,D]")
    starts = torch.empty((B, int(lib().kata_recur_spans(T)), D), dtype=torch.float32, device=x.device)
    y = _recur_fwd(x, r, i, lam, r_bias, i_bias, c, state, lengths, y, state_out, starts, workspace)
    return y, starts


@_on_stream
def recur_step(h, x, r, i, lam, r_bias=None, i_bias=None, c: float = 8.0, y=None):
    """One token of every sequence (kata_recur_step): x, r, i [B,D] -> y [B,D]; h [B,D] fp32 is
    updated in place."""
    import torch
    B, D = _dims(x, 2, "x [B,D]")
    code, dev = _dtype_code(x), x.get_device()
    if y is None:
        y = torch.empty((B, D), dtype=x.dtype, device=x.device)
    _check(lib().kata_recur_step(
        _tensor(h, "h", dev, (B, D), torch.float32), *_recur_inputs(x, r, i, lam, r_bias, i_bias),
        _tensor(y, "y", dev, (B, D), x.dtype, True), B, D, x.stride(0), r.stride(0), i.stride(0),
        y.stride(0), c, code, _stream(None, x.device)), "kata_recur_step")
    return y


@_on_stream
def recur_bwd(x, r, i, lam, r_bias, i_bias, dy, starts=None, c: float = 8.0, state=None,
              lengths=None, dstate=None, dx=None, dr=None, di=None, dstate_in=None,
              workspace=None):
    """Gradients (dx, dr, di, dlam, dr_bias, di_bias) of recur_fwd (kata_recur_bwd_ws) from dy [B,T,D];
    None where a bias is.  starts: recur_fwd_train's, or None (formed again); state and lengths as
    in the forward; dstate: the gradient of its state_out; dstate_in: where given, receives that
    of its state.  dx, dr, di may be given as views of one wider tensor; past a sequence's
    length they are not written."""
    import torch
    B, T, D = _dims(x, 3, "x [B,T,D]")
    code, f32, dev, shape, kind = _dtype_code(x), torch.float32, x.get_device(), (B, T, D), x.dtype
    # past a sequence's length: zeros, where the tensors are made here
    make = torch.empty if lengths is None else torch.zeros
    dx, dr, di = (make(shape, dtype=kind, device=x.device) if t is None else t for t in (dx, dr, di))
    dlam, drb, dib = (None if t is None else torch.empty((D,), dtype=f32, device=x.device)
                      for t in (lam, r_bias, i_bias))
    workspace = _workspace(workspace, recur_workspace_bytes(B, T, D, code, True), x)
    spans = int(lib().kata_recur_spans(T))
    _check(lib().kata_recur_bwd_ws(
        *_recur_inputs(x, r, i, lam, r_bias, i_bias), _optional(state, "state", dev, (B, D), f32),
        _optional(lengths, "lengths", dev, (B,), torch.int32),
        _optional(starts, "starts", dev, (B, spans, D), f32), _tensor(dy, "dy", dev, shape, kind, True),
        _optional(dstate, "dstate", dev, (B, D), f32), _tensor(dx, "dx", dev, shape, kind, True),
        _tensor(dr, "dr", dev, shape, kind, True), _tensor(di, "di", dev, shape, kind, True),
        dlam.data_ptr(), None if drb is None else drb.data_ptr(),
        None if dib is None else dib.data_ptr(), _optional(dstate_in, "dstate_in", dev, (B, D), f32), B,
        T, D, _recur_strides(x, r, i, dy, dx, dr, di), c, code, workspace.data_ptr(),
        workspace.numel(), _stream(None, x.device)), "kata_recur_bwd_ws")
    return dx, dr, di, dlam, drb, dib
