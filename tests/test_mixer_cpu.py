"""The mixer operators on the CPU: the fp64 reference's gradients against
differences, and what the C ABI refuses before it touches a GPU."""
from __future__ import annotations

import ctypes

import pytest
import torch

import mixer_reference as ref
import paper_2607_17419_amd as kata

FAKE = ctypes.c_void_p(0x10000)   # aligned, never dereferenced: validation fails first
FAKE2 = ctypes.c_void_p(0x20000)
FAKE3 = ctypes.c_void_p(0x30000)
WS = ctypes.c_void_p(0x100000)
NUL = ctypes.c_void_p(0)


# ---- the reference's gradients ------------------------------------------------------

def _directional(f, leaves, seed):
    """d/dh of f(leaves + h v) at 0: autograd's and the central difference's.  fp64: at
    h = 1e-5 the difference is off by about h^2 and by 1e-16 / h."""
    gen = torch.Generator().manual_seed(seed)
    vs = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in leaves]
    live = [t.clone().requires_grad_() for t in leaves]
    out = f(*live)
    dy = torch.randn(out.shape, generator=gen, dtype=torch.float64)
    grads = torch.autograd.grad(out, live, dy)
    exact = sum(float((g * v).sum()) for g, v in zip(grads, vs))
    h = 1e-5
    up, down = (f(*[t + s * h * v for t, v in zip(leaves, vs)]) for s in (1, -1))
    return exact, float((dy * (up - down)).sum()) / (2 * h)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


def test_reference_gradients_are_the_differences():
    gen = torch.Generator().manual_seed(0)
    x, w, b = _normal(gen, 2, 9, 5), _normal(gen, 5, 4), _normal(gen, 5)
    cases = [(lambda x, w, b: ref.conv(x, w, b)[0], (x, w, b))]
    q, wq, pos = _normal(gen, 2, 6, 3, 10), _normal(gen, 10), torch.arange(6).expand(2, 6)
    freq = torch.tensor([1.0, 0.1, 0.01], dtype=torch.float64)
    for kind in (0, 1, 2):
        for pairs in (False, True):
            cases.append((lambda q, wq, k=kind, p=pairs: ref.norm(q, wq, freq, pos, k, 1e-3, p),
                          (q, wq)))
    x, dt = _normal(gen, 2, 11, 4, 3), _normal(gen, 2, 11, 4)
    Bm, Cm, D, bias = _normal(gen, 2, 11, 2, 5), _normal(gen, 2, 11, 2, 5), _normal(gen, 4), None
    A = -torch.rand(4, generator=gen, dtype=torch.float64)
    cases.append((lambda *a: ref.scan(*a)[0], (x, dt, A, Bm, Cm, D, _normal(gen, 4))))
    cases.append((lambda *a: ref.scan(*a, soft=False)[0], (x, dt.abs(), A, Bm, Cm)))
    for i, (f, leaves) in enumerate(cases):
        exact, diff = _directional(f, leaves, i)
        assert abs(exact - diff) <= 1e-7 * (1 + abs(exact)), (i, exact, diff)


# ---- refusals -----------------------------------------------------------------------

def _conv_fwd(x=FAKE, w=FAKE, bias=NUL, s_in=NUL, lengths=NUL, y=FAKE2, s_out=NUL, B=2, T=8, D=16,
              W=4, xb=128, xt=16, yb=128, yt=16, act=1, dtype=1):
    return kata.lib().kata_conv_fwd(x, w, bias, s_in, lengths, y, s_out, B, T, D, W, xb, xt, yb, yt,
                                    act, dtype, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(x=NUL), 1), (dict(w=NUL), 1), (dict(y=NUL), 1), (dict(B=0), 1), (dict(T=0), 1),
    (dict(D=0), 1), (dict(W=0), 1), (dict(dtype=2), 1), (dict(act=2), 1), (dict(y=FAKE), 1),
    (dict(x=ctypes.c_void_p(0x10001)), 1), (dict(w=ctypes.c_void_p(0x10002)), 1),
    (dict(s_in=FAKE3, s_out=FAKE3), 1), (dict(s_out=FAKE), 1), (dict(lengths=ctypes.c_void_p(2)), 1),
    (dict(xt=-16), 1), (dict(xb=1 << 41), 1), (dict(yt=15), 1), (dict(yb=100), 1),
    (dict(B=1 << 20, T=1 << 20, D=1 << 10), 1),
    (dict(W=1), 2), (dict(W=5), 2), (dict(D=(1 << 20) + 1, yt=1 << 21, yb=1 << 25), 2),
    (dict(B=1, T=(1 << 30) + 1), 2),
])
def test_conv_fwd_rejects(how, expect):
    assert _conv_fwd(**how) == expect


def test_conv_step_and_bwd_reject():
    L = kata.lib()
    ok = [FAKE, FAKE2, FAKE, NUL, FAKE3, 2, 16, 4, 16, 16, 1, 1, NUL]
    for i, bad in ((0, NUL), (1, NUL), (2, NUL), (4, NUL), (4, FAKE2), (4, FAKE), (5, 0), (6, 0),
                   (8, -1), (9, 15), (10, 3), (11, 5)):
        args = list(ok)
        args[i] = bad
        assert L.kata_conv_step(*args) == 1, i
    ok[7] = 5
    assert L.kata_conv_step(*ok) == 2
    need = L.kata_conv_bwd_workspace_bytes(2, 8, 16, 4, 1)
    assert need > 0 and L.kata_conv_bwd_workspace_bytes(2, 8, 16, 5, 1) == 0
    ok = [FAKE, FAKE, NUL, FAKE2, FAKE3, NUL, NUL, 2, 8, 16, 4] + [128, 16] * 3 + [1, 1, WS, need, NUL]
    for i, bad in ((0, NUL), (1, NUL), (3, NUL), (4, NUL), (4, FAKE), (4, FAKE2), (11, -1), (13, -1),
                   (16, 8), (17, 7), (18, 9), (19, NUL), (19, ctypes.c_void_p(0x100010)),
                   (20, need - 1)):
        args = list(ok)
        args[i] = bad
        assert L.kata_conv_bwd_ws(*args) == 1, i


def _norm_args(**how):
    a = dict(q=FAKE, k=FAKE, wq=NUL, wk=NUL, pos=NUL, freq=FAKE, yq=FAKE2, yk=FAKE3, B=2, T=8, Hq=4,
             Hk=2, d=16, r=16, qs=(512, 64, 16), ks=(256, 32, 16), norm=1, eps=1e-6, pairs=0,
             dtype=1)
    a.update(how)
    return a


def _norm_fwd(**how):
    a = _norm_args(**how)
    return kata.lib().kata_qk_norm_fwd(*[a[n] for n in ("q", "k", "wq", "wk", "pos", "freq", "yq", "yk",
                                                        "B", "T", "Hq", "Hk", "d", "r")], *a["qs"],
                                       *a["ks"], a["norm"], a["eps"], a["pairs"], a["dtype"], NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(q=NUL), 1), (dict(k=NUL), 1), (dict(yq=NUL), 1), (dict(yk=NUL), 1), (dict(freq=NUL), 1),
    (dict(r=0), 1), (dict(r=7), 1), (dict(r=18), 1), (dict(B=0), 1), (dict(Hq=0), 1),
    (dict(Hk=-1), 1), (dict(Hk=0), 1), (dict(norm=3), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(pairs=2), 1), (dict(dtype=9), 1),
    (dict(yk=FAKE2), 1), (dict(yq=FAKE), 1), (dict(freq=ctypes.c_void_p(0x10004)), 1),
    (dict(qs=(-1, 64, 16)), 1), (dict(ks=(256, -32, 16)), 1),
    (dict(d=257, r=0, freq=NUL), 2), (dict(Hq=65535), 2), (dict(T=(1 << 30) + 1, B=1), 2),
])
def test_norm_fwd_rejects(how, expect):
    assert _norm_fwd(**how) == expect


def test_norm_bwd_rejects():
    L = kata.lib()
    need = L.kata_qk_norm_bwd_workspace_bytes(2, 8, 4, 2, 16, 1)
    assert need > 0 and L.kata_qk_norm_bwd_workspace_bytes(2, 8, 4, 2, 300, 1) == 0
    p = [ctypes.c_void_p(0x40000 + 0x1000 * i) for i in range(12)]
    ok = p[:6] + p[6:12] + [2, 8, 4, 2, 16, 16] + [512, 64, 16, 256, 32, 16] * 2 + \
        [1, 1e-6, 0, 1, 0, WS, need, NUL]
    for i, bad in ((0, NUL), (1, NUL), (5, NUL), (6, NUL), (7, NUL), (8, NUL), (9, NUL), (8, p[0]),
                   (9, p[7]), (9, p[8]), (17, 3), (18, -1), (25, 0), (26, 15), (28, 1), (30, 4),
                   (31, -1.0), (32, 2), (33, 2), (34, 2), (35, NUL), (36, need - 1)):
        args = list(ok)
        args[i] = bad
        assert L.kata_qk_norm_bwd_ws(*args) == 1, i
    ok[33], ok[34] = 0, 1  # fp32 rows with bf16 gradients
    assert L.kata_qk_norm_bwd_ws(*ok) == 2


def _ssm_ptrs(n):
    return [ctypes.c_void_p(0x40000 + 0x1000 * i) for i in range(n)]


@pytest.mark.parametrize("how,expect", [
    (dict(B=0), 1), (dict(T=0), 1), (dict(H=0), 1), (dict(G=0), 1), (dict(G=3), 1), (dict(N=0), 1),
    (dict(P=0), 1), (dict(soft=2), 1), (dict(dtype=4), 1), (dict(N=129), 2), (dict(P=257), 2),
    (dict(B=65535, H=2, G=1), 2), (dict(B=1, T=(1 << 30) + 1), 2),
    (dict(B=1 << 20, T=1 << 30, H=1 << 10, G=1), 1),
])
def test_ssm_sizes_reject(how, expect):
    L = kata.lib()
    a = dict(B=2, T=8, H=4, G=2, N=16, P=16, soft=1, dtype=1)
    a.update(how)
    p = _ssm_ptrs(15)
    sizes = [a[n] for n in ("B", "T", "H", "G", "N", "P")]
    assert L.kata_ssm_fwd_ws(*p[:11], *sizes, NUL, a["soft"], a["dtype"], WS, 1 << 40, NUL) == expect
    assert L.kata_ssm_bwd_ws(*p, *sizes, NUL, a["soft"], a["dtype"], WS, 1 << 40, NUL) == expect
    if a["soft"] == 1:
        assert L.kata_ssm_workspace_bytes(*sizes, a["dtype"], 1) == 0
    if "T" not in how:
        sizes.pop(1)
        assert L.kata_ssm_step(*p[:9], *sizes, NUL, a["soft"], a["dtype"], NUL) == expect


def test_ssm_pointers_reject():
    L = kata.lib()
    sizes = [2, 8, 4, 2, 16, 16]
    need = L.kata_ssm_workspace_bytes(*sizes, 1, 0)
    more = L.kata_ssm_workspace_bytes(*sizes, 1, 1)
    assert 0 < need < more
    p = _ssm_ptrs(15)
    odd = ctypes.c_void_p(0x90001)
    fwd = p[:11] + sizes + [NUL, 1, 1, WS, need, NUL]
    for i, bad in ((0, NUL), (1, NUL), (2, NUL), (3, NUL), (4, NUL), (9, NUL), (9, p[0]), (0, odd),
                   (5, odd), (7, ctypes.c_void_p(0x90008)), (10, p[7]), (8, odd), (20, NUL),
                   (20, ctypes.c_void_p(0x100080)), (21, need - 1)):
        args = list(fwd)
        args[i] = bad
        assert L.kata_ssm_fwd_ws(*args) == 1, i
    bwd = p + sizes + [NUL, 1, 1, WS, more, NUL]
    for i, bad in ((0, NUL), (2, NUL), (7, NUL), (8, NUL), (9, NUL), (11, NUL), (12, NUL), (8, p[0]),
                   (8, p[7]), (12, p[11]), (10, odd), (24, NUL), (25, more - 1)):
        args = list(bwd)
        args[i] = bad
        assert L.kata_ssm_bwd_ws(*args) == 1, i
    step = p[:9] + [2, 4, 2, 16, 16, NUL, 1, 1, NUL]
    for i, bad in ((0, NUL), (0, ctypes.c_void_p(0x90008)), (1, NUL), (8, NUL), (8, p[0]), (8, p[1])):
        args = list(step)
        args[i] = bad
        assert L.kata_ssm_step(*args) == 1, i


@pytest.mark.parametrize("field,value", [(0, -1), (1, 1 << 41), (5, -2), (7, -16), (11, -1), (13, 63),
                                         (14, 8), (12, 100)])
def test_ssm_strides_reject(field, value):
    L = kata.lib()
    s = [512, 64, 16, 32, 4, 1, 256, 32, 16, 256, 32, 16, 512, 64, 16]
    s[field] = value
    p = _ssm_ptrs(11)
    arr = (ctypes.c_longlong * 15)(*s)
    assert L.kata_ssm_fwd_ws(*p, 2, 8, 4, 2, 16, 16, arr, 1, 1, WS, 1 << 40, NUL) == 1


def test_launches_past_the_grid_are_refused():
    L = kata.lib()
    conv = dict(B=1 << 10, T=1 << 20, D=1 << 10, xb=1 << 30, xt=1 << 10, yb=1 << 30, yt=1 << 10)
    assert _conv_fwd(**conv) == 2
    assert L.kata_conv_bwd_workspace_bytes(1 << 10, 1 << 20, 1 << 10, 4, 1) == 0
    norm = dict(B=2, T=1 << 27, Hq=1, Hk=0, k=NUL, yk=NUL, d=256, r=0, freq=NUL,
                qs=(1 << 35, 256, 256))
    assert _norm_fwd(**norm) == 2
    assert L.kata_qk_norm_bwd_workspace_bytes(2, 1 << 27, 1, 0, 256, 1) == 0
    # a wave per head and chunk, and in the backward eight per group and chunk
    sizes = [1 << 15, 1 << 15, 1, 1, 16, 16]
    assert L.kata_ssm_workspace_bytes(*sizes, 1, 1) == 0
    assert L.kata_ssm_bwd_ws(*_ssm_ptrs(15), *sizes, NUL, 1, 1, WS, 1 << 62, NUL) == 2
    sizes[1] = 1 << 16
    assert L.kata_ssm_workspace_bytes(*sizes, 1, 0) == 0
    assert L.kata_ssm_fwd_ws(*_ssm_ptrs(11), *sizes, NUL, 1, 1, WS, 1 << 62, NUL) == 2


def test_outputs_apart_from_each_other_and_all_inputs():
    L = kata.lib()
    assert _conv_fwd(s_out=FAKE2) == 1 and _conv_fwd(w=FAKE3, s_out=FAKE3) == 1
    assert _conv_fwd(lengths=FAKE2) == 1
    assert _norm_fwd(wq=FAKE3) == 1 and _norm_fwd(pos=FAKE2) == 1
    p = _ssm_ptrs(15)
    sizes = [2, 8, 4, 2, 16, 16]
    need = L.kata_ssm_workspace_bytes(*sizes, 1, 1)
    for i, bad in ((9, p[2]), (10, p[9]), (10, p[5]), (9, p[8])):
        args = p[:11] + sizes + [NUL, 1, 1, WS, need, NUL]
        args[i] = bad
        assert L.kata_ssm_fwd_ws(*args) == 1, i
    for i, bad in ((10, p[2]), (13, p[10]), (14, p[8]), (14, p[6]), (24, p[0])):
        args = p + sizes + [NUL, 1, 1, WS, need, NUL]
        args[i] = bad
        assert L.kata_ssm_bwd_ws(*args) == 1, i
    step = p[:9] + [2, 4, 2, 16, 16, NUL, 1, 1, NUL]
    for i, bad in ((0, p[3]), (8, p[2]), (8, p[7])):
        args = list(step)
        args[i] = bad
        assert L.kata_ssm_step(*args) == 1, i


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8, 16)
    with pytest.raises(ValueError):
        kata.conv_fwd(x, torch.zeros(16, 4))
    with pytest.raises(ValueError):
        kata.qk_norm_fwd(x[..., None])
    with pytest.raises(ValueError):
        kata.ssm_step(torch.zeros(2, 4, 16, 16), x, x, x, x, x)
