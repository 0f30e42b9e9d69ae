"""The operators of a layer in 8 bits on the CPU: the fp64 reference's gradients against
differences, the reference's e4m3 against torch's, and what the C ABI refuses before it touches a
GPU."""
from __future__ import annotations

import ctypes

import pytest
import torch

import block_reference as ref
import paper_2607_17419_amd as kata
from test_mixer_cpu import _directional, _normal

FAKE = [ctypes.c_void_p(0x10000 * (k + 1)) for k in range(20)]  # aligned, never dereferenced
WS = ctypes.c_void_p(0x1000000)
NUL = ctypes.c_void_p(0)
ODD = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10002)


def test_reference_gradients_are_the_differences():
    gen = torch.Generator().manual_seed(0)
    cases = [(lambda s, w: ref.norm(s, w, 1e-3), (_normal(gen, 3, 7), _normal(gen, 7))),
             (lambda s: ref.norm(s, None, 0.0), (_normal(gen, 3, 7),))]
    x, r, i = (_normal(gen, 2, 9, 5) for _ in range(3))
    lam, rb, ib, h = (_normal(gen, *s) for s in ((5,), (5,), (5,), (2, 5)))
    cases.append((lambda *a: ref.recur(*a, c=3.0)[0], (x, r, i, lam, rb, ib)))
    cases.append((lambda x, r, i, lam, h: torch.cat([t.reshape(-1) for t in ref.recur(
        x, r, i, lam, state=h, lengths=[4, 9])]), (x, r, i, lam, h)))
    for k, (f, leaves) in enumerate(cases):
        exact, diff = _directional(f, leaves, k)
        assert abs(exact - diff) <= 1e-7 * (1 + abs(exact)), (k, exact, diff)


def test_reference_codes_are_e4m3():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    fine = every[every.isfinite()].double()
    assert torch.equal(ref.to_e4m3(fine), fine)
    half = torch.cat([(fine[1:127] + fine[:126]) / 2, torch.tensor([1.0, 447.0, 2.0 ** -10, 3e-4])]).float()
    near = torch.cat([half, torch.nextafter(half, half.new_tensor(1e9)), torch.nextafter(half, half * 0), -half])
    assert torch.equal(ref.to_e4m3(near.double()), near.to(torch.float8_e4m3fn).double())


# ---- refusals -----------------------------------------------------------------------

def _add_norm(x=FAKE[0], res=FAKE[1], w=FAKE[2], total=FAKE[3], y=FAKE[4], q=FAKE[5], scale=FAKE[6], M=4,
              D=16, xr=16, rr=16, sr=16, yr=16, qr=16, eps=1e-6, dtype=1):
    return kata.lib().kata_add_norm_fwd(x, res, w, total, y, q, scale, M, D, xr, rr, sr, yr, qr, eps,
                                        dtype, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(x=NUL), 1), (dict(y=NUL, q=NUL, scale=NUL), 1), (dict(res=NUL), 1), (dict(total=NUL), 1),
    (dict(q=NUL), 1), (dict(scale=NUL), 1), (dict(M=0), 1), (dict(D=0), 1), (dict(dtype=2), 1),
    (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(x=ODD), 1), (dict(w=HALF), 1),
    (dict(scale=HALF), 1), (dict(dtype=0, y=HALF), 1), (dict(y=FAKE[0]), 1), (dict(q=FAKE[4]), 1),
    (dict(total=FAKE[0]), 1), (dict(total=FAKE[1], sr=32), 1), (dict(res=FAKE[0], total=FAKE[0]), 1),
    (dict(xr=-1), 1), (dict(yr=15), 1), (dict(qr=8), 1), (dict(sr=0), 1), (dict(rr=1 << 41), 1),
    (dict(M=1 << 30, D=1 << 20), 1),
    (dict(D=32769, xr=1 << 16, rr=1 << 16, sr=1 << 16, yr=1 << 16, qr=1 << 16), 2),
    (dict(M=1 << 25), 2),
])
def test_add_norm_rejects(how, expect):
    assert _add_norm(**how) == expect


def _add_norm_bwd(s=FAKE[0], w=FAKE[1], dy=FAKE[2], ds=FAKE[3], dx=FAKE[4], dw=FAKE[5], M=4, D=16,
                  sr=16, yr=16, dr=16, xr=16, eps=1e-6, dtype=1, dyt=0, ws=WS, n=1 << 20):
    return kata.lib().kata_add_norm_bwd_ws(s, w, dy, ds, dx, dw, M, D, sr, yr, dr, xr, eps, dtype, dyt,
                                           ws, n, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(s=NUL), 1), (dict(dy=NUL), 1), (dict(dx=NUL), 1), (dict(dyt=2), 1), (dict(dyt=-1), 1),
    (dict(dtype=0, dyt=1), 2), (dict(dy=HALF), 1), (dict(ds=ODD), 1), (dict(dw=HALF), 1),
    (dict(dx=FAKE[0]), 1), (dict(dx=FAKE[2]), 1), (dict(dw=FAKE[1]), 1), (dict(xr=3), 1),
    (dict(ws=NUL), 1), (dict(ws=ctypes.c_void_p(0x1000010)), 1), (dict(n=8), 1), (dict(eps=-0.5), 1),
    (dict(ws=FAKE[0]), 1),
])
def test_add_norm_bwd_rejects(how, expect):
    assert _add_norm_bwd(**how) == expect


def _quant(x=FAKE[0], q=FAKE[1], scale=FAKE[2], qt=FAKE[3], st=FAKE[4], M=4, K=16, rows=1, xr=16, qr=16,
           tr=16, dtype=1):
    return kata.lib().kata_f8_quant(x, q, scale, qt, st, M, K, rows, xr, qr, tr, dtype, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(x=NUL), 1), (dict(q=NUL), 1), (dict(scale=NUL), 1), (dict(qt=NUL), 1), (dict(st=NUL), 1),
    (dict(q=NUL, scale=NUL, qt=NUL, st=NUL), 1), (dict(rows=2), 1), (dict(rows=0), 1), (dict(M=0), 1),
    (dict(K=-1), 1), (dict(dtype=5), 1), (dict(x=ODD), 1), (dict(scale=HALF), 1), (dict(st=HALF), 1),
    (dict(q=FAKE[0]), 1), (dict(qt=FAKE[1]), 1), (dict(qr=15), 1), (dict(tr=3), 1), (dict(xr=-16), 1),
    (dict(M=1 << 30, K=1 << 20), 1), (dict(M=(1 << 30) + 1, K=1, xr=1, qr=1, tr=1 << 31), 2),
    (dict(M=1 << 30, K=1 << 9), 2),
])
def test_f8_quant_rejects(how, expect):
    assert _quant(**how) == expect


def _gemm(a=FAKE[0], sa=FAKE[1], b=FAKE[2], sb=FAKE[3], c=FAKE[4], M=4, N=8, K=16, rows=128, ar=16, br=16,
          cr=8, dtype=1, ws=WS, n=1 << 24):
    return kata.lib().kata_f8_gemm_ws(a, sa, b, sb, c, M, N, K, rows, ar, br, cr, dtype, ws, n, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(a=NUL), 1), (dict(sa=NUL), 1), (dict(b=NUL), 1), (dict(sb=NUL), 1), (dict(c=NUL), 1),
    (dict(M=0), 1), (dict(N=0), 1), (dict(K=0), 1), (dict(rows=64), 1), (dict(dtype=3), 1), (dict(c=ODD), 1),
    (dict(dtype=0, c=HALF), 1), (dict(sa=HALF), 1), (dict(sb=ODD), 1), (dict(c=FAKE[0]), 1),
    (dict(ws=FAKE[4]), 1), (dict(ar=-1), 1), (dict(cr=7), 1), (dict(cr=0), 1), (dict(ws=NUL), 1),
    (dict(ws=ctypes.c_void_p(0x1000080)), 1), (dict(n=0), 1),
    (dict(M=1000, N=1000, K=8192, ar=8192, br=8192, cr=1000, n=1000), 1),
    (dict(M=1 << 30, N=1 << 20), 1), (dict(M=1 << 20, N=1 << 20, cr=1 << 20), 2),
])
def test_f8_gemm_rejects(how, expect):
    assert _gemm(**how) == expect


_Strides = ctypes.c_longlong * 14


def _strides(**how):
    s = dict(xb=128, xt=16, rb=128, rt=16, ib=128, it=16, yb=128, yt=16, dxb=128, dxt=16, drb=128, drt=16,
             dib=128, dit=16)
    s.update(how)
    return ctypes.byref(_Strides(*s.values()))


def _recur_fwd(x=FAKE[0], r=FAKE[1], i=FAKE[2], lam=FAKE[3], rb=FAKE[4], ib=FAKE[5], h=FAKE[6], ln=FAKE[7],
               y=FAKE[8], ho=FAKE[9], st=FAKE[10], B=2, T=8, D=16, s=None, c=8.0, dtype=1, ws=WS, n=1 << 24):
    return kata.lib().kata_recur_fwd_ws(x, r, i, lam, rb, ib, h, ln, y, ho, st, B, T, D, s, c, dtype, ws, n,
                                        NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(x=NUL), 1), (dict(r=NUL), 1), (dict(i=NUL), 1), (dict(lam=NUL), 1), (dict(y=NUL), 1),
    (dict(B=0), 1), (dict(T=0), 1), (dict(D=0), 1), (dict(c=0.0), 1), (dict(c=-1.0), 1),
    (dict(c=float("inf")), 1), (dict(dtype=9), 1), (dict(x=ODD), 1), (dict(r=ODD), 1), (dict(lam=HALF), 1),
    (dict(rb=HALF), 1), (dict(ib=ODD), 1), (dict(h=HALF), 1), (dict(ln=HALF), 1), (dict(ho=HALF), 1),
    (dict(st=HALF), 1), (dict(dtype=0, y=HALF), 1), (dict(y=FAKE[0]), 1), (dict(ho=FAKE[6]), 1),
    (dict(st=FAKE[9]), 1), (dict(ws=FAKE[8]), 1), (dict(s=_strides(xt=-1)), 1), (dict(s=_strides(yt=15)), 1),
    (dict(s=_strides(yb=100)), 1), (dict(s=_strides(ib=1 << 41)), 1), (dict(ws=NUL), 1), (dict(n=100), 1),
    (dict(ws=ctypes.c_void_p(0x1000040)), 1), (dict(B=1 << 20, T=1 << 20, D=1 << 10), 1),
    (dict(B=1, T=(1 << 30) + 1), 2), (dict(D=(1 << 20) + 1), 2), (dict(B=1 << 20, T=128, D=8192), 2),
])
def test_recur_fwd_rejects(how, expect):
    assert _recur_fwd(**how) == expect


def _recur_bwd(x=FAKE[0], r=FAKE[1], i=FAKE[2], lam=FAKE[3], rb=FAKE[4], ib=FAKE[5], h=FAKE[6], ln=FAKE[7],
               st=FAKE[8], dy=FAKE[9], dho=FAKE[10], dx=FAKE[11], dr=FAKE[12], di=FAKE[13], dl=FAKE[14],
               drb=FAKE[15], dib=FAKE[16], dhi=FAKE[17], B=2, T=8, D=16, s=None, c=8.0, dtype=1, ws=WS,
               n=1 << 24):
    return kata.lib().kata_recur_bwd_ws(x, r, i, lam, rb, ib, h, ln, st, dy, dho, dx, dr, di, dl, drb, dib,
                                        dhi, B, T, D, s, c, dtype, ws, n, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(dy=NUL), 1), (dict(dx=NUL), 1), (dict(dr=NUL), 1), (dict(di=NUL), 1), (dict(x=NUL), 1),
    (dict(dy=ODD), 1), (dict(dx=ODD), 1), (dict(st=HALF), 1), (dict(dho=HALF), 1), (dict(dl=HALF), 1),
    (dict(drb=HALF), 1), (dict(dib=HALF), 1), (dict(dhi=HALF), 1), (dict(dx=FAKE[9]), 1), (dict(dr=FAKE[11]), 1),
    (dict(dhi=FAKE[10]), 1), (dict(dl=FAKE[3]), 1), (dict(ws=FAKE[8]), 1), (dict(s=_strides(dxt=8)), 1),
    (dict(s=_strides(drb=16)), 1), (dict(s=_strides(dit=-16)), 1), (dict(n=100), 1), (dict(c=0.0), 1),
    (dict(B=1, T=(1 << 30) + 1), 2),
])
def test_recur_bwd_rejects(how, expect):
    assert _recur_bwd(**how) == expect


def _recur_step(h=FAKE[0], x=FAKE[1], r=FAKE[2], i=FAKE[3], lam=FAKE[4], rb=FAKE[5], ib=FAKE[6], y=FAKE[7],
                B=2, D=16, xb=16, rbs=16, ibs=16, yb=16, c=8.0, dtype=1):
    return kata.lib().kata_recur_step(h, x, r, i, lam, rb, ib, y, B, D, xb, rbs, ibs, yb, c, dtype, NUL)


@pytest.mark.parametrize("how,expect", [
    (dict(h=NUL), 1), (dict(x=NUL), 1), (dict(y=NUL), 1), (dict(lam=NUL), 1), (dict(h=HALF), 1),
    (dict(y=FAKE[0]), 1), (dict(h=FAKE[1]), 1), (dict(y=FAKE[1]), 1), (dict(B=0), 1), (dict(D=0), 1),
    (dict(yb=15), 1), (dict(xb=-1), 1), (dict(c=float("nan")), 1), (dict(dtype=-1), 1),
    (dict(D=(1 << 20) + 1, yb=1 << 21), 2),
])
def test_recur_step_rejects(how, expect):
    assert _recur_step(**how) == expect


def test_sizes():
    L = kata.lib()
    assert L.kata_add_norm_bwd_workspace_bytes(0, 8, 0) == 0 == L.kata_add_norm_bwd_workspace_bytes(8, 40000, 0)
    assert L.kata_add_norm_bwd_workspace_bytes(8, 100, 1) >= 400
    assert L.kata_f8_gemm_workspace_bytes(0, 1, 1) == 0 and L.kata_f8_gemm_workspace_bytes(1, 1, 1) > 0
    assert L.kata_recur_workspace_bytes(1, 1, 1, 2, 0) == 0 and L.kata_recur_workspace_bytes(1, 1, 1, 1, 1) > 0
    assert L.kata_recur_spans(0) == 0 == L.kata_recur_spans(-5)
    assert L.kata_recur_spans(1) == 1 and L.kata_recur_spans(1 << 30) >= 1
    big = L.kata_recur_workspace_bytes(1, 1 << 28, 128, 0, 1)
    assert big > 1 << 32  # sizes past 32 bits


def test_binding_wants_device_tensors():
    x, w = torch.zeros(4, 16), torch.zeros(16)
    f8 = torch.zeros(4, 16, dtype=torch.uint8).view(torch.float8_e4m3fn)
    for call in (lambda: kata.add_norm_fwd(x, w), lambda: kata.add_norm_f8_fwd(x, w),
                 lambda: kata.add_norm_bwd(x, w, x), lambda: kata.f8_quant(x),
                 lambda: kata.f8_gemm(f8, x, f8, x), lambda: kata.recur_fwd(x[None], x[None], x[None], w),
                 lambda: kata.recur_fwd_train(x[None], x[None], x[None], w),
                 lambda: kata.recur_bwd(x[None], x[None], x[None], w, None, None, x[None]),
                 lambda: kata.recur_step(x, x, x, x, w)):
        with pytest.raises(ValueError, match="device tensors"):
            call()


def test_rows_of_one_stride():
    t = torch.zeros(3, 5, 24)
    assert kata._rows(t[..., :16], "t") == (15, 16, 24)
    assert kata._rows(t[:, 2:3, 8:], "t") == (3, 16, 120)
    assert kata._rows(t[1:2, 2:3], "t") == (1, 24, 24)
    assert kata._rows(t.view(15, 24)[::2], "t") == (8, 24, 48)
    for bad in (t[:, :4], t[0, 0], t.transpose(0, 1)):
        with pytest.raises(ValueError):
            kata._rows(bad, "t")
