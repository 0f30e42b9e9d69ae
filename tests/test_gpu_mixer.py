"""The mixer operators on the GPU against their definitions in fp64
(mixer_reference.py), element by element.

Tolerances.  An output is rounded once to its type (`ROUND`, relative to the
value); sums of n fp32 terms and the rounded functions in them are off by at most
(n + 16) 2^-24 of the terms' magnitudes.  The bf16 scan also rounds a chunk's
weights and the state that y (dB) reads to bf16, each 2^-8 of the terms'
magnitudes, and its fp32-typed results keep 2^-17 of every state term."""
from __future__ import annotations

import pytest
import torch

import mixer_reference as ref
from gpu_helpers import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def kata():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_17419_amd as k
    k.lib()  # raises if libkata.so is missing: no fallback
    return k


def near(got, want, tol, what):
    """|got - want| <= tol element by element (tol a tensor)."""
    got, want = got.detach().cpu().double(), want.detach()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), what
    off = ((got - want).abs() - tol).max()
    worst = ((got - want).abs() / (tol.detach() + 1e-300)).max()
    log(f"  {what}: {float(worst):.3f} of the tolerance")
    assert off <= 0, (what, float(off))


def normal(gen, *shape, dtype=torch.float64, std=1.0):
    """fp64 values that the type holds exactly."""
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(dtype).double()


def up(t, dtype=F32):
    return None if t is None else t.to(dtype).to(DEV)


def wide(t, dtype, pad):
    """The same values as a view of a wider device tensor: `pad` elements before each row."""
    rows = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), dtype=dtype, device=DEV)
    rows[..., pad:] = t.to(dtype).to(DEV)
    return rows[..., pad:]


# ---- short convolution -------------------------------------------------------------

CONV = [(1, 1, 1, 2), (2, 3, 64, 4), (3, 17, 65, 3), (1, 200, 130, 4), (2, 33, 1152, 4),
        (4, 100, 24, 2), (1, 4099, 8, 4)]


def conv_mag(x, w, bias, state=None):
    y, _ = ref.conv(x.abs(), w.abs(), None if bias is None else bias.abs(), False,
                    None if state is None else state.abs())
    return y


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,D,W", CONV)
def test_conv_fwd_and_bwd(kata, B, T, D, W, dtype):
    gen = torch.Generator().manual_seed(B * T + D)
    x, dy = normal(gen, B, T, D, dtype=dtype), normal(gen, B, T, D, dtype=dtype)
    w, bias = normal(gen, D, W, dtype=F32), normal(gen, D, dtype=F32)
    for act, b, pad in ((1, bias, 0), (0, None, 3), (1, None, 8)):
        log(f"case conv B{B} T{T} D{D} W{W} {dtype} act{act} pad{pad}")
        xs, dys = wide(x, dtype, pad), wide(dy, dtype, pad)
        want = ref.conv(x, w, b, act == 1)[0]
        # silu's slope is below 1.1
        tol = ROUND(dtype) * want.abs() + 1.1 * (W + 16) * ref.EPS32 * conv_mag(x, w, b)
        got = kata.conv_fwd(xs, up(w), up(b), act=act)
        near(got, want, tol, "y")
        leaf = [t.clone().requires_grad_() for t in ((x, w) if b is None else (x, w, b))]
        grads = torch.autograd.grad(ref.conv(*leaf, silu_act=act == 1)[0], leaf, dy)
        dx, dw, db = kata.conv_bwd(xs, up(w), up(b), dys, act=act)
        # dpre is off by its factor's error: |act''| <= 0.5 times pre's error, and roundings
        err = (W + 20) * ref.EPS32 * (1.1 + 0.5 * conv_mag(x, w, b)) * dy.abs()
        ahead = torch.cat([err + 1.1 * (W + 2) * ref.EPS32 * dy.abs(), torch.zeros(B, W - 1, D)], 1)
        tol = sum(ahead[:, W - 1 - j:W - 1 - j + T] * w[:, j].abs() for j in range(W))
        near(dx, grads[0], ROUND(dtype) * grads[0].abs() + tol, "dx")
        # sums of B T terms: runs of 32 tokens per wave in order, then in pairs or fp64
        terms = err + 1.1 * (32 * ((B * ((T + 31) // 32) + 1023) // 1024) + 8) * ref.EPS32 * dy.abs()
        past = torch.cat([torch.zeros(B, W - 1, D), x.abs()], 1)
        tol = torch.stack([(terms * past[:, j:j + T]).sum((0, 1)) for j in range(W)], 1)
        near(dw, grads[1], tol + ref.EPS32 * grads[1].abs(), "dw")
        if b is not None:
            near(db, grads[2], terms.sum((0, 1)) + ref.EPS32 * grads[2].abs(), "db")
        else:
            assert db is None


def ROUND(dtype):
    return ref.ROUND[dtype]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("D,W", ((72, 4), (33, 2), (128, 3)))
def test_conv_padded_batch_states_and_steps(kata, D, W, dtype):
    """Lengths from none to all, the windows kept, then token by token onwards."""
    gen = torch.Generator().manual_seed(D)
    T, lengths = 21, [0, 1, W - 1, 16, 21, 50, -3]
    B = len(lengths)
    x, more = normal(gen, B, T, D, dtype=dtype), normal(gen, B, 5, D, dtype=dtype)
    w, bias, s0 = normal(gen, D, W, dtype=F32), normal(gen, D, dtype=F32), normal(gen, B, W - 1, D, dtype=dtype)
    n = torch.tensor(lengths).clamp(0, T)
    behind = (torch.arange(T)[None] >= n[:, None])
    xs = up(x, dtype)
    xs[behind.to(DEV)] = float("nan")  # never read
    for state in (None, s0):
        log(f"case conv lengths D{D} W{W} {dtype} state {state is not None}")
        y = torch.full((B, T, D), 7.0, dtype=dtype, device=DEV)
        y, last = kata.conv_fwd(xs, up(w), up(bias), state=up(state, dtype), y=y,
                                lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                final_state=True)
        want, rows = ref.conv(x, w, bias, True, state, lengths)
        assert (y.cpu()[behind] == 7.0).all()
        tol = ROUND(dtype) * want.abs() + 1.1 * (W + 16) * ref.EPS32 * conv_mag(x, w, bias, state)
        near(y.cpu().double().masked_fill(behind[..., None], 0), want, tol, "y")
        assert torch.equal(last.cpu().double(), rows)
        for t in range(5):
            out = kata.conv_step(last, up(more[:, t], dtype), up(w), up(bias))
            want, new = ref.conv(more[:, t:t + 1], w, bias, True, rows)
            tol = ROUND(dtype) * want.abs() + 1.1 * (W + 16) * ref.EPS32 * conv_mag(
                more[:, t:t + 1], w, bias, rows)
            near(out, want[:, 0], tol[:, 0], f"step {t}")
            rows = new
            assert torch.equal(last.cpu().double(), rows)


def test_conv_non_finite_stays_ahead(kata):
    x = torch.ones((1, 40, 16), dtype=BF16, device=DEV)
    x[0, 20, 3], x[0, 25, 5] = float("inf"), float("nan")
    y = kata.conv_fwd(x, torch.ones((16, 4), device=DEV), None, act=0).cpu().float()
    bad = torch.zeros((1, 40, 16), dtype=torch.bool)
    bad[0, 20:24, 3] = bad[0, 25:29, 5] = True
    assert torch.equal(~torch.isfinite(y), bad)


# ---- norms and rotation -------------------------------------------------------------

NORM = [(1, 1, 1, 0, 1, 0), (2, 5, 3, 1, 16, 16), (1, 70, 4, 4, 64, 64), (3, 9, 4, 2, 64, 32),
        (2, 33, 2, 2, 40, 20), (1, 17, 5, 1, 7, 4), (2, 11, 2, 1, 128, 128), (1, 6, 2, 2, 256, 64),
        (1, 3, 1, 1, 255, 2), (2, 130, 16, 4, 32, 32), (5, 1, 16, 16, 64, 64), (1, 40, 3, 2, 48, 8)]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,Hq,Hk,d,r", NORM)
def test_norm_fwd_and_bwd(kata, B, T, Hq, Hk, d, r, dtype):
    gen = torch.Generator().manual_seed(B * T + d)
    q, k = normal(gen, B, T, Hq, d, dtype=dtype), normal(gen, B, T, max(Hk, 1), d, dtype=dtype)
    ws = [normal(gen, d, dtype=F32), normal(gen, d, dtype=F32)]
    freq = 10000.0 ** (-2 * torch.arange(r // 2, dtype=torch.float64) / max(r, 1))
    far = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, T), generator=gen)
    at = torch.arange(T).expand(B, T)
    for kind, pairs, pos, weights, ydtype, pad in (
            (1, False, None, True, F32, 0), (1, True, far, True, dtype, 0), (2, False, far, False, F32, 3),
            (0, True, None, True, dtype, 4), (2, True, None, True, F32, 0), (0, False, far, False, F32, 0)):
        log(f"case norm B{B} T{T} Hq{Hq} Hk{Hk} d{d} r{r} {dtype} kind{kind} pairs{pairs} "
            f"pos{pos is not None} w{weights} dy {ydtype} pad{pad}")
        sides, grads_in = [], []
        for x, w, heads in ((q, ws[0], Hq), (k, ws[1], Hk)):
            if heads == 0:
                sides.append((None, None))
                grads_in.append(None)
                continue
            sides.append((wide(x, dtype, pad), up(w) if weights else None))
            grads_in.append(normal(gen, B, heads, T, d, dtype=ydtype))
        (qs, wq), (ks, wk) = sides
        how = dict(pos=None if pos is None else pos.int().to(DEV), norm=kind, eps=1e-5, pairs=pairs)
        fr = freq.to(DEV) if r else None
        out = kata.qk_norm_fwd(qs, ks, wq, wk, fr, **how)
        got = kata.qk_norm_bwd(qs, ks, wq, wk, fr, up(grads_in[0], ydtype), up(grads_in[1], ydtype), **how)
        for i, (x, heads) in enumerate(((q, Hq), (k, Hk))):
            if heads == 0:
                assert out[i] is None and got[i] is None and got[2 + i] is None
                continue
            w, dy, name = ws[i] if weights else None, grads_in[i], "qk"[i]
            p = at if pos is None else pos
            want = ref.norm(x, w, freq, p, kind, 1e-5, pairs)
            leaf = [x.clone().requires_grad_()] + ([w.clone().requires_grad_()] if weights else [])
            y = ref.norm(leaf[0], leaf[1] if weights else None, freq, p, kind, 1e-5, pairs)
            grads = torch.autograd.grad(y, leaf, dy)
            # magnitudes: the normalised row, its weights, both coordinates of a pair; the
            # norm's own factor is off by the error of a sum of d squares, halved
            hat = ref.norm(x, None, freq[:0], p, kind, 1e-5, pairs).transpose(1, 2).abs()
            wabs = 1.0 if w is None else w.abs()
            spread = ref.turn_mag(hat * wabs, r, pairs).transpose(1, 2)
            near(out[i], want, ROUND(dtype) * want.abs() + (d / 2 + 20) * ref.EPS32 * spread, name)
            # e = R^T dy, g = w e, dx = inv (g - hat mean(g hat))
            e = ref.turn_mag(dy.abs().transpose(1, 2), r, pairs)
            g, inv = e * wabs, hat_scale(x, kind)
            dot = (g * hat).sum(-1, keepdim=True) * hat / (d if kind == 1 else 1) if kind else 0
            tol = ROUND(dtype) * grads[0].abs() + (2 * d + 40) * ref.EPS32 * inv * (g + dot)
            near(got[i], grads[0], tol, "d" + name)
            if weights:
                # a lane sums its tokens and heads in fp32, at most 1024 x 256 / lanes at once
                n = heads * (1 + B * T // 1024) + d / 2 + 60
                near(got[2 + i], grads[1], n * ref.EPS32 * (e * hat).sum((0, 1, 2)), "dw" + name)
            else:
                assert got[2 + i] is None


def hat_scale(x, kind):
    if kind == 0:
        return 1.0
    ss = x.square().mean(-1, keepdim=True) if kind == 1 else x.square().sum(-1, keepdim=True)
    return 1 / torch.sqrt(ss + 1e-5)


# ---- selective scan -------------------------------------------------------------------

SSM = [(1, 1, 1, 1, 1, 1), (2, 7, 4, 2, 16, 16), (1, 64, 2, 1, 64, 64), (1, 65, 3, 1, 32, 64),
       (2, 130, 4, 4, 20, 48), (1, 300, 2, 2, 128, 64), (1, 100, 2, 1, 64, 130), (1, 33, 1, 1, 100, 7),
       (1, 1111, 2, 1, 16, 8)]


def ssm_inputs(B, T, H, G, N, P, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    x, dt = normal(gen, B, T, H, P, dtype=dtype), normal(gen, B, T, H, dtype=dtype)
    Bm, Cm = normal(gen, B, T, G, N, dtype=dtype), normal(gen, B, T, G, N, dtype=dtype)
    A = -(torch.rand(H, generator=gen, dtype=torch.float64) * 4 + 0.01).float().double()
    D, bias = normal(gen, H, dtype=F32), (normal(gen, H, dtype=F32) - 2.0).float().double()
    return gen, x, dt, A, Bm, Cm, D, bias


def ssm_tol(want, mag, dtype, N, T):
    n = (N + 64 + T // 16 + 40) * ref.EPS32
    if dtype == F32:
        return ROUND(dtype) * want.abs() + n * mag
    # W or the state it reads rounded: 2^-8 of a term
    return ROUND(dtype) * want.abs() + (2.0 ** -8 * 1.01 + 2.0 ** -17 + n) * mag


def state_tol(mag, N, T, dtype):
    return ((N + 64 + T // 16 + 40) * ref.EPS32 + (2.0 ** -17 if dtype == BF16 else 0)) * mag


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P", SSM)
def test_ssm_fwd(kata, B, T, H, G, N, P, dtype):
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, B * T + N)
    S0 = normal(gen, B, H, N, P, dtype=F32)
    for soft, d, b, state, pad in ((True, D, bias, None, 0), (True, None, None, S0, 8), (False, D, None, S0, 3)):
        log(f"case ssm B{B} T{T} H{H} G{G} N{N} P{P} {dtype} softplus{soft} state{state is not None} pad{pad}")
        u = dt if soft else dt.abs().to(dtype).double()
        y, S = kata.ssm_fwd(wide(x, dtype, pad), wide(u, dtype, pad), up(A), wide(Bm, dtype, pad),
                            wide(Cm, dtype, pad), up(d), up(b), softplus=soft, state=up(state), final_state=True)
        want, last = ref.scan(x, u, A, Bm, Cm, d, b, soft, state)
        mag, smag = ref.scan_mag(x, u, A, Bm, Cm, d, b, soft, state, None)
        near(y, want, ssm_tol(want, mag, dtype, N, T), "y")
        near(S, last, state_tol(smag, N, T, dtype), "state")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P", SSM)
def test_ssm_bwd(kata, B, T, H, G, N, P, dtype):
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, B * T + P)
    dy = normal(gen, B, T, H, P, dtype=dtype)
    for soft, d, b, pad in ((True, D, bias, 0), (False, None, None, 5)):
        log(f"case ssm grads B{B} T{T} H{H} G{G} N{N} P{P} {dtype} softplus{soft} pad{pad}")
        u = dt if soft else dt.abs().to(dtype).double()
        got = kata.ssm_bwd(wide(x, dtype, pad), wide(u, dtype, pad), up(A), wide(Bm, dtype, pad),
                           wide(Cm, dtype, pad), up(d), up(b), wide(dy, dtype, pad), softplus=soft)
        want = ref.scan_grads(x, u, A, Bm, Cm, d, b, dy, soft)
        mags = ref.scan_grads_mag(x, u, A, Bm, Cm, d, b, dy, soft)
        for g, r, m, name in zip(got, want, mags, ("dx", "ddt", "dA", "dB", "dC", "dD", "dbias")):
            if r is None:
                assert g is None
                continue
            if name in ("dx", "dB", "dC"):
                # dB, dC: sums over H / G heads more
                tol = ssm_tol(r, m, dtype, max(N, P) + H // G, T)
            else:
                # products of fp32 sums over N, P and a chunk's pairs, two of them in a row
                n = (2 * (N + P + 128) + T // 16) * ref.EPS32 + (2.0 ** -16 if dtype == BF16 else 0)
                tol = n * m + (ROUND(dtype) if name == "ddt" else ref.EPS32) * r.abs()
            near(g, r, tol, name)


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_ssm_padded_batch_then_steps(kata, dtype):
    """Lengths from none to all with and without a first state, then steps onwards."""
    lengths, T, H, G, N, P = [0, 1, 63, 64, 65, 200, 999, -1], 200, 4, 2, 32, 40
    B = len(lengths)
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T + 4, H, G, N, P, dtype, 5)
    S0 = normal(gen, B, H, N, P, dtype=F32)
    behind = torch.arange(T)[None] >= torch.tensor(lengths)[:, None]
    dev = [up(t[:, :T], dtype) for t in (x, dt, Bm, Cm)]
    for t in dev:
        t[behind.to(DEV)] = float("nan")  # never read
    for state in (None, S0):
        log(f"case ssm lengths {dtype} state {state is not None}")
        y = torch.full((B, T, H, P), 7.0, dtype=dtype, device=DEV)
        y, S = kata.ssm_fwd(dev[0], dev[1], up(A), dev[2], dev[3], up(D), up(bias), state=up(state), y=y,
                            lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), final_state=True)
        assert (y.cpu()[behind] == 7.0).all()
        args = (x[:, :T], dt[:, :T], A, Bm[:, :T], Cm[:, :T], D, bias)
        want, last = ref.scan(*args, True, state, lengths)
        mag, smag = ref.scan_mag(*args, True, state, lengths)
        near(y.cpu().double().masked_fill(behind[..., None, None], 0), want, ssm_tol(want, mag, dtype, N, T), "y")
        near(S, last, state_tol(smag, N, T, dtype), "state")
        for t in range(T, T + 4):
            one = (x[:, t:t + 1], dt[:, t:t + 1], A, Bm[:, t:t + 1], Cm[:, t:t + 1], D, bias)
            out = kata.ssm_step(S, up(x[:, t], dtype), up(dt[:, t], dtype), up(A), up(Bm[:, t], dtype),
                                up(Cm[:, t], dtype), up(D), up(bias))
            want, last = ref.scan(*one, True, last)
            mag, smag = ref.scan_mag(*one, True, smag, None)
            # the state carries the prompt's error along
            tol = ROUND(dtype) * want.abs() + (N + 16) * ref.EPS32 * mag
            near(out, want[:, 0], (tol + state_tol(mag, N, T, dtype))[:, 0], f"step {t - T}")
            near(S, last, state_tol(smag, N, T, dtype), f"state {t - T}")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,H,G,N,P", ((1, 1, 1, 1, 1), (3, 4, 2, 64, 64), (2, 3, 1, 20, 50), (2, 2, 2, 128, 256),
                                       (1, 5, 1, 100, 255), (70, 16, 1, 64, 64)))
def test_ssm_step(kata, B, H, G, N, P, dtype):
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, 1, H, G, N, P, dtype, N + P)
    S0 = normal(gen, B, H, N, P, dtype=F32)
    for soft, d, b, pad in ((True, D, bias, 0), (False, None, None, 3)):
        log(f"case ssm step B{B} H{H} G{G} N{N} P{P} {dtype} softplus{soft}")
        u = dt if soft else dt.abs().to(dtype).double()
        S = up(S0)
        y = kata.ssm_step(S, wide(x, dtype, pad)[:, 0], wide(u, dtype, pad)[:, 0], up(A), wide(Bm, dtype, pad)[:, 0],
                          wide(Cm, dtype, pad)[:, 0], up(d), up(b), softplus=soft)
        want, last = ref.scan(x, u, A, Bm, Cm, d, b, soft, S0)
        mag, smag = ref.scan_mag(x, u, A, Bm, Cm, d, b, soft, S0, None)
        near(y, want[:, 0], (ROUND(dtype) * want.abs() + (N + 40) * ref.EPS32 * mag)[:, 0], "y")
        near(S, last, 40 * ref.EPS32 * smag, "state")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_ssm_strong_and_weak_decays(kata, dtype):
    """Steps that wipe the state out between steps that barely move it, and growth."""
    B, T, H, G, N, P = 1, 150, 3, 1, 16, 16
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, 9)
    dt = torch.full((B, T, H), 1e-3, dtype=torch.float64)
    dt[:, ::7] = 300.0
    dt[:, 40] = 1e30
    dt = dt.to(dtype).double()
    A = torch.tensor([-16.0, -1e-4, 0.01], dtype=torch.float64).float().double()
    dt[:, :, 2] = 0.5
    log(f"case ssm decays {dtype}")
    y, S = kata.ssm_fwd(up(x, dtype), up(dt, dtype), up(A), up(Bm, dtype), up(Cm, dtype), softplus=False, final_state=True)
    want, last = ref.scan(x, dt, A, Bm, Cm, soft=False)
    mag, smag = ref.scan_mag(x, dt, A, Bm, Cm, None, None, False, None, None)
    near(y, want, ssm_tol(want, mag, dtype, N, T), "y")
    near(S, last, state_tol(smag, N, T, dtype), "state")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_ssm_non_finite_stays_ahead(kata, dtype):
    """Values that are not finite reach no earlier token, no other sequence or head."""
    B, T, H, G, N, P = 2, 140, 4, 2, 32, 70
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, 3)
    clean = kata.ssm_fwd(*(up(t, dtype) for t in (x, dt)), up(A), up(Bm, dtype), up(Cm, dtype), up(D), up(bias))
    clean = clean.cpu().double()
    args = (x, dt, A, Bm, Cm, D, bias, True, None)
    tol = ssm_tol(ref.scan(*args)[0], ref.scan_mag(*args, None)[0], dtype, N, T)
    for name, where, bad in (("x", (0, 70, 1, 66), float("inf")), ("x", (0, 5, 1, 3), float("nan")),
                             ("dt", (0, 90, 1), float("nan")), ("Bm", (0, 100, 0, 2), float("inf")),
                             ("Cm", (0, 33, 0, 2), float("nan"))):
        t = dict(x=x.clone(), dt=dt.clone(), Bm=Bm.clone(), Cm=Cm.clone())
        t[name][where] = bad
        log(f"case ssm {dtype} {bad} in {name} at {where}")
        y = kata.ssm_fwd(up(t["x"], dtype), up(t["dt"], dtype), up(A), up(t["Bm"], dtype), up(t["Cm"], dtype),
                         up(D), up(bias))
        reach = torch.zeros((B, T, H, P), dtype=torch.bool)
        heads = slice(where[2], where[2] + 1) if name in ("x", "dt") else slice(0, 2)
        last = where[1] + 1 if name == "Cm" else T
        cols = slice(where[3], where[3] + 1) if name == "x" else slice(0, P)
        reach[0, where[1]:last, heads, cols] = True
        # the sums that such a value touched are formed again in another order: each is within
        # its tolerance of the exact value, so the two differ by twice that at most
        y = y.cpu().double()
        assert torch.isfinite(y[~reach]).all()
        assert ((y - clean).abs() <= 2 * tol)[~reach].all()
        assert not torch.isfinite(y[0, where[1], heads, cols]).any()


def test_ssm_spans_joined(kata):
    """Few heads over a long sequence: spans, with a state before them and short lengths."""
    B, T, H, G, N, P = 2, 3000, 1, 1, 16, 16
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, F32, 11)
    S0, lengths = normal(gen, B, H, N, P, dtype=F32), [3000, 700]
    A = torch.tensor([-0.02], dtype=torch.float64).float().double()  # states that last
    log("case ssm spans")
    y = torch.zeros((B, T, H, P), device=DEV)
    y, S = kata.ssm_fwd(up(x), up(dt), up(A), up(Bm), up(Cm), up(D), up(bias), state=up(S0), y=y,
                        lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), final_state=True)
    want, last = ref.scan(x, dt, A, Bm, Cm, D, bias, True, S0, lengths)
    mag, smag = ref.scan_mag(x, dt, A, Bm, Cm, D, bias, True, S0, lengths)
    near(y, want, ssm_tol(want, mag, F32, N, T), "y")
    near(S, last, state_tol(smag, N, T, F32), "state")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P", ((1, 100, 2, 1, 48, 96), (2, 70, 2, 2, 128, 256), (1, 130, 3, 1, 24, 72)))
def test_ssm_several_blocks_of_columns(kata, B, T, H, G, N, P, dtype):
    """Heads of more than 64 columns in whole aligned pieces, the last block full or not."""
    test_ssm_fwd(kata, B, T, H, G, N, P, dtype)
    test_ssm_bwd(kata, B, T, H, G, N, P, dtype)


# ---- layouts, streams, graphs ---------------------------------------------------------

def far(t, dtype, batch, token):
    """The same values with these strides over batch and token, in a buffer of their extent."""
    strides = [batch, token, *t.stride()[2:]]
    end = 1 + sum((n - 1) * s for n, s in zip(t.shape, strides))
    v = torch.empty(end, dtype=dtype, device=DEV).as_strided(t.shape, strides)
    return v.copy_(t)


@pytest.mark.parametrize("batch,token", ((1 << 32, 0), (64, 1 << 24)))
def test_offsets_past_32_bits(kata, batch, token):
    """Sequences 2^32 elements apart, and tokens 2^24 apart whose offsets pass 2^32."""
    B, T, H, G, N, P = (2, 70, 1, 1, 32, 64) if token == 0 else (1, 300, 1, 1, 32, 64)
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, BF16, 41)
    dy = normal(gen, B, T, H, P, dtype=BF16)
    ins = [up(t, BF16) for t in (x, dt, Bm, Cm, dy)]
    rest = (up(A), up(D), up(bias))
    w, wq = up(normal(gen, P, 4, dtype=F32)), up(normal(gen, P, dtype=F32))
    freq = kata.rope_frequencies(P, device=DEV)

    def calls(x, dt, Bm, Cm, dy, **out):
        y, S = kata.ssm_fwd(x, dt, rest[0], Bm, Cm, *rest[1:], final_state=True, **out)
        u, g = x.flatten(2), dy.flatten(2)
        return [y, S, *kata.ssm_bwd(x, dt, rest[0], Bm, Cm, *rest[1:], dy), kata.conv_fwd(u, w),
                *kata.conv_bwd(u, w, None, g)[:2], kata.qk_norm_fwd(x, None, wq, None, freq)[0],
                *kata.qk_norm_bwd(x, None, wq, None, freq, y.transpose(1, 2).contiguous())[::2]]
    want = calls(*ins)
    if token == 0:
        views = [far(t, BF16, batch, t.stride(1)) for t in ins]
        y = far(torch.zeros_like(ins[0]), BF16, batch, P)
    else:
        views = [far(t, BF16, batch, token) for t in ins]
        y = far(torch.zeros_like(ins[0]), BF16, batch, token)
    for a, b in zip(calls(*views, y=y), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("T", (1, 70))
def test_ssm_tokens_broadcast_with_stride_zero(kata, T, dtype):
    """The same token over and over by a token stride of 0, also where there is but one."""
    B, H, G, N, P = 2, 2, 1, 32, 64
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, 1, H, G, N, P, dtype, 31)
    dy = normal(gen, B, 1, H, P, dtype=dtype)

    def again(t):
        s = list(t.stride())
        s[1] = 0
        return t.as_strided((t.shape[0], T, *t.shape[2:]), s)
    ins = [again(up(t, dtype)) for t in (x, dt, Bm, Cm, dy)]
    full = [t.clone(memory_format=torch.contiguous_format) for t in ins]
    rest = (up(D), up(bias))
    for a, b in zip(*([*kata.ssm_fwd(*t[:2], up(A), *t[2:4], *rest, final_state=True),
                       *kata.ssm_bwd(*t[:2], up(A), *t[2:4], *rest, t[4])] for t in (ins, full))):
        assert torch.equal(a, b)


def test_other_orders_of_dimensions(kata):
    """Time-major activations and outputs, and heads broadcast with stride 0."""
    B, T, H, G, N, P = 3, 90, 4, 1, 32, 32
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, BF16, 4)
    ins = [up(t, BF16) for t in (x, dt, Bm, Cm)]
    flat = kata.ssm_fwd(ins[0], ins[1], up(A), ins[2], ins[3], up(D), up(bias))
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in ins]
    y = torch.empty((T, B, H, P), dtype=BF16, device=DEV).transpose(0, 1)
    kata.ssm_fwd(turned[0], turned[1], up(A), turned[2], turned[3], up(D), up(bias), y=y)
    assert torch.equal(y, flat)
    # head-major, as the attention entry points hold values
    y = torch.empty((B, H, T, P), dtype=BF16, device=DEV).transpose(1, 2)
    kata.ssm_fwd(ins[0].transpose(1, 2).contiguous().transpose(1, 2), ins[1], up(A), ins[2], ins[3], up(D),
                 up(bias), y=y)
    assert torch.equal(y, flat)
    one = ins[0][:, :, :1].expand(B, T, H, P)
    assert torch.equal(kata.ssm_fwd(one, ins[1], up(A), ins[2], ins[3], up(D), up(bias)),
                       kata.ssm_fwd(one.contiguous(), ins[1], up(A), ins[2], ins[3], up(D), up(bias)))
    u = up(normal(gen, 4, 50, 24, dtype=BF16), BF16)
    w = up(normal(gen, 24, 4, dtype=F32))
    flat = kata.conv_fwd(u, w)
    out = torch.empty((50, 4, 24), dtype=BF16, device=DEV).transpose(0, 1)
    assert torch.equal(kata.conv_fwd(u.transpose(0, 1).contiguous().transpose(0, 1), w, y=out), flat)
    with pytest.raises(kata.KataError):
        kata.conv_fwd(u, w, y=torch.empty((1, 50, 24), dtype=BF16, device=DEV).expand(4, 50, 24))


def _calls(kata, dtype=BF16):
    """Every entry point as (name, fn, what it updates in place)."""
    B, T, H, G, N, P = 2, 200, 4, 1, 64, 64
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, 21)
    x, dt, Bm, Cm = (up(t, dtype) for t in (x, dt, Bm, Cm))
    A, D, bias = up(A), up(D), up(bias)
    dy = up(normal(gen, B, T, H, P, dtype=dtype), dtype)
    u, w, b = x.reshape(B, T, H * P), up(normal(gen, H * P, 4, dtype=F32)), up(normal(gen, H * P, dtype=F32))
    freq = kata.rope_frequencies(P, device=DEV)
    wq = up(normal(gen, P, dtype=F32))
    gq = up(normal(gen, B, H, T, P, dtype=F32))
    S, win = up(normal(gen, B, H, N, P, dtype=F32)), up(normal(gen, B, 3, H * P, dtype=dtype), dtype)
    return [
        ("conv_fwd", lambda: kata.conv_fwd(u, w, b, final_state=True), []),
        ("conv_bwd", lambda: kata.conv_bwd(u, w, b, dy.reshape(B, T, H * P)), []),
        ("conv_step", lambda: kata.conv_step(win, u[:, 0], w, b), [win]),
        ("qk_norm_fwd", lambda: kata.qk_norm_fwd(x, x, wq, wq, freq), []),
        ("qk_norm_bwd", lambda: kata.qk_norm_bwd(x, x, wq, wq, freq, gq, gq), []),
        ("ssm_fwd", lambda: kata.ssm_fwd(x, dt, A, Bm, Cm, D, bias, final_state=True), []),
        ("ssm_bwd", lambda: kata.ssm_bwd(x, dt, A, Bm, Cm, D, bias, dy), []),
        ("ssm_step", lambda: kata.ssm_step(S, x[:, 0], dt[:, 0], A, Bm[:, 0], Cm[:, 0], D, bias), [S]),
    ]


def _flat(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def test_graphs_replay_the_eager_results(kata):
    for name, fn, held in _calls(kata):
        log(f"case graph {name}")
        before = [t.clone() for t in held]
        want = [t.clone() for t in _flat(fn())] + [t.clone() for t in held]

        def reset():
            for t, o in zip(held, before):
                t.copy_(o)
        reset()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = fn()
        for _ in range(3):
            reset()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(_flat(out) + held, want):
                assert torch.equal(a, b), name
            reset()
            for a, b in zip([t for t in _flat(fn())] + held, want):  # eager between the replays
                assert torch.equal(a, b), name


def test_two_streams_at_once(kata):
    """The same calls on two streams, each with its own outputs and workspace."""
    calls = [c for c in _calls(kata) if not c[2]]
    want = [[t.clone() for t in _flat(fn())] for _, fn, _ in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append([_flat(fn()) for _, fn, _ in calls])
    torch.cuda.synchronize()
    for out in outs:
        for (name, _, _), a, b in zip(calls, out, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), name
    side = torch.cuda.Stream()
    x = torch.randn((2, 50, 64), device=DEV)
    w = torch.randn((64, 4), device=DEV)
    torch.cuda.synchronize()
    y = kata.conv_fwd(x, w, stream=side)
    side.synchronize()
    assert torch.equal(y, kata.conv_fwd(x, w))


# ---- together ---------------------------------------------------------------------------

def test_mixer_training_step(kata):
    """Projection rows -> convolution -> norms with rotation -> KATA, forward and gradients back
    to the rows, against fp64.  The attention's own bound (2e-2 of each gradient's norm)
    covers the chain: its inputs are rounded to bf16 as here."""
    B, T, H, d = 1, 200, 2, 64
    gen = torch.Generator().manual_seed(2)
    rows = normal(gen, B, T, 3 * H * d, dtype=BF16)
    w, bias = normal(gen, 3 * H * d, 4, dtype=F32, std=0.5), normal(gen, 3 * H * d, dtype=F32, std=0.1)
    wq, wk = (1 + normal(gen, d, dtype=F32, std=0.1)).float().double(), torch.ones(d, dtype=torch.float64)
    freq, at = 10000.0 ** (-2 * torch.arange(d // 2, dtype=torch.float64) / d), torch.arange(T).expand(B, T)
    dout = normal(gen, B, H, T, d, dtype=F32)

    dev, wd, bd = up(rows, BF16), up(w), up(bias)
    u = kata.conv_fwd(dev, wd, bd)
    uq, uk, uv = (u[..., i * H * d:(i + 1) * H * d].unflatten(-1, (H, d)) for i in range(3))
    fr = freq.to(DEV)
    q, k = kata.qk_norm_fwd(uq, uk, up(wq), up(wk), fr, norm=kata.NORM_L2)
    v, _ = kata.qk_norm_fwd(uv, norm=kata.NORM_NONE)
    assert torch.equal(v, uv.transpose(1, 2))
    out, den = kata.fwd_chunked_train(q, k, v, 64)
    dq, dk, dv = kata.bwd_chunked(q, k, v, out, up(dout), 64, den=den)
    du = torch.empty_like(u)
    dxq, dxk, dxv = (du[..., i * H * d:(i + 1) * H * d].unflatten(-1, (H, d)) for i in range(3))
    _, _, dwq, dwk = kata.qk_norm_bwd(uq, uk, up(wq), up(wk), fr, dq, dk, norm=kata.NORM_L2, dxq=dxq, dxk=dxk)
    kata.qk_norm_bwd(uv, dq=dv, norm=kata.NORM_NONE, dxq=dxv)
    dx, dw, db = kata.conv_bwd(dev, wd, bd, du)

    leaf = [t.clone().requires_grad_() for t in (rows, w, bias, wq, wk)]

    class Rounded(torch.autograd.Function):  # a bf16 rounding, its gradient passed on
        @staticmethod
        def forward(ctx, t):
            return t.to(BF16).double()

        @staticmethod
        def backward(ctx, g):
            return g
    c = Rounded.apply(ref.conv(leaf[0], leaf[1], leaf[2])[0])
    rq, rk, rv = (c[..., i * H * d:(i + 1) * H * d].unflatten(-1, (H, d)) for i in range(3))
    rq = Rounded.apply(ref.norm(rq, leaf[3], freq, at, 2, 1e-6, False))
    rk = Rounded.apply(ref.norm(rk, leaf[4], freq, at, 2, 1e-6, False))
    weight = (rq @ rk.transpose(-1, -2)).square().tril()
    o = (weight @ rv.transpose(1, 2)) / weight.sum(-1, keepdim=True)
    grads = torch.autograd.grad(o, leaf, dout)
    for g, r, name in zip((out, dx, dw, db, dwq, dwk), (o.detach(), *grads),
                          ("out", "rows", "w", "bias", "wq", "wk")):
        off = float((g.cpu().double() - r).norm() / r.norm())
        log(f"  {name}: {off:.2e}")
        assert off <= 2e-2, name


def test_mixer_decode_continues_the_prompt(kata):
    """A prompt through convolution, norms and KATA's prefill, then tokens one by one: each
    equals the forward over all tokens (fp32, the attention's 1e-5)."""
    B, T, more, H, d = 2, 40, 6, 2, 32
    gen = torch.Generator().manual_seed(6)
    rows = up(normal(gen, B, T + more, 3 * H * d, dtype=F32))
    w, bias = up(normal(gen, 3 * H * d, 4, dtype=F32, std=0.5)), up(normal(gen, 3 * H * d, dtype=F32, std=0.1))
    freq = kata.rope_frequencies(d, device=DEV)
    how = dict(freq=freq, norm=kata.NORM_L2)

    def heads(u):
        return [u[..., i * H * d:(i + 1) * H * d].unflatten(-1, (H, d)) for i in range(3)]
    uq, uk, uv = heads(kata.conv_fwd(rows, w, bias))
    q, k = kata.qk_norm_fwd(uq, uk, **how)
    full = kata.fwd_chunked(q, k, uv.transpose(1, 2).contiguous(), 32)
    u, window = kata.conv_fwd(rows[:, :T], w, bias, final_state=True)
    uq, uk, uv = heads(u)
    _, k = kata.qk_norm_fwd(uq, uk, **how)
    S, z = kata.prefill_state(k, uv.transpose(1, 2).contiguous())
    for t in range(T, T + more):
        u = kata.conv_step(window, rows[:, t], w, bias)
        uq, uk, uv = heads(u[:, None])
        pos = torch.full((B, 1), t, dtype=torch.int32, device=DEV)
        q, k = kata.qk_norm_fwd(uq, uk, pos=pos, **how)
        o = kata.decode_step(S, z, q[:, :, 0], k[:, :, 0], uv[:, 0].contiguous())
        assert float((o - full[:, :, t]).abs().max()) <= 1e-5


def test_state_space_decode_continues_the_prompt(kata):
    """Convolution over x|B|C and the scan: a prompt of unequal lengths, then tokens one by one,
    against the same over each whole sequence (fp32; both within their own tolerance)."""
    B, T, more, H, G, N, P = 3, 90, 5, 4, 1, 32, 32
    gen, _, dt, A, _, _, D, bias = ssm_inputs(B, T + more, H, G, N, P, F32, 8)
    width = H * P + 2 * G * N
    rows = normal(gen, B, T + more, width, dtype=F32)
    w, cb = up(normal(gen, width, 4, dtype=F32, std=0.5)), up(normal(gen, width, dtype=F32, std=0.1))
    A, D, bias = up(A), up(D), up(bias)
    lengths = torch.tensor([T, 1, 37], dtype=torch.int32, device=DEV)

    def parts(u):
        return (u[..., :H * P].unflatten(-1, (H, P)), u[..., H * P:H * P + G * N].unflatten(-1, (G, N)),
                u[..., H * P + G * N:].unflatten(-1, (G, N)))
    rows, dt = up(rows), up(dt)
    u, window = kata.conv_fwd(rows[:, :T], w, cb, lengths=lengths, final_state=True)
    x, Bm, Cm = parts(u)
    _, S = kata.ssm_fwd(x, dt[:, :T], A, Bm, Cm, D, bias, lengths=lengths, final_state=True)
    got = []
    at = lengths.long()
    each = torch.arange(B, device=DEV)
    for i in range(more):
        u = kata.conv_step(window, rows[each, at + i], w, cb)
        x, Bm, Cm = parts(u)
        got.append(kata.ssm_step(S, x, dt[each, at + i], A, Bm, Cm, D, bias))
    got = torch.stack(got, 1).cpu()
    for b, n in enumerate(lengths.tolist()):
        u = kata.conv_fwd(rows[b:b + 1, :n + more], w, cb)
        x, Bm, Cm = parts(u)
        y = kata.ssm_fwd(x, dt[b:b + 1, :n + more], A, Bm, Cm, D, bias)[:, n:].cpu()
        mag = ref.scan_mag(*(t.cpu().double() for t in (x, dt[b:b + 1, :n + more], A, Bm, Cm, D, bias)), True,
                           None, None)[0][:, n:]
        near(got[b:b + 1], y.double(), 2 * (N + 64 + T // 16 + 40) * ref.EPS32 * mag + ref.EPS32 * y.abs(), f"seq {b}")
