"""Where the mixer operators' results keep fewer bits than their type: sums that cancel,
parameters that stand in a matrix operand, states that are returned.

Tolerances count the roundings that a result of its type needs, as in
test_gpu_mixer.py, or hold the kernel's error against that of the definition itself
evaluated in fp32, token by token."""
from __future__ import annotations

import math

import pytest
import torch

import mixer_reference as ref
from gpu_helpers import log
from test_gpu_mixer import (BF16, DEV, F32, ROUND, kata, near, normal, ssm_inputs, ssm_tol,  # noqa: F401
                            state_tol, up)

pytestmark = pytest.mark.gpu


def layer_inputs(B, T, H, G, N, P, dtype, seed):
    """What the scan meets in a layer: x, B and C behind a SiLU, decays of 1 to 16, steps of
    1e-3 to 1e-1 around each head's own."""
    gen = torch.Generator().manual_seed(seed)

    def act(*shape):
        return ref.silu(normal(gen, *shape)).to(dtype).double()
    x, Bm, Cm = act(B, T, H, P), act(B, T, G, N), act(B, T, G, N)
    dt, dy = normal(gen, B, T, H, dtype=dtype, std=0.5), normal(gen, B, T, H, P, dtype=dtype, std=0.1)
    A = -(1 + 15 * torch.rand(H, generator=gen, dtype=torch.float64)).float().double()
    at = torch.exp(math.log(1e-3) + math.log(100) * torch.rand(H, generator=gen, dtype=torch.float64))
    bias = (at + torch.log(-torch.expm1(-at))).float().double()
    return x, dt, A, Bm, Cm, normal(gen, H, dtype=F32), bias, dy


# ---- sums that cancel ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("small", (7, 24, 32, 45))
def test_ssm_pairs_across_a_token_alone_reach_its_step(kata, dtype, small):  # noqa: F811
    """The first tokens of a chunk 2^-20 of the others: of the pairs behind them not even the
    rounding errors may reach their steps' gradients."""
    B, T, H, G, N, P = 1, 64 if dtype == BF16 else 32, 3, 1, 16, 16
    small = small if dtype == BF16 else small // 2
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, small)
    dy = normal(gen, B, T, H, P, dtype=dtype)
    x[:, :small] *= 2.0 ** -20
    dy[:, :small] *= 2.0 ** -20
    log(f"case ssm pairs {dtype} small {small}")
    got = kata.ssm_bwd(up(x, dtype), up(dt, dtype), up(A), up(Bm, dtype), up(Cm, dtype), up(D), up(bias), up(dy, dtype))
    want = ref.scan_grads(x, dt, A, Bm, Cm, D, bias, dy)[1]
    mag = ref.scan_grads_mag(x, dt, A, Bm, Cm, D, bias, dy)[1]
    # two products of fp32 sums over N, P and a chunk's pairs
    near(got[1], want, 2 * (N + P + 128) * ref.EPS32 * mag + ROUND(dtype) * want.abs(), "ddt")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_ssm_parameter_gradients_as_near_as_fp32(kata, dtype):  # noqa: F811
    """dA and dt_dbias of heads, each a sum over tokens that may cancel: together no further off
    than twice the definition evaluated in fp32.  (The kernel's sums have as many roundings to fp32
    as the definition's, or fewer; twice, as the error of a few dozen heads is itself a sample.)"""
    off = {"dA": [], "dbias": []}
    for seed, (B, T, H, G, N, P) in enumerate(((1, 200, 16, 1, 64, 64), (2, 130, 16, 2, 32, 64),
                                               (1, 150, 16, 1, 128, 64), (1, 90, 16, 4, 16, 128))):
        log(f"case ssm parameters {dtype} T{T} N{N} P{P}")
        x, dt, A, Bm, Cm, D, bias, dy = layer_inputs(B, T, H, G, N, P, dtype, seed)
        got = kata.ssm_bwd(up(x, dtype), up(dt, dtype), up(A), up(Bm, dtype), up(Cm, dtype), up(D), up(bias),
                           up(dy, dtype))
        want = ref.scan_grads(x, dt, A, Bm, Cm, D, bias, dy)
        plain = ref.scan_grads(*(t.float() for t in (x, dt, A, Bm, Cm, D, bias, dy)))
        for i, name in ((2, "dA"), (6, "dbias")):
            scale = want[i].square().mean().sqrt()
            off[name].append(torch.stack([(got[i].cpu().double() - want[i]) / scale,
                                          (plain[i].double() - want[i]) / scale]))
    for name, parts in off.items():
        ours, plain = torch.cat(parts, 1).square().mean(1).sqrt().tolist()
        log(f"  {name}: {ours:.2e}, in fp32 {plain:.2e}")
        assert ours <= 2 * plain, (name, ours, plain)


# ---- steps of masked tokens --------------------------------------------------------------

@pytest.mark.parametrize("dtype", (BF16, F32))
def test_ssm_steps_of_masked_tokens_are_zero(kata, dtype):  # noqa: F811
    """dt of -inf, of the type's lowest value and of large negative ones: a step of 0, which
    leaves the state as it is, in a sequence, its gradients and token by token."""
    B, T, H, G, N, P = 1, 90, 2, 1, 16, 16
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, 17)
    dy = normal(gen, B, T, H, P, dtype=dtype)
    low = torch.finfo(dtype).min
    for at, value in ((0, low), (5, -math.inf), (17, -2.3e38), (31, -2.5e38), (40, -1e30), (63, low), (64, -math.inf),
                      (70, -200.0), (71, -104.5), (72, -100.0), (73, -88.0), (89, low)):
        dt[:, at, 0] = value
    dt = dt.to(dtype).double()
    log(f"case ssm masked tokens {dtype}")
    ins = [up(t, dtype) for t in (x, dt, Bm, Cm)]
    rest = (up(D), up(bias))
    y, S = kata.ssm_fwd(ins[0], ins[1], up(A), ins[2], ins[3], *rest, final_state=True)
    want, last = ref.scan(x, dt, A, Bm, Cm, D, bias)
    mag, smag = ref.scan_mag(x, dt, A, Bm, Cm, D, bias, True, None, None)
    near(y, want, ssm_tol(want, mag, dtype, N, T), "y")
    near(S, last, state_tol(smag, N, T, dtype), "state")
    S = torch.zeros_like(S)
    for t in range(T):
        out = kata.ssm_step(S, ins[0][:, t], ins[1][:, t], up(A), ins[2][:, t], ins[3][:, t], *rest)
        near(out, want[:, t], ssm_tol(want, mag, dtype, N, T)[:, t], f"step {t}")
    near(S, last, state_tol(smag, N, T, dtype), "state of the steps")
    got = kata.ssm_bwd(ins[0], ins[1], up(A), ins[2], ins[3], *rest, up(dy, dtype))
    grads = ref.scan_grads(x, dt, A, Bm, Cm, D, bias, dy)
    mags = ref.scan_grads_mag(x, dt, A, Bm, Cm, D, bias, dy)
    # a gate below fp32's smallest normal value, as of the tokens of -88 to -104, may be lost: off by
    # 2^-126 of what it multiplies, the magnitudes of the same call with the steps themselves as dt
    steps = ref.softplus(dt + bias)
    lost = 2.0 ** -126 * ref.scan_grads_mag(x, steps, A, Bm, Cm, D, None, dy, False)[1]
    for g, r, m, name in zip(got, grads, mags, ("dx", "ddt", "dA", "dB", "dC", "dD", "dbias")):
        if name in ("dx", "dB", "dC"):
            tol = ssm_tol(r, m, dtype, N + H, T)
        elif name == "ddt":
            tol = (2 * (N + P + 128) + T) * ref.EPS32 * m + ROUND(dtype) * r.abs() + lost
        else:
            tol = (2 * (N + P + 128) + T) * ref.EPS32 * m + ref.EPS32 * r.abs()
        near(g, r, tol, name)
    assert (got[1][0, [0, 5, 17, 31, 40, 63, 64, 70, 89], 0] == 0).all()


def test_ssm_steps_and_gates_to_fp32(kata):  # noqa: F811
    """Of one token with one feature all is a product: y = C B step x and ddt = dy C B x gate, each
    from a step or gate of fp32 precision wherever z = dt + bias lies, and seven roundings."""
    B, H = 300, 4
    gen = torch.Generator().manual_seed(3)
    dt = torch.linspace(-84, 24, B * H, dtype=torch.float64).view(B, 1, H).float().double()
    x, dy, Bm, Cm = (normal(gen, B, 1, H, 1, dtype=F32) for _ in range(4))
    A, bias = torch.full((H,), -1.0, dtype=torch.float64), normal(gen, H, dtype=F32)
    log("case ssm steps and gates")
    args = (up(x), up(dt), up(A), up(Bm), up(Cm), None, up(bias))
    y, S = kata.ssm_fwd(*args, final_state=True)
    step = ref.softplus(dt + bias)[..., None]
    near(S, (step * Bm * x)[:, 0, :, :, None], 8 * ref.EPS32 * (step * Bm * x).abs()[:, 0, :, :, None], "state")
    near(y, step * Bm * Cm * x, 8 * ref.EPS32 * (step * Bm * Cm * x).abs(), "y")
    one = [t[:, 0] for t in (args[0], args[1], args[3], args[4])]
    y = kata.ssm_step(torch.zeros_like(S), one[0], one[1], args[2], one[2], one[3], None, args[6])
    near(y, (step * Bm * Cm * x)[:, 0], 8 * ref.EPS32 * (step * Bm * Cm * x).abs()[:, 0], "y of a step")
    ddt = kata.ssm_bwd(*args, up(dy))[1]
    want = (dy * x * Bm * Cm)[..., 0] * torch.sigmoid(dt + bias)
    # (a few lie below 2^-126, where fp32's steps are 2^-149 and a rounding is off by half of one)
    near(ddt, want, 8 * ref.EPS32 * want.abs() + 2.0 ** -150, "ddt")


# ---- states over many chunks --------------------------------------------------------------

def test_ssm_state_rounded_once_a_chunk(kata):  # noqa: F811
    """The state of 2048 fp32 tokens, decays of 1 and all terms positive, in 64 chunks: the state
    before it and a chunk's own sum are added with one rounding, off by 2^-24 of the state then at
    most, so by 2^-24 / sqrt(3) rms; the states grow evenly, so all of them together are off by
    sqrt(64 / 3 + 1) times that, the 1 for what is rounded within a chunk, on 1/64 of the state."""
    B, T, H, G, N, P = 64, 2048, 16, 1, 16, 16  # a workgroup for each head: no spans
    gen = torch.Generator().manual_seed(5)
    x, Bm = normal(gen, B, T, H, P, dtype=F32).abs(), normal(gen, B, T, G, N, dtype=F32).abs()
    dt = normal(gen, B, T, H, dtype=F32).abs()
    log("case ssm state of many chunks")
    _, S = kata.ssm_fwd(up(x), up(dt), torch.zeros(H, device=DEV), up(Bm), up(Bm), softplus=False, final_state=True)
    terms = (x * dt[..., None]).to(DEV)
    want = torch.matmul(Bm.to(DEV)[:, :, 0].transpose(1, 2).contiguous(), terms.flatten(2))
    want = want.view(B, N, H, P).transpose(1, 2)
    off = ((S.double() - want) / want).square().mean().sqrt().item()
    log(f"  state: {off:.2e}")
    assert off <= ref.EPS32 * math.sqrt((64 / 3 + 1) / 3), off


# ---- the skip parameter ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P", ((2, 70, 3, 1, 32, 64), (1, 100, 2, 1, 64, 130), (1, 130, 4, 2, 100, 40)))
def test_ssm_skip_parameter_keeps_its_bits(kata, B, T, H, G, N, P, dtype):  # noqa: F811
    """D x and D dy far above the state's terms: D is fp32, so they are off by the output's
    rounding and 2^-17 (D as two bf16 parts) at most; 2^-8 is for the state's terms alone."""
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, T)
    dy = normal(gen, B, T, H, P, dtype=dtype)
    D, dt = (D * 1000).float().double(), dt - 3
    dt = dt.to(dtype).double()
    log(f"case ssm skip T{T} N{N} P{P} {dtype}")
    args = (x, dt, A, Bm, Cm)
    ins = (up(x, dtype), up(dt, dtype), up(A), up(Bm, dtype), up(Cm, dtype), up(D), up(bias))
    want = ref.scan(*args, D, bias)[0]
    terms = ref.scan_mag(*args, None, bias, True, None, None)[0]
    skip = D.abs()[:, None] * x.abs()
    tol = ssm_tol(want, terms, dtype, N, T) + (2.0 ** -17 + 64 * ref.EPS32) * skip
    near(kata.ssm_fwd(*ins), want, tol, "y")
    near(kata.ssm_fwd(*ins, final_state=True)[0], want, tol, "y with a state")
    dx = kata.ssm_bwd(*ins, up(dy, dtype))[0]
    want = ref.scan_grads(*args, D, bias, dy)[0]
    terms = ref.scan_grads_mag(*args, None, bias, dy)[0]
    near(dx, want, ssm_tol(want, terms, dtype, max(N, P) + H // G, T)
         + (2.0 ** -17 + 64 * ref.EPS32) * D.abs()[:, None] * dy.abs(), "dx")


def test_ssm_returned_state_keeps_fp32(kata):  # noqa: F811
    """States of a few tokens' memory from bf16 calls: step, decay, their product, its product with
    x and the seven sums of a chunk are rounded to fp32, 11 roundings of 2^-24 at most, 2^-24 / sqrt(3)
    rms each.  (Terms in two bf16 parts would be off by 2^-18.)"""
    B, T, H, G, N, P = 4, 190, 16, 1, 32, 64
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, BF16, 23)
    dt = dt.abs().to(BF16).double() + 0.5
    dt, A = dt.to(BF16).double(), torch.full((H,), -2.0, dtype=torch.float64)
    log("case ssm returned state")
    _, S = kata.ssm_fwd(up(x, BF16), up(dt, BF16), up(A), up(Bm, BF16), up(Cm, BF16), softplus=False,
                        final_state=True)
    want = ref.scan(x, dt, A, Bm, Cm, soft=False)[1]
    mag = ref.scan_mag(x, dt, A, Bm, Cm, None, None, False, None, None)[1]
    off = ((S.cpu().double() - want) / mag).square().mean().sqrt().item()
    log(f"  state: {off:.2e}")
    assert off <= ref.EPS32 * math.sqrt(11 / 3), off


def test_ssm_skip_gradient_of_terms_that_cancel(kata):  # noqa: F811
    """dD of one column of bf16 values: every x dy is exact in fp32, and so are their sums in fp64.
    The second half of the tokens is the first's with dy turned around, but for one token."""
    B, T, H, G, N, P = 1, 1000, 4, 1, 16, 1
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, BF16, 31)
    dy = normal(gen, B, T, H, P, dtype=BF16)
    x[:, T // 2:], dy[:, T // 2:] = x[:, :T // 2], -dy[:, :T // 2]
    dy[:, 700] += 2.0 ** -7 * dy[:, 700]
    dy = dy.to(BF16).double()
    log("case ssm dD cancels")
    got = kata.ssm_bwd(up(x, BF16), up(dt, BF16), up(A), up(Bm, BF16), up(Cm, BF16), up(D), up(bias), up(dy, BF16))
    want = (x * dy).sum((0, 1, 3))
    assert (want != 0).all()
    near(got[5], want, ref.EPS32 * want.abs(), "dD")


def test_ssm_parameter_gradients_turn_with_dy(kata):  # noqa: F811
    """The gradients of -dy are the negatives but for what the bf16 matrix cores do not round
    evenly: they cut off what stands below the last bit of the largest term, by 1.2e-10 of a sum's size
    on average where the terms are of one size, 1.8e-9 where small ones are added to it.  Of 64 x B T sums
    with one sign that is 1.2e-10 sqrt(64 B T) = 1.7e-7 of a dA whose terms have both signs; three times
    that is allowed of the mean over 16 heads."""
    B, T, H, G, N, P = 8, 4096, 16, 1, 64, 64
    gen = torch.Generator(device=DEV).manual_seed(8)

    def act(*shape):
        return torch.nn.functional.silu(torch.randn(shape, generator=gen, device=DEV)).to(BF16)
    x, Bm, Cm = act(B, T, H, P), act(B, T, G, N), act(B, T, G, N)
    dt = (torch.randn((B, T, H), generator=gen, device=DEV) * 0.5).to(BF16)
    dy = (torch.randn((B, T, H, P), generator=gen, device=DEV) * 0.1).to(BF16)
    A, bias = torch.full((H,), -1.0, device=DEV), torch.full((H,), -4.0, device=DEV)
    log("case ssm turned dy")
    dA, ddA = (kata.ssm_bwd(x, dt, A, Bm, Cm, None, bias, g)[2].double() for g in (dy, -dy))
    off = ((dA + ddA) / 2).mean().abs() / dA.square().mean().sqrt()
    log(f"  dA: {off.item():.2e}")
    assert off <= 3 * 1.2e-10 * math.sqrt(64 * B * T), off.item()
