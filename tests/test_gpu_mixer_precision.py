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
from test_gpu_mixer import BF16, DEV, F32, ROUND, kata, near, normal, ssm_inputs, up  # noqa: F401

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
