"""The operators of a layer in 8 bits on the GPU at the ends of their ranges, against their
definitions in fp64 (block_reference.py): rows whose sums leave fp32, values that are middles
between two codes, scales whose product leaves fp32, gates that cancel their biases.

Tolerances as in test_gpu_block.py; where results may be subnormal, half of the type's least step
is added (2^-150, bf16 2^-134) for each rounding on the way."""
from __future__ import annotations

import pytest
import torch

import block_reference as ref
from gpu_helpers import log
from test_gpu_block import EPS, F8, bits, kata, laid, operand  # noqa: F401  (kata: the fixture)
from test_gpu_mixer import BF16, DEV, F32, near, normal, up

pytestmark = pytest.mark.gpu
LEAST = {F32: 2.0 ** -149, BF16: 2.0 ** -133}


# ---- residual norm -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("size,dsize", ((1e36, 1.0), (1e-36, 1.0), (1e-25, 1e-21), (1e-37, 1e-30), (1e15, 1e30),
                                        (1e-8, 1e-33)))
@pytest.mark.parametrize("M,D", ((5, 130), (3, 4100), (2100, 96), (1, 9000)))
def test_add_norm_gradients_whose_sums_leave_fp32(kata, M, D, size, dsize, dtype):  # noqa: F811
    """The sum of s (w dy) past fp32's range at either end, with gradients that follow s, so that
    most of them is taken off by that sum."""
    log(f"case add_norm_bwd M{M} D{D} s {size} dy {dsize} {dtype}")
    gen = torch.Generator().manual_seed(M + D)
    unit = normal(gen, M, D)
    s, w = (unit * size).to(dtype).double(), normal(gen, D, dtype=F32)
    dy = (dsize * (unit * w.sign() + 0.5 * normal(gen, M, D))).to(dtype).double()
    dy[0, ::2] = 0.0
    leaf = [s.clone().requires_grad_(), w.clone().requires_grad_()]
    grads = torch.autograd.grad(ref.norm(*leaf, 0.0), leaf, dy)
    dx, dw = kata.add_norm_bwd(up(s, dtype), up(w), up(dy, dtype), eps=0.0)
    inv = 1 / torch.sqrt(s.square().mean(-1, keepdim=True))
    g, hat = (dy * w).abs(), (s * inv).abs()
    mag = inv * (g + hat * (g * hat).mean(-1, keepdim=True))
    near(dx, grads[0], ref.ROUND[dtype] * grads[0].abs() + (2 * D + 40) * EPS * mag + LEAST[dtype], "dx")
    near(dw, grads[1], (M // 1024 + D / 2 + 60) * EPS * (dy.abs() * hat).sum(0), "dw")


@pytest.mark.parametrize("M,D", ((3, 200), (2100, 96)))
def test_add_norm_rows_without_gradients(kata, M, D):  # noqa: F811
    """Rows whose dy is 0 (tokens that a loss leaves out) hand on dsum as it is."""
    gen = torch.Generator().manual_seed(D)
    s, dy, dsum = (normal(gen, M, D, dtype=BF16) for _ in range(3))
    w = up(normal(gen, D, dtype=F32))
    out = torch.arange(M) % 3 == 1
    dy[out] = 0.0
    dx, dw = kata.add_norm_bwd(up(s, BF16), w, up(dy, BF16), up(dsum, BF16))
    assert torch.equal(dx.cpu().double()[out], dsum[out])
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
