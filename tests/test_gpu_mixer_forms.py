"""The mixer operators' calls and forms that test_gpu_mixer.py does not reach: arguments by
name, missing ones, and what the launch rules choose for many tokens or heads."""
from __future__ import annotations

import pytest
import torch

import mixer_reference as ref
from gpu_helpers import log
from test_gpu_mixer import (BF16, DEV, F32, ROUND, conv_mag, hat_scale, kata, near, normal,  # noqa: F401
                            ssm_inputs, ssm_tol, state_tol, up)

pytestmark = pytest.mark.gpu


# ---- the binding ------------------------------------------------------------------------

def test_arguments_by_name(kata):  # noqa: F811
    gen = torch.Generator().manual_seed(1)
    x, w = up(normal(gen, 2, 9, 16, dtype=F32)), up(normal(gen, 16, 4, dtype=F32))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = kata.conv_fwd(w=w, x=x, stream=side)
    side.synchronize()
    assert torch.equal(y, kata.conv_fwd(x, w))
    q = x.view(2, 9, 2, 8)
    assert torch.equal(kata.qk_norm_fwd(q=q)[0], kata.qk_norm_fwd(q)[0])


def test_norm_gradients_need_the_outputs(kata):  # noqa: F811
    q = torch.zeros((1, 3, 2, 8), device=DEV)
    dq = torch.zeros((1, 2, 3, 8), device=DEV)
    for k, grads in ((None, dict()), (q, dict(dq=dq)), (None, dict(dq=dq, dk=dq)), (q, dict(dk=dq))):
        with pytest.raises(ValueError, match="expected dq"):
            kata.qk_norm_bwd(q, k, **grads)


def test_ssm_step_reads_no_token_strides(kata):  # noqa: F811
    """kata_ssm_step with token strides of anything, as in a struct that is not cleared."""
    B, H, G, N, P = 3, 2, 1, 16, 16
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, 1, H, G, N, P, F32, 6)
    x, dt, Bm, Cm = (up(t)[:, 0].contiguous() for t in (x, dt, Bm, Cm))
    A, D, bias = up(A), up(D), up(bias)
    S0 = up(normal(gen, B, H, N, P, dtype=F32))
    S = S0.clone()
    want = kata.ssm_step(S, x, dt, A, Bm, Cm, D, bias)
    for junk in (-1, -(1 << 62), (1 << 63) - 1, 7):
        strides = [H * P, junk, P, H, junk, 1, G * N, junk, N, G * N, junk, N, H * P, junk, P]
        again, y = S0.clone(), torch.zeros_like(x)
        rc = kata.lib().kata_ssm_step(*(t.data_ptr() for t in (again, x, dt, A, Bm, Cm, D, bias, y)), B, H, G, N, P,
                                      kata._SsmStrides(*strides), 1, kata.KATA_F32,
                                      torch.cuda.current_stream().cuda_stream)
        assert rc == kata.KATA_OK, junk
        assert torch.equal(y, want) and torch.equal(again, S)
