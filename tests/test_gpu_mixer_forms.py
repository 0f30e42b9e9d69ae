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


# ---- what the launch rules choose for many tokens or heads ---------------------------------
# Each test says by the sizes which form it takes; where a call has a workspace, its bytes are
# those of that form.

def up256(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,D,W", ((2, 1000, 4168, 4), (1, 1000, 1101, 3)))
def test_conv_long_runs(kata, B, T, D, W, dtype):  # noqa: F811
    """Forward: 65536 threads or more, in pieces or one by one, walk 16 tokens each; backward of
    1024 waves or more: 32."""
    pieces = D % 8 == 0
    assert B * -(-T // 16) * D // ((8 if dtype == BF16 else 4) if pieces else 1) >= 65536
    waves = B * -(-T // 32) * -(-D // 256)
    run = 32 if waves >= 1024 else 8
    assert (run == 32) == pieces
    slices = min(256, -(-(B * -(-T // run)) // 4))
    assert kata.lib().kata_conv_bwd_workspace_bytes(B, T, D, W, 1) == up256(slices * D * (W + 1) * 4)
    many_conv(kata, B, T, D, W, dtype)


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_conv_several_runs_a_wave(kata, dtype):  # noqa: F811
    """Backward of 33000 tokens: 1032 runs of 32 on 256 x 4 waves."""
    assert kata.lib().kata_conv_bwd_workspace_bytes(1, 33000, 24, 2, 1) == up256(256 * 24 * 3 * 4)
    many_conv(kata, 1, 33000, 24, 2, dtype)


def many_conv(kata, B, T, D, W, dtype):  # noqa: F811
    from test_gpu_mixer import test_conv_fwd_and_bwd as check
    check(kata, B, T, D, W, dtype)


def test_conv_long_runs_of_a_padded_batch(kata):  # noqa: F811
    """Runs of 16 with lengths that end inside and before them, a first state and the last rows."""
    B, T, D, W, dtype = 6, 400, 3600, 4, BF16
    gen = torch.Generator().manual_seed(12)
    assert B * -(-T // 16) * D // 8 >= 65536
    lengths = [400, 0, 1, 17, 399, 32]
    x, state = normal(gen, B, T, D, dtype=dtype), normal(gen, B, W - 1, D, dtype=dtype)
    w, bias = normal(gen, D, W, dtype=F32), normal(gen, D, dtype=F32)
    behind = torch.arange(T)[None] >= torch.tensor(lengths)[:, None]
    xs = up(x, dtype)
    xs[behind.to(DEV)] = float("nan")  # never read
    log("case conv long runs with lengths")
    y = torch.full((B, T, D), 7.0, dtype=dtype, device=DEV)
    y, last = kata.conv_fwd(xs, up(w), up(bias), state=up(state, dtype), y=y, final_state=True,
                            lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))
    want, rows = ref.conv(x, w, bias, True, state, lengths)
    assert (y.cpu()[behind] == 7.0).all()
    tol = ROUND(dtype) * want.abs() + 1.1 * (W + 16) * ref.EPS32 * conv_mag(x, w, bias, state)
    near(y.cpu().double().masked_fill(behind[..., None], 0), want, tol, "y")
    assert torch.equal(last.cpu().double(), rows)


def norm_parts(B, T, H, d):
    """Heads of a forward's workgroup, and of the backward's: tokens a lane group walks, heads,
    partial sums."""
    lanes = 2 if d <= 16 else 4 if d <= 32 else 8 if d <= 64 else 16 if d <= 128 else 32
    n = -(-B * T * lanes // 256)

    def split(blocks):
        return -(-H // min(-(-512 // blocks), H))
    walk = -(-n // 512)
    blocks = -(-n // walk)
    return split(n), walk, split(blocks), blocks * -(-H // split(blocks))


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,Hq,Hk,d,r,forward,walk,backward", (
    (1, 1500, 5, 3, 256, 64, 3, 1, 3),   # some heads of a token at a time, queries and keys among them
    (3, 1500, 5, 2, 256, 256, 7, 2, 4),  # forward all heads, four and then the rest; two tokens a group
    (2, 4095, 5, 2, 256, 32, 7, 2, 7),   # backward all heads as well
    (2, 8500, 6, 0, 64, 40, 6, 2, 3),    # rows in single elements, no keys
    (1, 70000, 1, 1, 16, 16, 2, 2, 1)))
def test_norm_heads_in_turn(kata, B, T, Hq, Hk, d, r, forward, walk, backward, dtype):  # noqa: F811
    from test_gpu_mixer import test_norm_fwd_and_bwd as check
    parts = norm_parts(B, T, Hq + Hk, d)
    assert parts[:3] == (forward, walk, backward)
    assert kata.lib().kata_qk_norm_bwd_workspace_bytes(B, T, Hq, Hk, d, 1) == up256(parts[3] * 2 * d * 4)
    check(kata, B, T, Hq, Hk, d, r, dtype)


def ssm_parts(B, T, H, G, N, P, dtype):
    """Spans, heads of a gradients' workgroup, and the bytes of both workspaces."""
    L = 64 if dtype == BF16 else 32
    NC, blocks, room = -(-T // L), -(-P // 64), 256 if N > 64 else 512
    BHP = B * H * blocks
    n = max(1, min(-(-1024 // BHP), NC // (2 if BHP * (NC // 4) < 256 else 4)))
    spans = -(-NC // -(-NC // n))
    split = min(-(-room // (B * G * NC)), H // G)
    heads = -(-(H // G) // split)
    parts = -(-(H // G) // heads)
    NP = 32 if N <= 32 else 64 if N <= 64 else 128
    logs, gaps = up256(B * H * NC * L * 16), B * H * (spans - 1)
    fwd = logs + up256(gaps * N * P * 4) + up256(gaps * 8)
    bwd = (logs + up256(2 * gaps * N * P * 4) + up256(2 * gaps * 8) + up256(2 * BHP * NC * 64 * NP * 4)
           + up256(B * NC * 3 * H * 8) + (2 * up256(parts * B * T * G * N * 4) if parts > 1 else 0))
    return spans, heads, fwd, bwd


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P,heads", (
    (64, 130, 5, 1, 16, 16, {BF16: 2, F32: 3}),  # of five heads two (three) at a time, the rest less
    (128, 200, 3, 1, 16, 24, 3), (128, 200, 6, 2, 40, 8, 3),  # all of a group's heads
    (128, 200, 2, 1, 8, 72, 2),  # heads of two blocks of columns
    (64, 200, 3, 1, 72, 8, 3), (64, 200, 2, 1, 100, 72, 2)))  # eight waves
def test_ssm_gradients_heads_in_turn(kata, B, T, H, G, N, P, heads, dtype):  # noqa: F811
    from test_gpu_mixer import test_ssm_bwd as check
    spans, got, fwd, bwd = ssm_parts(B, T, H, G, N, P, dtype)
    code = 1 if dtype == BF16 else 0
    assert got == (heads[dtype] if isinstance(heads, dict) else heads)
    assert kata.ssm_workspace_bytes(B, T, H, G, N, P, code) == fwd
    assert kata.ssm_workspace_bytes(B, T, H, G, N, P, code, True) == bwd
    check(kata, B, T, H, G, N, P, dtype)


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,H,G,N,P,several", ((1, 60, 2, 1, 64, 64, False), (64, 300, 16, 1, 16, 16, False),
                                                 (1, 1100, 2, 1, 64, 64, True), (2, 700, 3, 1, 100, 40, True),
                                                 (1, 900, 2, 2, 20, 130, True)))
def test_ssm_fwd_without_a_state(kata, B, T, H, G, N, P, several, dtype):  # noqa: F811
    """y of the calls that return no state, in one span and in several."""
    n = ssm_parts(B, T, H, G, N, P, dtype)[0]
    assert n > 2 if several else n == 1
    gen, x, dt, A, Bm, Cm, D, bias = ssm_inputs(B, T, H, G, N, P, dtype, B * T + N)
    A = A / 8
    A = A.float().double()
    S0 = normal(gen, B, H, N, P, dtype=F32)
    for state in (None, S0):
        log(f"case ssm no state B{B} T{T} H{H} G{G} N{N} P{P} {dtype} state{state is not None} spans{n}")
        y = kata.ssm_fwd(up(x, dtype), up(dt, dtype), up(A), up(Bm, dtype), up(Cm, dtype), up(D), up(bias),
                         state=up(state))
        want = ref.scan(x, dt, A, Bm, Cm, D, bias, True, state)[0]
        mag = ref.scan_mag(x, dt, A, Bm, Cm, D, bias, True, state, None)[0]
        near(y, want, ssm_tol(want, mag, dtype, N, T), "y")
