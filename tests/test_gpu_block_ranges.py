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


# ---- e4m3: values that are middles between two codes -------------------------------------

@pytest.mark.parametrize("rows", (1, 128))
def test_f8_quant_middles_go_to_the_even_code(kata, rows):  # noqa: F811
    """x = top v / 448 for the middles v that a top of 16 bits has in fp32 (those of significand 21,
    and 7 below the normal range): x 448 / top is v itself, a tie, whatever top / 448 rounds to."""
    gen = torch.Generator().manual_seed(5)
    n = 640
    middles = torch.tensor([21.0 * 2.0 ** k for k in range(-10, 5)] + [7 * 2.0 ** -10], dtype=torch.float64)
    tops = torch.randint(1, 1 << 16, (n // 128, n // 128), generator=gen).double()
    tops = tops.repeat_interleave(128, 0).repeat_interleave(128, 1)
    v = middles[torch.randint(0, len(middles), (n, n), generator=gen)]
    sign = torch.randint(0, 2, (n, n), generator=gen) * 2.0 - 1
    x = sign * tops * v / 448
    at = torch.arange(128)
    for i in range(0, n, 128):
        for j in range(0, n, 128):
            x[i + at, j + at] = tops[i + at, j + at]  # the largest of every row and column of a block
    assert torch.equal(x.float().double(), x) and torch.equal(x * 448 / tops, (x * 448 / tops).float().double())
    x = x.float()
    got = kata.f8_quant(up(x), rows=rows, transposed=True)
    for g, w, name in zip(got, (*ref.quantise(x, rows), *ref.quantise(x.t(), rows)), ("q", "scale", "qt", "scale_t")):
        assert torch.equal(g.float().cpu().double(), w.double()), name


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("weight", (False, True))
@pytest.mark.parametrize("M,D", ((2048, 1000), (200, 3100)))
def test_add_norm_middles_go_to_the_even_code(kata, M, D, weight, dtype):  # noqa: F811
    """Rows (and weights) of 8 bits, whose quotients by their block's largest are middles in one of
    500 values.  The row's factor stands in both and leaves the quotient; products of 16 bits
    times 448 are exact in fp64, and so is a quotient that has few bits."""
    gen = torch.Generator().manual_seed(D)
    x = normal(gen, M, D, dtype=BF16)
    w = normal(gen, D, dtype=BF16) if weight else None
    q, _, _ = kata.add_norm_f8_fwd(up(x, dtype), up(w))
    v = x if w is None else x * w
    top = torch.nn.functional.pad(v.abs(), (0, -D % 128)).unflatten(1, (-1, 128)).amax(-1)
    v = v * 448 / ref.spread(top, 1, M, D)
    ties = ref.to_e4m3(v * (1 - 2.0 ** -40)) != ref.to_e4m3(v * (1 + 2.0 ** -40)).clamp(-448, 448)
    assert 1e-4 * v.numel() < int(ties.sum())
    assert torch.equal(q.float().cpu().double(), ref.to_e4m3(v))


def test_add_norm_codes_at_the_least_scale(kata):  # noqa: F811
    """A block whose largest value is at most 448 x 2^-126: codes of y 2^126."""
    gen = torch.Generator().manual_seed(2)
    x, w = normal(gen, 5, 300, dtype=F32), normal(gen, 300, dtype=F32)
    w[128:256] = (w[128:256] * 2.0 ** -121).float().double()
    q, scale, _ = kata.add_norm_f8_fwd(up(x), up(w))
    want = ref.norm(x, w, float(torch.tensor(1e-6)))
    assert (scale[:, 1] == 2.0 ** -126).all()
    v = want[:, 128:256] * 2.0 ** 126
    # w is of 24 bits: no middles but by chance (none within 2^-40)
    assert torch.equal(ref.to_e4m3(v * (1 - 2.0 ** -40)), ref.to_e4m3(v * (1 + 2.0 ** -40)))
    assert torch.equal(q.float().cpu().double()[:, 128:256], ref.to_e4m3(v))


# ---- product: scales whose product leaves fp32 -------------------------------------------

def far_operands(gen, M, N, K, rows, how):
    """Codes and scales: `apart`: every third block's scales are about 2^66 each and its codes share
    no k (a product of 0), the others' 2^90 and 2^-90; `faint`: 2^66 each, codes of 2^-9;
    `low`: 2^-70 and 2^-50; `least`: blocks without values beside ordinary ones."""
    (a, sa), (b, sb) = operand(gen, M, K, 1), operand(gen, N, K, rows)
    kb, k = torch.arange(sa.shape[1]), torch.arange(K)
    third = kb % 3 == 0
    if how == "apart":
        sa = torch.where(third, sa * 2.0 ** 72, sa * 2.0 ** 90)
        sb = torch.where(third, sb * 2.0 ** 72, sb * 2.0 ** -90)
        of = third[k // 128]
        a[:, of & (k % 128 >= 64)] = 0.0
        b[:, of & (k % 128 < 64)] = 0.0
    elif how == "faint":
        a, b = a.sign() * 2.0 ** -9, b.sign() * 2.0 ** -9
        sa, sb = torch.full_like(sa, 2.0 ** 66), torch.full_like(sb, 2.0 ** 66)
    elif how == "low":
        sa, sb = sa * 2.0 ** -70, sb * 2.0 ** -50
    else:
        a[:, third[k // 128]] = 0.0
        sa = torch.where(third, 2.0 ** -126, sa)
        b[:, ~third[k // 128]] = 0.0
        sb = torch.where(third, sb, 2.0 ** -126)
    return (a, sa.float()), (b, sb.float())


FAR = [(33, 130, 1000, "even"), (64, 40, 4500, "even"), (8, 8200, 700, "even"), (100, 300, 1152, "even"),
       (100, 300, 1152, "odd"), (70, 200, 2500, "even"), (70, 200, 2500, "odd")]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("rows", (1, 128))
@pytest.mark.parametrize("M,N,K,lay", FAR)
def test_f8_gemm_scales_whose_product_leaves_fp32(kata, M, N, K, lay, rows, dtype):  # noqa: F811
    gen = torch.Generator().manual_seed(M + N + K)
    for how in ("apart", "faint", "low", "least"):
        (a, sa), (b, sb) = far_operands(gen, M, N, K, rows, how)
        want, mag, top = ref.product(a, sa, b, sb, rows)
        assert float(want.abs().max()) < 3e38
        tol = ref.ROUND[dtype] * want.abs() + (2 * min(K, 128) + ref.blocks(K) + 32) * EPS * mag + LEAST[dtype]
        if dtype == BF16:
            tol = tol + 7 * 2.0 ** -13 * top
        log(f"case f8_gemm scales {how} M{M} N{N} K{K} rows{rows} {dtype} {lay}")
        c = kata.f8_gemm(laid(a, lay), up(sa), laid(b, lay), up(sb), dtype=dtype)
        near(c, want, tol, "c")


@pytest.mark.parametrize("lay", ("even", "odd"))
@pytest.mark.parametrize("rows", (1, 128))
def test_f8_gemm_large_tiles(kata, rows, lay):  # noqa: F811
    """The largest tiles, on aligned and unaligned rows, of ordinary scales and of far ones."""
    M, N, K = 4096, 4097, 700
    gen = torch.Generator().manual_seed(rows)
    at = torch.randperm(M, generator=gen)[:24]
    at[:4] = torch.tensor([0, M - 1, M // 2, 255])
    for how in ("ordinary", "apart", "low"):
        log(f"case f8_gemm large {how} rows{rows} {lay}")
        if how == "ordinary":
            (a, sa), (b, sb) = operand(gen, M, K, 1), operand(gen, N, K, rows)
        else:
            (a, sa), (b, sb) = far_operands(gen, M, N, K, rows, how)
        c = kata.f8_gemm(laid(a, lay), up(sa), laid(b, lay), up(sb))
        want, mag, top = ref.product(a[at], sa[at], b, sb, rows)
        tol = 2.0 ** -8 * want.abs() + (256 + ref.blocks(K) + 32) * EPS * mag + 7 * 2.0 ** -13 * top
        near(c[at.to(DEV)], want, tol, "rows")
        whole = (a.double() * ref.spread(sa, 1, M, K)) @ (b.double() * ref.spread(sb, rows, N, K)).t()
        off = float((c.cpu().double() - whole).norm() / whole.norm())
        assert off <= 2.0 ** -8, off


def test_f8_gemm_far_scales_in_one_block_only(kata):  # noqa: F811
    """Far scales in one group of blocks and ordinary ones in the others, and the ones that spread."""
    gen = torch.Generator().manual_seed(11)
    M, N, K = 150, 200, 1700
    for at, dtype in ((0, F32), (5, F32), (13, F32), (5, BF16)):
        (a, sa), (b, sb) = operand(gen, M, K, 1), operand(gen, N, K, 128)
        a[:, at * 128:at * 128 + 128] = 0.0
        sa[:, at], sb[:, at] = 3e19, 3e19
        want, mag, top = ref.product(a, sa, b, sb, 128)
        tol = ref.ROUND[dtype] * want.abs() + (288 + ref.blocks(K)) * EPS * mag + (7 * 2.0 ** -13 * top if dtype == BF16 else 0)
        near(kata.f8_gemm(laid(a, "even"), up(sa), laid(b, "even"), up(sb), dtype=dtype), want, tol, "c")
        sa[7, at] = float("inf")
        sb[1, (at + 1) % 13] = float("nan")
        c = kata.f8_gemm(laid(a, "even"), up(sa), laid(b, "even"), up(sb), dtype=dtype).cpu()
        bad = torch.zeros((M, N), dtype=torch.bool)
        bad[7] = bad[:, 128:] = True
        assert torch.equal(~torch.isfinite(c), bad)
        assert torch.equal(c[~bad].double().sub(want[~bad]).abs() <= tol[~bad], torch.ones(int((~bad).sum()), dtype=torch.bool))


# ---- gated linear recurrence: gates that cancel their biases --------------------------------

@pytest.mark.parametrize("dtype", (BF16, F32))
def test_recur_gates_that_cancel_their_biases(kata, dtype):  # noqa: F811
    """Biases up to 3000 against gates as far on the other side: what is left of them is exact, and
    results are as near as without either."""
    B, T, D = 2, 200, 16
    gen = torch.Generator().manual_seed(7)
    base = torch.tensor([20.0, -20.0, 43.0, -43.0, 300.0, -300.0, 3008.0, -3008.0], dtype=torch.float64).repeat(2)
    x, dy = normal(gen, B, T, D, dtype=dtype), normal(gen, B, T, D, dtype=dtype)
    r, i = ((base + normal(gen, B, T, D)).to(dtype).double() for _ in range(2))
    bias = (-base + 0.37).float().double()
    lam = (torch.rand(D, generator=gen, dtype=torch.float64) * 4 - 5).float().double()
    dev = [up(t, dtype) for t in (x, r, i)] + [up(lam), up(bias), up(bias)]
    log(f"case recur cancelled gates {dtype}")
    leaf = [t.clone().requires_grad_() for t in (x, r, i, lam, bias, bias)]
    want, h = ref.recur(*leaf)
    err = ref.recur_errors(x, r, i, lam, bias, bias, 8.0, None, None, dy)
    y, last = kata.recur_fwd(*dev, final_state=True)
    near(y, want, ref.ROUND[dtype] * want.abs() + err["y"], "y")
    near(last, h, err["h"] + EPS * h.abs(), "state")
    grads = torch.autograd.grad((want * dy).sum(), leaf)
    for g, w, name in zip(kata.recur_bwd(*dev, up(dy, dtype)), grads, ("dx", "dr", "di", "dlam", "drb", "dib")):
        near(g, w, (ref.ROUND[dtype] if g.dim() == 3 else EPS) * w.abs() + err[name], name)
    state = torch.zeros((B, D), device=DEV)
    out = kata.recur_step(state, *(t[:, 0].contiguous() for t in dev[:3]), *dev[3:])
    near(state, want[:, 0], err["y"][:, 0] + EPS * want[:, 0].abs(), "step")
    near(out, want[:, 0], ref.ROUND[dtype] * want[:, 0].abs() + err["y"][:, 0], "step's output")


@pytest.mark.parametrize("T", (20, 70, 300))
def test_recur_forgets_large_states(kata, T):  # noqa: F811
    """Rates at which a = 0, or at which a run's tokens leave less than fp32 holds, meet states and
    gradients of 1e37: what a run adds to what is left of them is at most 2^-149 of each."""
    big, few = 1e37, 1e37 * 2.0 ** -148
    x = torch.linspace(-2, 2, T * 2, device=DEV).view(1, T, 2)
    gate, zeros = torch.zeros_like(x), torch.zeros(2, device=DEV)
    lam = torch.tensor([3e38, 30.0], device=DEV)  # the second: 8 x 30 / 2 = 120 a token
    h0 = torch.full((1, 2), big, device=DEV)
    _, starts = kata.recur_fwd_train(x, gate, gate, lam, zeros, zeros, state=h0)
    assert (starts[:, 1:].abs() <= 1.0 + few).all()  # sigmoid(0) x
    dh = torch.empty_like(h0)
    kata.recur_bwd(x, gate, gate, lam, zeros, zeros, torch.zeros_like(x), state=h0, dstate=h0, dstate_in=dh)
    assert (dh.abs() <= few).all()
    # 16 tokens of rate 6 leave e^-96 of a state, which fp32 has as a subnormal number: a run's
    # factor is off by up to 2^-149, what it hands on decays on; rates are off by 16 2^-24
    lam = torch.log(torch.expm1(torch.full((2,), 1.5, dtype=torch.float64))).float().to(DEV)
    y = kata.recur_fwd(torch.zeros_like(x), gate, gate, lam, zeros, zeros, state=h0).cpu().double()[0]
    t = torch.arange(T, dtype=torch.float64)
    want = float(h0[0, 0]) * torch.exp(-6.0 * (t + 1))
    tol = (6 * (t + 1) * 16 * EPS + 2.0 ** -20) * want + LEAST[F32]
    tol = tol + (t >= 16) * few * torch.exp(-6.0 * (t % 16 + 1))
    assert ((y - want[:, None]).abs() <= tol[:, None]).all()
