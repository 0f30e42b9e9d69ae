"""The operators of a layer in 8 bits on the GPU against their definitions in fp64
(block_reference.py), element by element.

Tolerances.  An output is rounded once to its type (`ROUND`, relative to the value); sums of n
fp32 terms and the rounded functions in them are off by at most (n + 16) 2^-24 of the terms'
magnitudes.  Codes: half a step of e4m3 is 2^-4 of the value, 2^-10 of the scale below its normal
range.  The matrix instruction for e4m3, which products in bf16 come from, cuts a product to 2^-13
of its group's largest, at most seven times in a group of eight."""
from __future__ import annotations

import pytest
import torch

import block_reference as ref
from gpu_helpers import log
from test_gpu_mixer import BF16, DEV, F32, near, normal, up, wide

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
EPS = ref.EPS32


@pytest.fixture(scope="module")
def kata():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_17419_amd as k
    k.lib()  # raises if libkata.so is missing: no fallback
    return k


def flat(*outs):
    return [t for o in outs for t in (o if isinstance(o, tuple) else (o,)) if t is not None]


def bits(t):
    return t.contiguous().view(torch.uint8) if t.dtype is F8 else t


# ---- residual norm -------------------------------------------------------------------

NORM = [(1, 1), (3, 7), (5, 64), (2, 130), (300, 1024), (2100, 96), (2050, 1000), (2049, 2048), (4, 2049),
        (3, 4100), (2, 8192), (2, 9000), (1, 32768), (3, 127)]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("M,D", NORM)
def test_add_norm(kata, M, D, dtype):
    gen = torch.Generator().manual_seed(M + D)
    x, res = normal(gen, M, D, dtype=dtype), normal(gen, M, D, dtype=dtype, std=2.0)
    dsum = normal(gen, M, D, dtype=dtype)
    w = normal(gen, D, dtype=F32)
    for with_res, weight, pad, ydt in ((True, w, 0, dtype), (False, None, 0, F32), (True, w, 3, F32),
                                       (True, None, 8, dtype)):
        log(f"case add_norm M{M} D{D} {dtype} res{with_res} w{weight is not None} pad{pad} dy {ydt}")
        xs = wide(x, dtype, pad)
        rs = wide(res, dtype, pad) if with_res else None
        s = (x.float() + res.float()).to(dtype).double() if with_res else x
        want = ref.norm(s, weight, 1e-6)
        y, total = kata.add_norm_fwd(xs, up(weight), rs)
        assert torch.equal(total.cpu().double(), s)
        assert with_res or total is xs
        # the factor is off by half of a sum of D squares' error
        spread = (D / 2 + 20) * EPS * want.abs()
        near(y, want, ref.ROUND[dtype] * want.abs() + spread, "y")
        q, scale, total = kata.add_norm_f8_fwd(xs, up(weight), rs)
        assert torch.equal(total.cpu().double(), s)
        kb = ref.blocks(D)
        tops = torch.nn.functional.pad(want.abs(), (0, kb * 128 - D)).unflatten(1, (kb, 128)).amax(-1)
        near(scale, tops / 448, (D / 2 + 24) * EPS * tops / 448 + 2.0 ** -126, "scale")
        value = q.float().cpu().double() * ref.spread(scale.cpu(), 1, M, D)
        step = ref.spread(scale.cpu(), 1, M, D) * 2.0 ** -10
        near(value, want, torch.maximum(2.0 ** -4 * want.abs(), step) + 2 * spread, "codes")
        both = torch.empty((M, D), dtype=dtype, device=DEV)
        q2, scale2, _ = kata.add_norm_f8_fwd(xs, up(weight), rs, y=both)
        assert torch.equal(bits(q), bits(q2)) and torch.equal(scale, scale2) and torch.equal(both, y)
        # gradients
        dy = normal(gen, M, D, dtype=ydt)
        leaf = [s.clone().requires_grad_()] + ([] if weight is None else [weight.clone().requires_grad_()])
        grads = torch.autograd.grad(ref.norm(leaf[0], leaf[1] if weight is not None else None, 1e-6), leaf, dy)
        more = dsum if with_res else None
        dx, dw = kata.add_norm_bwd(total, up(weight), wide(dy, ydt, pad), None if more is None else wide(more, dtype, pad))
        inv = 1 / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6)
        g, hat = (dy * (1.0 if weight is None else weight)).abs(), (s * inv).abs()
        mag = inv * (g + hat * (g * hat).mean(-1, keepdim=True))
        want = grads[0] + (0 if more is None else more)
        near(dx, want, ref.ROUND[dtype] * want.abs() + (2 * D + 40) * EPS * mag, "dx")
        if weight is None:
            assert dw is None
        else:
            # a lane adds its rows (at most M / 1024 and eight) in fp32; each term's hat as y
            near(dw, grads[1], (M // 1024 + D / 2 + 60) * EPS * (dy.abs() * hat).sum(0), "dw")


def test_add_norm_in_place_and_leading_dimensions(kata):
    gen = torch.Generator().manual_seed(1)
    x, res = (up(normal(gen, 3, 5, 72, dtype=BF16), BF16) for _ in range(2))
    w = up(normal(gen, 72, dtype=F32))
    y, total = kata.add_norm_fwd(x, w, res)
    assert y.shape == x.shape and total.shape == x.shape
    one, s1 = kata.add_norm_fwd(x.view(15, 72), w, res.view(15, 72))
    assert torch.equal(one.view_as(y), y) and torch.equal(s1.view_as(total), total)
    q, scale, _ = kata.add_norm_f8_fwd(x, w, res)
    assert q.shape == x.shape and scale.shape == (3, 5, 1) and q.stride(1) % 16 == 0
    kept = res.clone()
    y2, total2 = kata.add_norm_fwd(x, w, kept, sum=kept)
    assert total2 is kept and torch.equal(kept, total) and torch.equal(y2, y)
    with pytest.raises(kata.KataError):
        kata.add_norm_fwd(x, w, res, y=x)
    with pytest.raises(kata.KataError):
        kata.add_norm_fwd(x, w, res, sum=x)
    with pytest.raises(ValueError):
        kata.add_norm_fwd(x, w, sum=torch.empty_like(x))
    with pytest.raises(ValueError):
        kata.add_norm_fwd(x.transpose(0, 1), w)
    with pytest.raises(TypeError):
        kata.add_norm_fwd(x, w, res.float())
    with pytest.raises(TypeError):
        kata.add_norm_fwd(x.half(), w)


def test_add_norm_non_finite_and_zero_rows(kata):
    x = torch.ones((6, 300), dtype=F32, device=DEV)
    x[1, 5], x[3, 299], x[4] = float("inf"), float("nan"), 0.0
    y, _ = kata.add_norm_fwd(x)
    q, scale, _ = kata.add_norm_f8_fwd(x)
    fine = [0, 2, 4, 5]
    assert torch.isfinite(y[fine]).all() and (y[4] == 0).all()
    assert y[3].isnan().all() and not torch.isfinite(y[1, 5])
    assert q.float()[3].isnan().all()
    assert (q.float()[4] == 0).all() and (scale[4] == 2.0 ** -126).all()
    assert torch.equal(bits(q)[0], bits(q)[5])


@pytest.mark.parametrize("size", (1e25, 1e-25))
@pytest.mark.parametrize("M,D", ((5, 130), (3, 4100), (2100, 96)))
def test_add_norm_rows_whose_squares_leave_fp32(kata, M, D, size):
    gen = torch.Generator().manual_seed(M)
    s, w, dy = (normal(gen, *n, dtype=F32) for n in ((M, D), (D,), (M, D)))
    s = (s * size).float().double()
    y, _ = kata.add_norm_fwd(up(s), up(w), eps=0.0)
    leaf = [s.clone().requires_grad_(), w.clone().requires_grad_()]
    want = ref.norm(*leaf, 0.0)
    near(y, want.detach(), (D / 2 + 22) * EPS * want.detach().abs(), "y")
    grads = torch.autograd.grad(want, leaf, dy)
    dx, dw = kata.add_norm_bwd(up(s), up(w), up(dy), eps=0.0)
    inv = 1 / torch.sqrt(s.square().mean(-1, keepdim=True))
    g, hat = (dy * w).abs(), (s * inv).abs()
    near(dx, grads[0], (2 * D + 40) * EPS * inv * (g + hat * (g * hat).mean(-1, keepdim=True)), "dx")
    near(dw, grads[1], (M // 1024 + D / 2 + 60) * EPS * (dy.abs() * hat).sum(0), "dw")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("M,D", ((2048, 1000), (200, 5000)))
def test_add_norm_codes_are_the_exact_ones(kata, M, D, dtype):
    """Codes to nearest of the exact quotients, wherever fp64 can tell the two apart: weights are
    of 24 bits, so that a quotient within 2^-40 of a middle would be chance (none is)."""
    gen = torch.Generator().manual_seed(D)
    x, w = normal(gen, M, D, dtype=dtype), normal(gen, D, dtype=F32)
    q, _, _ = kata.add_norm_f8_fwd(up(x, dtype), up(w))
    want = ref.norm(x, w, float(torch.tensor(1e-6)))  # the call takes eps in fp32
    kb = ref.blocks(D)
    top = torch.nn.functional.pad(want.abs(), (0, kb * 128 - D)).unflatten(1, (kb, 128)).amax(-1)
    v = want * 448 / ref.spread(top, 1, M, D)
    assert torch.equal(ref.to_e4m3(v * (1 - 2.0 ** -40)), ref.to_e4m3(v * (1 + 2.0 ** -40)).clamp(-448, 448))
    assert torch.equal(q.float().cpu().double(), ref.to_e4m3(v))


# ---- e4m3 ------------------------------------------------------------------------------

QUANT = [(1, 1), (1, 200), (128, 128), (130, 257), (7, 1000), (257, 64), (300, 384), (129, 131)]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("rows", (1, 128))
@pytest.mark.parametrize("M,K", QUANT)
def test_f8_quant_is_its_definition(kata, M, K, rows, dtype):
    """Every bit: fp32 divisions and products are rounded as IEEE says, on both sides, and codes of fp32
    values are those of the quotients themselves."""
    gen = torch.Generator().manual_seed(M * K)
    x = normal(gen, M, K, dtype=F32) * torch.exp(3 * normal(gen, M, 1, dtype=F32))
    x[0, 0] = 0.0
    if M > 3:
        x[1], x[2], x[3] = 0.0, x[2] * 2.0 ** -130, x[3] * 2.0 ** 100  # no values, subnormals, large ones
    x = x.to(dtype).float()
    want = (*ref.quantise(x, rows, dtype == BF16), *ref.quantise(x.t(), rows, dtype == BF16))
    for pad in (0, 3, 8):
        log(f"case f8_quant M{M} K{K} rows{rows} {dtype} pad{pad}")
        got = kata.f8_quant(wide(x.double(), dtype, pad), rows=rows, transposed=True)
        for g, r, name in zip(got, want, ("q", "scale", "qt", "scale_t")):
            assert torch.equal(g.float().cpu().double(), r.double()), name
    q, scale = kata.f8_quant(up(x, dtype), rows=rows)
    assert torch.equal(bits(q), bits(got[0])) and torch.equal(scale, got[1])
    tight = [torch.empty((M, K), dtype=F8, device=DEV), torch.empty((K, M), dtype=F8, device=DEV)]
    out = kata.f8_quant(up(x, dtype), rows=rows, transposed=True, q=tight[0], qt=tight[1])
    assert torch.equal(bits(out[0]), bits(got[0])) and torch.equal(bits(out[2]), bits(got[2]))


@pytest.mark.parametrize("rows", (1, 128))
def test_f8_quant_beside_the_middles(kata, rows):
    """fp32 values within three steps of the middles between neighbouring codes, the least
    (subnormal) codes' too."""
    gen = torch.Generator().manual_seed(3)
    codes = torch.arange(127, dtype=torch.uint8).view(F8).float().double()  # 0 to 448
    middles = (codes[1:] + codes[:-1]) / 2
    M = 640
    x = torch.empty((M, 128), dtype=F32)
    x[:, 0] = torch.rand(M, generator=gen) + 1.0
    x[:, 0] = x[torch.arange(M) // 128 * 128, 0]  # one for each block of either form
    x[:, 1:127] = (middles * x[:, :1].double() / 448).float()
    x[:, 127] = 0.0
    for k in range(3):
        x[:, 1:127] = torch.where((torch.arange(M) % 7 > 3 + k)[:, None], x[:, 1:127].nextafter(torch.tensor(9.0)), x[:, 1:127])
        x[:, 1:127] = torch.where((torch.arange(M) % 7 < 3 - k)[:, None], x[:, 1:127].nextafter(torch.tensor(0.0)), x[:, 1:127])
    got = kata.f8_quant(up(x), rows=rows, transposed=True)
    want = (*ref.quantise(x, rows), *ref.quantise(x.t(), rows))
    for g, w, name in zip(got, want, ("q", "scale", "qt", "scale_t")):
        assert torch.equal(g.float().cpu().double(), w.double()), name


def test_f8_quant_writes_its_rows_only_and_keeps_non_finite_in_their_blocks(kata):
    x = torch.ones((130, 200), device=DEV)
    x[2, 3], x[129, 190] = float("nan"), float("inf")
    codes = torch.full((130, 240), 7, dtype=torch.uint8, device=DEV)
    turned = torch.full((200, 160), 7, dtype=torch.uint8, device=DEV)
    q, scale, qt, scale_t = kata.f8_quant(x, transposed=True, q=codes.view(F8)[:, :200],
                                          qt=turned.view(F8)[:, :130])
    assert (codes[:, 200:] == 7).all() and (turned[:, 130:] == 7).all()
    bad = torch.zeros((130, 2), dtype=torch.bool, device=DEV)
    bad[129, 1] = True
    assert torch.equal(~torch.isfinite(scale), bad) and (scale[~bad] == torch.tensor(1.0) / 448).all()
    bad = torch.zeros((130, 200), dtype=torch.bool, device=DEV)
    bad[2, 3] = bad[129, 190] = True
    assert torch.equal(q.float().isnan(), bad) and torch.equal(qt.float().isnan(), bad.t())
    with pytest.raises(ValueError):
        kata.f8_quant(x, rows=64)
    with pytest.raises(ValueError):
        kata.f8_quant(x, qt=qt)


def operand(gen, n, K, rows, wild=False):
    x = normal(gen, n, K, dtype=F32) * torch.exp(normal(gen, n, 1, dtype=F32))
    if wild:
        x = x * torch.exp(4 * normal(gen, n, K, dtype=F32))
    return ref.quantise(x.float(), rows)


def laid(q, how):
    """Codes on the device: rows from multiples of 16 bytes on, next to each other, or off by one."""
    n, K = q.shape
    pad, skip = {"even": (-K % 16, 0), "tight": (0, 0), "odd": (1 + -K % 16, 1)}[how]
    raw = torch.full((n * (K + pad) + 16,), 0x7F, dtype=torch.uint8, device=DEV)  # NaN around the rows
    t = raw[skip:skip + n * (K + pad)].view(n, K + pad)[:, :K]
    t.copy_(q.float().to(F8).view(torch.uint8).to(DEV))
    return t.view(F8)


GEMM = [(1, 1, 1), (3, 5, 17), (16, 16, 128), (17, 33, 129), (8, 200, 512), (33, 130, 1000), (64, 96, 2200),
        (65, 130, 257), (100, 300, 1152), (128, 128, 128), (200, 640, 4096), (300, 257, 640), (50, 16, 8200)]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("rows", (1, 128))
@pytest.mark.parametrize("M,N,K", GEMM)
def test_f8_gemm(kata, M, N, K, rows, dtype):
    gen = torch.Generator().manual_seed(M * N + K)
    for wild in (False, True):
        (a, sa), (b, sb) = operand(gen, M, K, 1, wild), operand(gen, N, K, rows, wild)
        want, mag, top = ref.product(a, sa, b, sb, rows)
        tol = ref.ROUND[dtype] * want.abs() + (2 * min(K, 128) + ref.blocks(K) + 32) * EPS * mag
        if dtype == BF16:
            tol = tol + 7 * 2.0 ** -13 * top
        for how in ("even", "tight", "odd"):
            log(f"case f8_gemm M{M} N{N} K{K} rows{rows} {dtype} wild{wild} {how}")
            c = kata.f8_gemm(laid(a, how), up(sa), laid(b, how), up(sb), dtype=dtype)
            near(c, want, tol, "c")
    out = torch.full((M, N + 3), 7.0, dtype=dtype, device=DEV)
    again = kata.f8_gemm(laid(a, "odd"), up(sa), laid(b, "odd"), up(sb), out=out[:, 3:])
    assert torch.equal(again, c) and (out[:, :3] == 7).all()


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("M,N,K,rows", ((4096, 4097, 200, 128), (4100, 4096, 130, 1), (1152, 1024, 8200, 1),
                                        (2000, 1152, 1000, 128)))
def test_f8_gemm_many_tiles(kata, M, N, K, rows, dtype):
    """What the launch rule gives larger tiles, and split sums: rows from everywhere."""
    gen = torch.Generator().manual_seed(K)
    (a, sa), (b, sb) = operand(gen, M, K, 1), operand(gen, N, K, rows)
    log(f"case f8_gemm M{M} N{N} K{K} rows{rows} {dtype}")
    c = kata.f8_gemm(laid(a, "even"), up(sa), laid(b, "even"), up(sb), dtype=dtype)
    A = a.double() * ref.spread(sa, 1, M, K)
    B = b.double() * ref.spread(sb, rows, N, K)
    want = A @ B.t()
    at = torch.randperm(M, generator=gen)[:24]
    at[:4] = torch.tensor([0, M - 1, M // 2, 255])
    _, mag, top = ref.product(a[at], sa[at], b, sb, rows)
    tol = ref.ROUND[dtype] * want[at].abs() + (2 * min(K, 128) + ref.blocks(K) + 32) * EPS * mag
    near(c[at.to(DEV)], want[at], tol + (7 * 2.0 ** -13 * top if dtype == BF16 else 0), "rows")
    # all of it: a rounding of the result, and what ordinary operands lose to cut products
    off = float((c.cpu().double() - want).norm() / want.norm())
    assert off <= (2.0 ** -8 if dtype == BF16 else 1e-6), off
    slow = kata.f8_gemm(laid(a[at], "odd"), up(sa[at]), laid(b, "odd"), up(sb), dtype=dtype)
    near(slow, want[at], tol + (7 * 2.0 ** -13 * top if dtype == BF16 else 0), "unaligned rows")


def test_f8_gemm_non_finite_scales_shapes(kata):
    gen = torch.Generator().manual_seed(3)
    for M in (40, 90):
        (a, sa), (b, sb) = operand(gen, M, 300, 1), operand(gen, 260, 300, 128)
        a, b = laid(a, "even"), laid(b, "even")
        a.view(torch.uint8)[5, 299] = 0x7F
        b.view(torch.uint8)[7, 0] = 0xFF
        sa[9, 2] = float("inf")
        c = kata.f8_gemm(a, up(sa), b, up(sb))
        bad = torch.zeros((M, 260), dtype=torch.bool, device=DEV)
        bad[5] = bad[9] = bad[:, 7] = True
        assert torch.equal(~torch.isfinite(c), bad)
    lead = kata.f8_gemm(a.unflatten(0, (9, 10)), up(sa).unflatten(0, (9, 10)), b, up(sb))
    assert lead.shape == (9, 10, 260)
    assert torch.equal(lead.view(90, 260).nan_to_num(), c.nan_to_num())
    with pytest.raises(ValueError):
        kata.f8_gemm(a, up(sa), b[:, :200], up(sb))
    with pytest.raises(ValueError):
        kata.f8_gemm(a, up(sa)[:, :2].contiguous(), b, up(sb))
    with pytest.raises(TypeError):
        kata.f8_gemm(a.view(torch.uint8), up(sa), b, up(sb))
    with pytest.raises(TypeError):
        kata.f8_gemm(a, up(sa), b, up(sb), dtype=torch.float16)


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_f8_gemm_single_rows_and_repeated_rows(kata, dtype):
    """One row of either operand with any stride, and a row that stands for many."""
    gen = torch.Generator().manual_seed(6)
    (a, sa), (b, sb) = operand(gen, 90, 200, 1), operand(gen, 150, 200, 128)
    da, db, ua, ub = laid(a, "even"), laid(b, "even"), up(sa), up(sb)
    whole = kata.f8_gemm(da, ua, db, ub, dtype=dtype)
    row = da[:1].as_strided((1, 200), (7, 1))
    near(kata.f8_gemm(row, ua[:1], db, ub, dtype=dtype), whole[:1].cpu().double(),
         2 * ref.ROUND[dtype] * whole[:1].cpu().double().abs() + 2.0 ** -20, "one row of a")
    col = kata.f8_gemm(da, ua, db[:1].as_strided((1, 200), (3, 1)), ub[:1], dtype=dtype)
    near(col, whole[:, :1].cpu().double(), 2 * ref.ROUND[dtype] * whole[:, :1].cpu().double().abs() + 2.0 ** -20, "one of b")
    for rows in (5, 90):
        same_rows = da[3:4].expand(rows, 200)
        got = kata.f8_gemm(same_rows, ua[3:4].expand(rows, 2).contiguous(), db, ub, dtype=dtype)
        near(got, whole[3:4].expand(rows, 150).cpu().double(),
             2 * ref.ROUND[dtype] * whole[3:4].cpu().double().abs().expand(rows, 150) + 2.0 ** -20, "repeated rows")


def test_offsets_past_32_bits(kata):
    """Rows of one tensor further apart than 2^32 elements."""
    gen = torch.Generator().manual_seed(4)
    far = (1 << 32) + 16
    raw = torch.zeros((far + 4096,), dtype=torch.uint8, device=DEV)
    (a, sa), (b, sb) = operand(gen, 2, 256, 1), operand(gen, 80, 256, 128)
    for k in range(2):
        raw[k * far:k * far + 256] = a[k].float().to(F8).view(torch.uint8).to(DEV)
    at = raw.view(F8).as_strided((2, 256), (far, 1))
    b, sa, sb = laid(b, "even"), up(sa), up(sb)
    assert torch.equal(kata.f8_gemm(at, sa, b, sb), kata.f8_gemm(laid(a, "even"), sa, b, sb))
    # as the other operand of a tall product
    many, scales = b.repeat(2, 1), sb.repeat_interleave(128, 0)[:80].repeat(2, 1).contiguous()
    assert torch.equal(kata.f8_gemm(many, scales, at, sa), kata.f8_gemm(many, scales, laid(a, "even"), sa))
    del raw, at
    x = torch.zeros((far + 4096,), dtype=BF16, device=DEV)
    near_x = up(normal(gen, 2, 300, dtype=BF16), BF16)
    x[:300], x[far:far + 300] = near_x[0], near_x[1]
    xs = x.as_strided((2, 300), (far, 1))
    for p, q in zip(kata.add_norm_f8_fwd(xs), kata.add_norm_f8_fwd(near_x)):
        assert torch.equal(bits(p), bits(q))
    for p, q in zip(kata.f8_quant(xs, transposed=True), kata.f8_quant(near_x, transposed=True)):
        assert torch.equal(bits(p), bits(q))
    lam = up(normal(gen, 100, dtype=F32))
    seq = x.as_strided((2, 3, 100), (far, 100, 1))
    flat_seq = near_x.view(2, 3, 100)
    y = torch.empty((far + 4096,), dtype=BF16, device=DEV).as_strided((2, 3, 100), (far, 100, 1))
    kata.recur_fwd(seq, seq, seq, lam, y=y)
    assert torch.equal(y, kata.recur_fwd(flat_seq, flat_seq, flat_seq, lam))


# ---- gated linear recurrence ---------------------------------------------------------------

def recur_inputs(B, T, D, dtype, seed, slow=True):
    gen = torch.Generator().manual_seed(seed)
    x, r, i = (normal(gen, B, T, D, dtype=dtype) for _ in range(3))
    # decays from a token's to thousands of tokens', and some beyond
    lam = (torch.rand(D, generator=gen, dtype=torch.float64) * (14 if slow else 4) - (12 if slow else 2)).float().double()
    rb, ib = normal(gen, D, dtype=F32, std=0.5), normal(gen, D, dtype=F32, std=0.5)
    return gen, x, r, i, lam, rb, ib


RECUR = [(1, 1, 1), (2, 2, 3), (3, 15, 64), (1, 16, 130), (2, 17, 128), (1, 127, 5), (2, 128, 66), (1, 129, 257),
         (2, 300, 40), (1, 1000, 34), (1, 2500, 8)]


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("B,T,D", RECUR)
def test_recur(kata, B, T, D, dtype):
    gen, x, r, i, lam, rb, ib = recur_inputs(B, T, D, dtype, B * T + D)
    h0, dh = normal(gen, B, D, dtype=F32), normal(gen, B, D, dtype=F32)
    dy = normal(gen, B, T, D, dtype=dtype)
    for bias, state, dstate, pad, c in ((True, h0, dh, 0, 8.0), (False, None, None, 3, 1.0), (True, None, dh, 8, 8.0)):
        log(f"case recur B{B} T{T} D{D} {dtype} bias{bias} state{state is not None} pad{pad} c{c}")
        p = (rb, ib) if bias else (None, None)
        ins = [wide(t, dtype, pad) for t in (x, r, i)]
        dev = [*ins, up(lam), up(p[0]), up(p[1])]
        leaf = [None if t is None else t.clone().requires_grad_() for t in (x, r, i, lam, *p, state)]
        y, h = ref.recur(*leaf[:6], c, leaf[6])
        live = [t for t in leaf if t is not None]
        got = iter(torch.autograd.grad((y * dy).sum() + (0 if dstate is None else (h * dstate).sum()), live))
        want = [None if t is None else next(got) for t in leaf]
        err = ref.recur_errors(x, r, i, lam, *p, c, state, None, dy, dstate)
        R = ref.ROUND[dtype]
        out, last = kata.recur_fwd(*dev, c=c, state=up(state), final_state=True)
        near(out, y, R * y.abs() + err["y"], "y")
        near(last, h, err["h"] + EPS * h.abs(), "state")
        y2, starts = kata.recur_fwd_train(*dev, c=c, state=up(state))
        assert torch.equal(y2, out)
        dstate_in = None if state is None else torch.empty((B, D), device=DEV)
        how = dict(c=c, state=up(state), dstate=up(dstate), dstate_in=dstate_in)
        grads = kata.recur_bwd(*dev, wide(dy, dtype, pad), starts, **how)
        names = ("dx", "dr", "di", "dlam", "drb", "dib")
        for g, w, name in zip(grads, want, names):
            if w is None:
                assert g is None
                continue
            near(g, w, (R if name in ("dx", "dr", "di") else EPS) * w.abs() + err[name], name)
        if state is not None:
            near(dstate_in, want[6], err["dstate"], "dstate")
        kept = None if dstate_in is None else dstate_in.clone()
        again = kata.recur_bwd(*dev, wide(dy, dtype, pad), None, **how)
        assert all(torch.equal(u, v) for u, v in zip(flat(grads), flat(again)))
        assert kept is None or torch.equal(kept, dstate_in)


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("D", (48, 33))
def test_recur_padded_batch_then_steps(kata, dtype, D):
    """Lengths from none to all, forward, gradients, then token by token onwards."""
    lengths, T = [0, 1, 15, 16, 17, 128, 129, 300, 999, -1], 300
    B = len(lengths)
    gen, x, r, i, lam, rb, ib = recur_inputs(B, T + 4, D, dtype, D)
    h0, dh, dy = normal(gen, B, D, dtype=F32), normal(gen, B, D, dtype=F32), normal(gen, B, T, D, dtype=dtype)
    behind = torch.arange(T)[None] >= torch.tensor(lengths)[:, None]
    dev = [up(t[:, :T], dtype) for t in (x, r, i)]
    dys = up(dy, dtype)
    for t in (*dev, dys):
        t[behind.to(DEV)] = float("nan")  # never read
    par = [up(lam), up(rb), up(ib)]
    ln = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for state in (None, h0):
        log(f"case recur lengths D{D} {dtype} state {state is not None}")
        y = torch.full((B, T, D), 7.0, dtype=dtype, device=DEV)
        y, last = kata.recur_fwd(*dev, *par, state=up(state), lengths=ln, y=y, final_state=True)
        assert (y.cpu()[behind] == 7.0).all()
        ins = [t[:, :T] for t in (x, r, i)]
        leaf = [t.clone().requires_grad_() for t in (*ins, lam, rb, ib)]
        want, h = ref.recur(*leaf, 8.0, state, lengths)
        err = ref.recur_errors(*ins, lam, rb, ib, 8.0, state, lengths, dy, dh)
        near(y.cpu().double().masked_fill(behind[..., None], 0), want.detach(), ref.ROUND[dtype] * want.abs() + err["y"], "y")
        near(last, h.detach(), err["h"] + EPS * h.abs(), "state")
        grads = torch.autograd.grad((want * dy).sum() + (h * dh).sum(), leaf)
        for starts in (None, kata.recur_fwd_train(*dev, *par, state=up(state), lengths=ln)[1]):
            outs = [torch.full((B, T, D), 7.0, dtype=dtype, device=DEV) for _ in range(3)]
            back = torch.empty((B, D), device=DEV)
            got = kata.recur_bwd(*dev, *par, dys, starts, state=up(state), lengths=ln, dstate=up(dh), dx=outs[0],
                                 dr=outs[1], di=outs[2], dstate_in=back)
            for g, w, name in zip(got, grads, ("dx", "dr", "di", "dlam", "drb", "dib")):
                g = g.cpu()
                if name in ("dx", "dr", "di"):
                    assert (g[behind] == 7.0).all()
                    g = g.double().masked_fill(behind[..., None], 0)
                near(g, w, (ref.ROUND[dtype] if g.dim() == 3 else EPS) * w.abs() + err[name], name)
            assert torch.equal(back[0], up(dh)[0])  # of no tokens: passed through
        own = kata.recur_bwd(*dev, *par, dys, lengths=ln)
        assert all((t.cpu()[behind] == 0).all() for t in own[:3])
        h, e = h.detach(), err["h"]
        for t in range(T, T + 4):
            one = [v[:, t:t + 1] for v in (x, r, i)]
            out = kata.recur_step(last, *(up(v[:, 0], dtype) for v in one), *par)
            w, h2 = ref.recur(*one, lam, rb, ib, 8.0, h)
            e = ref.recur_errors(*one, lam, rb, ib, 8.0, h, None)["h"] + e  # the prompt's error, carried
            near(last, h2, e + EPS * h2.abs(), f"state {t - T}")
            near(out, w[:, 0], ref.ROUND[dtype] * w[:, 0].abs() + e, f"step {t - T}")
            h = h2


def test_recur_lengths_at_groups_of_spans(kata):
    """Sequences that end where spans, and groups of sixteen spans, of either direction end."""
    lengths, T, D = [1023, 1024, 1025, 2047, 2048, 2049, 4096, 4100], 4100, 10
    B = len(lengths)
    gen, x, r, i, lam, rb, ib = recur_inputs(B, T, D, F32, 77)
    h0, dh, dy = normal(gen, B, D, dtype=F32), normal(gen, B, D, dtype=F32), normal(gen, B, T, D, dtype=F32)
    leaf = [t.clone().requires_grad_() for t in (x, r, i, lam, rb, ib, h0)]
    y, h = ref.recur(*leaf[:6], 8.0, leaf[6], lengths)
    grads = torch.autograd.grad((y * dy).sum() + (h * dh).sum(), leaf)
    err = ref.recur_errors(x, r, i, lam, rb, ib, 8.0, h0, lengths, dy, dh)
    dev, ln = [up(t) for t in (x, r, i, lam, rb, ib)], torch.tensor(lengths, dtype=torch.int32, device=DEV)
    out, last = kata.recur_fwd(*dev, state=up(h0), lengths=ln, y=torch.zeros((B, T, D), device=DEV), final_state=True)
    near(out, y.detach(), EPS * y.detach().abs() + err["y"], "y")
    near(last, h.detach(), err["h"] + EPS * h.detach().abs(), "state")
    for starts in (None, kata.recur_fwd_train(*dev, state=up(h0), lengths=ln)[1]):
        back = torch.empty((B, D), device=DEV)
        got = kata.recur_bwd(*dev, up(dy), starts, state=up(h0), lengths=ln, dstate=up(dh), dstate_in=back)
        for g, w, name in zip((*got, back), grads, ("dx", "dr", "di", "dlam", "drb", "dib", "dstate")):
            near(g, w, EPS * w.abs() + err[name], name)


def test_recur_extreme_gates(kata):
    """Gates shut and open to their limits: rates of 0 (a = 1) and far past 1."""
    B, T, D = 1, 140, 8
    x = torch.full((B, T, D), 0.5, dtype=torch.float64)
    r, i = torch.zeros_like(x), torch.zeros_like(x)
    r[:, 60:70], r[:, 70:80], r[:, 80:90] = -200.0, 200.0, -3e38
    i[:, 30:40], i[:, 40:50] = -200.0, 200.0
    lam = torch.tensor([-200.0, -80.0, -20.0, -5.0, 0.0, 5.0, 30.0, 100.0], dtype=torch.float64)
    dev = [up(t) for t in (x, r, i)]
    y, h = kata.recur_fwd(*dev, up(lam), final_state=True)
    want, last = ref.recur(x, r.clamp(min=-1e4), i, lam)
    assert torch.isfinite(y).all()
    err = ref.recur_errors(x, r.clamp(min=-1e4, max=300), i, lam, None, None, 8.0, None, None)
    near(y, want, EPS * want.abs() + err["y"] + 2.0 ** -120, "y")
    grads = kata.recur_bwd(*dev, up(lam), None, None, torch.ones_like(dev[0]))
    assert all(torch.isfinite(g).all() for g in grads if g is not None)
    shut = kata.recur_fwd(dev[0], torch.full_like(dev[1], float("-inf")), dev[2], up(lam), state=torch.ones((1, D), device=DEV))
    assert (shut == 1).all()
    grads = kata.recur_bwd(dev[0], torch.full_like(dev[1], float("-inf")), dev[2], up(lam), None, None, torch.ones_like(dev[0]))
    assert all((g == 0).all() for g in grads if g is not None)


@pytest.mark.parametrize("T,lengths", ((20, [5, 20]), (300, [130, 64])))
def test_recur_extreme_parameters(kata, T, lengths):
    """Parameters at fp32's ends, in padded batches: a rate without bound (the state forgets all),
    biases that hold a gate open or shut, a rate of 0 (the state stays)."""
    big = 3.3e38
    lam = torch.tensor([big, 0.0, 0.0, -big, big], device=DEV)
    rb = torch.tensor([0.0, big, -big, 0.0, -big], device=DEV)
    ib = torch.tensor([0.0, big, 0.0, 0.0, -big], device=DEV)
    x = torch.linspace(-2, 2, 2 * T * 5, device=DEV).view(2, T, 5)
    gate = torch.zeros_like(x)
    h0 = torch.full((2, 5), 0.75, device=DEV)
    ln = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    y = torch.full_like(x, 7.0)
    y, h = kata.recur_fwd(x, gate, gate, lam, rb, ib, state=h0, lengths=ln, y=y, final_state=True)
    there = (torch.arange(T, device=DEV)[None] < ln[:, None])
    assert torch.isfinite(y).all() and torch.isfinite(h).all() and (y[~there] == 7.0).all()
    assert torch.equal(y[..., 0][there], x[..., 0][there] * 0.5)        # take = 1/2, a = 0
    assert (y[..., 2:][there] == 0.75).all() and (h[:, 2:] == 0.75).all()
    grads = kata.recur_bwd(x, gate, gate, lam, rb, ib, torch.ones_like(x), state=h0, lengths=ln)
    assert all(torch.isfinite(g).all() for g in grads)
    for b in range(2):
        one = kata.recur_fwd(x[b:b + 1, :lengths[b]], gate[:1, :lengths[b]], gate[:1, :lengths[b]], lam, rb, ib,
                             state=h0[:1])
        assert torch.equal(one[0], y[b, :lengths[b]])


@pytest.mark.parametrize("lam,r", ((3.3e38, 0.0), (1e30, 3.0), (300.0, 50.0)))
def test_recur_gradients_without_memory(kata, lam, r):
    """Rates at which a = 0: h = sigmoid(i) x, so that dx = dy / 2, di = dy x / 4 and the rest is 0,
    with states far above 1.  Powers of two: nothing is rounded but sigmoid(0) = rcp(2), exact."""
    x = torch.tensor([2.0, -64.0, 1024.0], device=DEV).repeat(2, 70, 1)
    gate, dy = torch.zeros_like(x), torch.full_like(x, 4.0)
    h0 = torch.full((2, 3), 4096.0, device=DEV)
    lam, zeros, dh = torch.full((3,), lam, device=DEV), torch.zeros(3, device=DEV), torch.empty_like(h0)
    dx, dr, di, dlam, drb, dib = kata.recur_bwd(x, torch.full_like(x, r), gate, lam, zeros, zeros, dy, state=h0,
                                                dstate_in=dh)
    assert (dx == 2).all() and torch.equal(di, x) and torch.equal(dib, x.sum((0, 1)))
    for zero in (dr, dlam, drb, dh):
        assert (zero.abs() <= 1e-30).all()


def test_recur_non_finite_stays_ahead(kata):
    x = torch.ones((2, 300, 6), dtype=F32, device=DEV)
    x[0, 140, 2], x[0, 200, 3] = float("inf"), float("nan")
    g = torch.zeros_like(x)
    y = kata.recur_fwd(x, g, g, torch.zeros(6, device=DEV)).cpu()
    bad = torch.zeros((2, 300, 6), dtype=torch.bool)
    bad[0, 140:, 2] = bad[0, 200:, 3] = True
    assert torch.equal(~torch.isfinite(y), bad)


def test_recur_layouts_of_one_projection(kata):
    """x, r, i as parts of one tensor, gradients into the parts of another; time-major rows."""
    gen, x, r, i, lam, rb, ib = recur_inputs(2, 200, 48, BF16, 3)
    par = [up(lam), up(rb), up(ib)]
    flat_in = [up(t, BF16) for t in (x, r, i)]
    rows = torch.cat(flat_in, -1)
    parts = [rows[..., k * 48:(k + 1) * 48] for k in range(3)]
    want = kata.recur_fwd(*flat_in, *par)
    assert torch.equal(kata.recur_fwd(*parts, *par), want)
    dy = up(normal(gen, 2, 200, 48, dtype=BF16), BF16)
    grads = kata.recur_bwd(*flat_in, *par, dy)
    d = torch.empty_like(rows)
    dparts = [d[..., k * 48:(k + 1) * 48] for k in range(3)]
    got = kata.recur_bwd(*parts, *par, dy, dx=dparts[0], dr=dparts[1], di=dparts[2])
    assert torch.equal(torch.cat(grads[:3], -1), d)
    assert all(torch.equal(u, v) for u, v in zip(grads[3:], got[3:]))
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in flat_in]
    y = torch.empty((200, 2, 48), dtype=BF16, device=DEV).transpose(0, 1)
    kata.recur_fwd(*turned, *par, y=y)
    assert torch.equal(y, want)
    with pytest.raises(kata.KataError):
        kata.recur_fwd(*flat_in, *par, y=torch.empty((1, 200, 48), dtype=BF16, device=DEV).expand(2, 200, 48))
    with pytest.raises(kata.KataError):
        kata.recur_fwd(*flat_in, *par, c=0.0)
    with pytest.raises(ValueError):
        kata.recur_fwd(flat_in[0], flat_in[1][:, :100], flat_in[2], *par)


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_recur_many_spans(kata, dtype):
    """A long sequence in many spans, against fp64 by doubling; the same bits each time."""
    B, T, D = 2, 20000, 130
    gen, x, r, i, lam, rb, ib = recur_inputs(B, T, D, dtype, 9)
    dev = [up(t, dtype) for t in (x, r, i)] + [up(lam), up(rb), up(ib)]
    dy = up(normal(gen, B, T, D, dtype=dtype), dtype)
    log(f"case recur long B{B} T{T} D{D} {dtype}")
    ins = [t.double() for t in dev]
    _, a, beta, take, _ = ref.gates(*ins, 8.0)

    def scan(a, b):
        k = 1
        while k < T:
            b = torch.cat([b[:, :k], a[:, k:] * b[:, :-k] + b[:, k:]], 1)
            a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
            k *= 2
        return b
    y, h = kata.recur_fwd(*dev, final_state=True)
    want = scan(a, beta * take * ins[0])
    # roundings of a over the ~1e4 tokens that the slowest channels remember: 2^-24 each
    off = float((y.double() - want).norm() / want.norm())
    assert off <= ref.ROUND[dtype] + 1e-5, off
    off = float((h.double() - want[:, -1]).norm() / want[:, -1].norm())
    assert off <= 1e-5, off
    y2, starts = kata.recur_fwd_train(*dev)
    grads = kata.recur_bwd(*dev, dy, starts)
    G = scan(torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1).flip(1), dy.double().flip(1)).flip(1)
    off = float((grads[0].double() - G * beta * take).norm() / (G * beta * take).norm())
    assert off <= ref.ROUND[dtype] + 1e-5, off
    for _ in range(3):
        again, h2 = kata.recur_fwd(*dev, final_state=True)
        assert torch.equal(again, y) and torch.equal(h2, h)
        assert all(torch.equal(u, v) for u, v in zip(grads, kata.recur_bwd(*dev, dy, starts)))


# ---- streams and graphs ----------------------------------------------------------------------

def _calls(kata):
    """Every entry point as (name, fn, what it updates in place)."""
    gen, x, r, i, lam, rb, ib = recur_inputs(2, 400, 256, BF16, 21)
    x, r, i = (up(t, BF16) for t in (x, r, i))
    par = [up(lam), up(rb), up(ib)]
    dy, dsum = (up(normal(gen, 2, 400, 256, dtype=BF16), BF16) for _ in range(2))
    w, h = up(normal(gen, 256, dtype=F32)), up(normal(gen, 2, 256, dtype=F32))
    ln = torch.tensor([400, 150], dtype=torch.int32, device=DEV)
    a, sa = operand(gen, 800, 2048, 1)
    b, sb = operand(gen, 300, 2048, 128)
    a, sa, b, sb = laid(a, "even"), up(sa), laid(b, "even"), up(sb)
    _, starts = kata.recur_fwd_train(x, r, i, *par)
    y0 = torch.zeros_like(x)
    return [
        ("add_norm_fwd", lambda: kata.add_norm_fwd(x, w, r), []),
        ("add_norm_f8_fwd", lambda: kata.add_norm_f8_fwd(x, w, r), []),
        ("add_norm_bwd", lambda: kata.add_norm_bwd(x, w, dy, dsum), []),
        ("f8_quant", lambda: kata.f8_quant(x, transposed=True), []),
        ("f8_quant blocks", lambda: kata.f8_quant(x, rows=128, transposed=True), []),
        ("f8_gemm", lambda: kata.f8_gemm(a, sa, b, sb), []),
        ("f8_gemm fp32", lambda: kata.f8_gemm(a, sa, b, sb, dtype=F32), []),
        ("f8_gemm few rows", lambda: kata.f8_gemm(a[:9], sa[:9], b, sb), []),
        ("recur_fwd", lambda: kata.recur_fwd(x, r, i, *par, final_state=True), []),
        ("recur_fwd lengths", lambda: kata.recur_fwd(x, r, i, *par, state=h, lengths=ln, y=y0, final_state=True), []),
        ("recur_bwd", lambda: kata.recur_bwd(x, r, i, *par, dy, starts), []),
        ("recur_bwd alone", lambda: kata.recur_bwd(x, r, i, *par, dy, dstate=w.expand(2, 256).contiguous()), []),
        ("recur_step", lambda: kata.recur_step(h, x[:, 0], r[:, 0], i[:, 0], *par), [h]),
    ]


def same(p, q):
    return torch.equal(bits(p), bits(q))


def test_graphs_replay_the_eager_results(kata):
    for name, fn, held in _calls(kata):
        log(f"case graph {name}")
        before = [t.clone() for t in held]
        want = [t.clone() for t in flat(fn())] + [t.clone() for t in held]

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
            assert all(same(u, v) for u, v in zip(flat(out) + held, want)), name
            reset()
            assert all(same(u, v) for u, v in zip(flat(fn()) + held, want)), name  # eager between the replays


def test_two_graphs_share_a_workspace(kata):
    """One after the other on one stream, whatever the other left in it."""
    gen, x, r, i, lam, rb, ib = recur_inputs(2, 700, 96, F32, 5)
    ins = [up(t) for t in (x, r, i)] + [up(lam), up(rb), up(ib)]
    dy = torch.ones_like(ins[0])
    code = kata.KATA_F32
    ws = torch.empty(kata.recur_workspace_bytes(2, 700, 96, code, True), dtype=torch.uint8, device=DEV)
    want_y, want_g = kata.recur_fwd(*ins), kata.recur_bwd(*ins, dy)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        y = kata.recur_fwd(*ins, workspace=ws)
    with torch.cuda.graph(graphs[1]):
        grads = kata.recur_bwd(*ins, dy, workspace=ws)
    for k in range(4):
        ws.fill_((0, 255, 127, 1)[k])
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and all(torch.equal(u, v) for u, v in zip(grads, want_g))


def test_two_streams_at_once(kata):
    calls = [c for c in _calls(kata) if not c[2] and c[0] != "recur_fwd lengths"]
    want = [[t.clone() for t in flat(fn())] for _, fn, _ in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            outs.append([flat(fn()) for _, fn, _ in calls])
    torch.cuda.synchronize()
    for out in outs:
        for (name, _, _), u, v in zip(calls, out, want):
            assert all(same(p, q) for p, q in zip(u, v)), name
    side = torch.cuda.Stream()
    x = torch.randn((50, 64), device=DEV)
    torch.cuda.synchronize()
    q, scale = kata.f8_quant(x, stream=side)
    side.synchronize()
    assert torch.equal(bits(q), bits(kata.f8_quant(x)[0]))


# ---- together ---------------------------------------------------------------------------

def test_layer_training_step(kata):
    """Residual norm in 8 bits -> projection -> convolution and recurrence -> quantiser -> projection
    -> residual norm, and all gradients back, each stage against fp64 on what the stage before
    it gave."""
    B, T, D, W = 2, 150, 192, 256
    M = B * T
    gen = torch.Generator().manual_seed(8)
    x, res = normal(gen, B, T, D, dtype=BF16), normal(gen, B, T, D, dtype=BF16)
    g1, g2 = (1 + normal(gen, D, dtype=F32, std=0.1)).float().double(), torch.ones(D, dtype=torch.float64)
    win, wout = normal(gen, 3 * W, D, dtype=F32, std=D ** -0.5), normal(gen, D, W, dtype=F32, std=W ** -0.5)
    cw, cb = normal(gen, W, 4, dtype=F32, std=0.5), normal(gen, W, dtype=F32, std=0.1)
    lam = (torch.rand(W, generator=gen, dtype=torch.float64) * 4 - 5).float().double()
    w1, s1, w1t, s1t = kata.f8_quant(up(win), rows=128, transposed=True)
    w2, s2, w2t, s2t = kata.f8_quant(up(wout), rows=128, transposed=True)

    def product(a, sa, b, sb, rows, got, what, dtype=BF16):
        a, b = a.float().cpu().reshape(-1, a.shape[-1]), b.float().cpu()
        want, mag, top = ref.product(a, sa.cpu().reshape(a.shape[0], -1), b, sb.cpu(), rows)
        tol = ref.ROUND[dtype] * want.abs() + (288 + ref.blocks(a.shape[1])) * EPS * mag
        if dtype == BF16:
            tol = tol + 7 * 2.0 ** -13 * top
        near(got.reshape(want.shape), want, tol, what)

    a1, as1, total = kata.add_norm_f8_fwd(up(x, BF16), up(g1), up(res, BF16))
    rows = kata.f8_gemm(a1, as1, w1, s1)
    product(a1, as1, w1, s1, 128, rows, "in")
    px, pr, pi = (rows[..., k * W:(k + 1) * W] for k in range(3))
    u = kata.conv_fwd(px, up(cw), up(cb))
    y, starts = kata.recur_fwd_train(u, pr, pi, up(lam))
    ins = [t.cpu().double() for t in (u, pr, pi)]
    want, _ = ref.recur(*ins, lam)
    near(y, want, 2.0 ** -8 * want.abs() + ref.recur_errors(*ins, lam, None, None, 8.0, None, None)["y"], "y")
    a2, as2 = kata.f8_quant(y)
    o = kata.f8_gemm(a2, as2, w2, s2)
    product(a2, as2, w2, s2, 128, o, "out")
    n, total2 = kata.add_norm_fwd(o, up(g2), total)
    assert torch.equal(total2, (o.float() + total.float()).to(BF16))

    # back: the second norm, the projections in 8 bits, the recurrence, the convolution, the first
    dn = up(normal(gen, B, T, D, dtype=BF16), BF16)
    do, dg2 = kata.add_norm_bwd(total2, up(g2), dn)
    dq, dqs, dqt, dqts = kata.f8_quant(do, transposed=True)
    yt = kata.f8_quant(y, transposed=True)[2:]
    dyy = kata.f8_gemm(dq, dqs, w2t, s2t)
    product(dq, dqs, w2t, s2t, 128, dyy, "dy")
    dw2 = kata.f8_gemm(dqt, dqts, *yt, dtype=F32)
    product(dqt, dqts, *yt, 1, dw2, "dw out", F32)
    drows = torch.empty((B, T, 3 * W), dtype=BF16, device=DEV)
    dparts = [drows[..., k * W:(k + 1) * W] for k in range(3)]
    du, _, _, dlam, _, _ = kata.recur_bwd(u, pr, pi, up(lam), None, None, dyy, starts, dr=dparts[1], di=dparts[2])
    kata.conv_bwd(px, up(cw), up(cb), du, dx=dparts[0])
    e, es, et, ets = kata.f8_quant(drows, transposed=True)
    da = kata.f8_gemm(e, es, w1t, s1t)
    product(e, es, w1t, s1t, 128, da, "da")
    at = kata.f8_quant(kata.add_norm_fwd(up(x, BF16), up(g1), up(res, BF16))[0], transposed=True)[2:]
    dw1 = kata.f8_gemm(et, ets, *at, dtype=F32)
    product(et, ets, *at, 1, dw1, "dw in", F32)
    dx, dg1 = kata.add_norm_bwd(total, up(g1), da, do)

    # and as a whole: the codes' roundings (2^-4 of a value, 2.6% rms) in and behind each of four
    # products leave every gradient within 15% of the layer's without them
    leaf = [t.clone().requires_grad_() for t in (x, win, wout, cw, cb, lam, g1)]
    t1 = leaf[0] + res
    p = ref.norm(t1, leaf[6], 1e-6) @ leaf[1].t()
    rows64 = torch.cat([torch.zeros(B, 3, W, dtype=torch.float64), p[..., :W]], 1)
    pre = sum(rows64[:, j:j + T] * leaf[3][:, j] for j in range(4)) + leaf[4]
    z, _ = ref.recur(pre * torch.sigmoid(pre), p[..., W:2 * W], p[..., 2 * W:], leaf[5])
    n64 = ref.norm(z @ leaf[2].t() + t1, g2, 1e-6)
    grads = torch.autograd.grad(n64, (leaf[0], leaf[1], leaf[2], leaf[5], leaf[6]), dn.cpu().double())
    for g, w, name in zip((n, dx, dw1, dw2, dlam, dg1), (n64.detach(), *grads), ("n", "dx", "win", "wout", "lam", "g1")):
        off = float((g.cpu().double() - w).norm() / w.norm())
        log(f"  whole {name}: {off:.2e}")
        assert off <= 0.15, name


def test_layer_decode_continues_the_prompt(kata):
    """A prompt of unequal lengths through norm, 8-bit projection, convolution and recurrence, then
    tokens one by one, against the same over each whole sequence."""
    B, T, more, D = 3, 90, 5, 128
    gen = torch.Generator().manual_seed(9)
    x = up(normal(gen, B, T + more, D, dtype=F32))
    g, lam = up(1 + normal(gen, D, dtype=F32, std=0.1)), up(normal(gen, D, dtype=F32) - 3)
    w8, ws = kata.f8_quant(up(normal(gen, 3 * D, D, dtype=F32, std=D ** -0.5)), rows=128)
    cw = up(normal(gen, D, 4, dtype=F32, std=0.5))

    def project(x):
        a, sa, _ = kata.add_norm_f8_fwd(x, g)
        rows = kata.f8_gemm(a, sa, w8, ws, dtype=F32)
        return [rows[..., k * D:(k + 1) * D] for k in range(3)]
    lengths = torch.tensor([T, 1, 37], dtype=torch.int32, device=DEV)
    px, pr, pi = project(x)
    u, window = kata.conv_fwd(px[:, :T], cw, lengths=lengths, final_state=True)
    _, h = kata.recur_fwd(u, pr[:, :T], pi[:, :T], lam, lengths=lengths, final_state=True)
    each, at, got = torch.arange(B, device=DEV), lengths.long(), []
    for k in range(more):
        qx, qr, qi = project(x[each, at + k])
        got.append(kata.recur_step(h, kata.conv_step(window, qx, cw), qr, qi, lam))
    got = torch.stack(got, 1).cpu().double()
    for b, n in enumerate(lengths.tolist()):
        part = [t[b:b + 1, :n + more] for t in (px, pr, pi)]
        u = kata.conv_fwd(part[0], cw)
        y = kata.recur_fwd(u, part[1], part[2], lam)[:, n:].cpu().double()
        err = ref.recur_errors(*(t.cpu().double() for t in (u, part[1], part[2], lam)), None, None, 8.0, None, None)["y"][:, n:]
        # the projection of one token sums its blocks in another order: 256 fp32 roundings of
        # terms whose sums stay below 16, through gates of slope 1/4 and the state
        near(got[b:b + 1], y, 2 * err + 2.0 ** -8 * EPS ** 0.5, f"sequence {b}")
