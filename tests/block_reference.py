"""The operators of a layer in 8 bits from their definitions, in fp64 on the CPU: residual norm,
e4m3 codes with block scales, their product, and the gated linear recurrence, token by token.
Gradients are autograd's of these definitions (test_block_cpu.py holds them against
differences); recur_errors counts the recurrence's roundings along its own terms."""
from __future__ import annotations

import torch

EPS32 = 2.0 ** -24                                       # a rounding to fp32, relative
ROUND = {torch.float32: EPS32, torch.bfloat16: 2.0 ** -8}  # a rounding to the output type
BLOCK = 128


def blocks(n):
    return -(-n // BLOCK)


# ---- residual norm -------------------------------------------------------------------

def norm(s, w, eps):
    y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps)
    return y if w is None else y * w


# ---- e4m3 ------------------------------------------------------------------------------

def to_e4m3(v):
    """fp64 values (magnitudes to 464) to the nearest values of e4m3, ties to even; NaN stays."""
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1].clamp(min=-5) - 4)
    return torch.where(v.isnan(), v, torch.round(v / step) * step)


def quantise(x, rows, bf16=False):
    """x [M,K] fp32 -> (codes' values, scales fp32), as the library defines them: the scale an fp32
    division; codes of fp32 values to nearest of x / scale (fp64: x 448 is exact in it, and a
    quotient of 24 bits by 24 that is no middle itself is further from one than 2^-52 of it), of
    bf16 values (bf16) fp32's reciprocal and product, then to nearest."""
    M, K = x.shape
    mb, kb = -(-M // rows), blocks(K)
    cut = torch.zeros((mb * rows, kb * BLOCK), dtype=torch.float32)
    cut[:M, :K] = x
    cut = cut.view(mb, rows, kb, BLOCK)
    top = cut.abs().nan_to_num(nan=0.0, posinf=float("inf")).amax((1, 3))
    scale = torch.maximum(top / torch.tensor(448.0), torch.tensor(2.0 ** -126))
    if bf16:
        v = (cut * (torch.tensor(1.0) / scale)[:, None, :, None]).double()
    else:
        whole = top.double() / 448 > 2.0 ** -126
        v = torch.where(whole[:, None, :, None], cut.double() * 448 / top.double()[:, None, :, None],
                        cut.double() * 2.0 ** 126)
    return to_e4m3(v).reshape(mb * rows, kb * BLOCK)[:M, :K], scale


def spread(scale, rows, M, K):
    return scale.double().repeat_interleave(rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]


def product(a, sa, b, sb, rows):
    """Codes' values [M,K], [N,K] with their scales -> c, the sum of its terms' magnitudes, and the
    sum over groups of eight products of the largest magnitude (scaled)."""
    A = a.double() * spread(sa, 1, *a.shape)
    B = b.double() * spread(sb, rows, *b.shape)
    pad = -a.shape[1] % 8
    Ag, Bg = (torch.nn.functional.pad(t.abs(), (0, pad)).unflatten(1, (-1, 8)) for t in (A, B))
    top = torch.zeros(A.shape[0], B.shape[0], dtype=torch.float64)
    for g in range(Ag.shape[1]):
        top += (Ag[:, None, g] * Bg[None, :, g]).amax(-1)
    return A @ B.t(), A.abs() @ B.abs().t(), top


# ---- gated linear recurrence ---------------------------------------------------------------

def softplus(z):
    return torch.where(z > 40, z, torch.log1p(torch.exp(z.clamp(max=40))))


def gates(x, r, i, lam, rb, ib, c):
    """rate, a, beta, take, sig."""
    sig = torch.sigmoid(r if rb is None else r + rb)
    take = torch.sigmoid(i if ib is None else i + ib)
    rate = c * softplus(lam) * sig
    a = torch.exp(-rate)
    # for large rates from a itself: expm1's gradient is formed as 1 + its value, which loses a^2
    room = torch.where(rate > 0.5, 1 - a * a, -torch.expm1(-2 * rate))
    return rate, a, torch.sqrt(room), take, sig


def recur(x, r, i, lam, rb=None, ib=None, c=8.0, state=None, lengths=None):
    """x, r, i [B,T,D] -> y (zeros past lengths), the last state [B,D]."""
    B, T, D = x.shape
    _, a, beta, take, _ = gates(x, r, i, lam, rb, ib, c)
    h = x.new_zeros((B, D)) if state is None else state
    n = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    ys = []
    for t in range(T):
        live = torch.tensor([t < m for m in n])[:, None]
        h = torch.where(live, a[:, t] * h + beta[:, t] * take[:, t] * x[:, t], h)
        ys.append(torch.where(live, h, torch.zeros_like(h)))
    return torch.stack(ys, 1), h


def recur_errors(x, r, i, lam, rb, ib, c, state, lengths, dy=None, dstate=None):
    """Bounds of what fp32 roundings add, following the terms.  A rate is off by (12 + |r|)
    2^-24 of itself (sigmoid from exp2 and reciprocal, softplus, three products); so a by that
    times the rate, and four roundings (its own, a product's, what joins runs of tokens); beta
    u by (24 + |r| + |i|) 2^-24.  Returns {"y", "h"} and with dy the gradients' too."""
    B, T, D = x.shape
    rate, a, beta, take, sig = gates(x, r, i, lam, rb, ib, c)
    rz = (r if rb is None else r + rb).abs()
    iz = (i if ib is None else i + ib).abs()
    n = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    live = (torch.arange(T)[None] < torch.tensor(n)[:, None])[..., None]
    off_a = ((12 + rz) * rate + 4) * EPS32
    off_b = (24 + rz + iz) * EPS32
    b = (beta * take * x).abs()
    M = x.new_zeros((B, D)) if state is None else state.abs()
    E = torch.zeros_like(M)
    Ms, Es, before, Eb = [], [], [], []
    for t in range(T):
        before.append(M)
        Eb.append(E)
        new_M = a[:, t] * M + b[:, t]
        new_E = a[:, t] * (E + off_a[:, t] * M) + off_b[:, t] * b[:, t] + EPS32 * new_M
        M, E = (torch.where(live[:, t], u, v) for u, v in ((new_M, M), (new_E, E)))
        Ms.append(M)
        Es.append(E)
    out = {"y": torch.stack(Es, 1) * live, "h": E}
    if dy is None:
        return out
    G = x.new_zeros((B, D)) if dstate is None else dstate.abs()
    EG = torch.zeros_like(G)
    terms = {k: torch.zeros_like(x) for k in ("dx", "dr", "di", "by", "mr", "mi", "mby")}
    u = (take * x).abs()
    ratio = torch.where(beta > 0, rate / beta, torch.zeros_like(rate))
    for t in reversed(range(T)):
        new_G = dy[:, t].abs() + G  # G holds a_{t+1} G_{t+1}
        new_E = EG + EPS32 * new_G
        off = (48 + 2 * rz[:, t] + 2 * iz[:, t]) * EPS32
        inner = rate[:, t] * before[t] + u[:, t] * a[:, t] * ratio[:, t]
        by = new_G * a[:, t] * inner
        e_by = a[:, t] * (new_E * inner + new_G * (rate[:, t] * Eb[t] + (off + off_a[:, t]) * inner))
        du, e_du = new_G * beta[:, t], new_E * beta[:, t] + off * new_G * beta[:, t]
        rest, left = 1 - sig[:, t], 1 - take[:, t]
        for k, v in (("by", e_by), ("dr", e_by * rest), ("dx", e_du * take[:, t]),
                     ("di", e_du * u[:, t] * left), ("mby", by), ("mr", by * rest),
                     ("mi", du * u[:, t] * left)):
            terms[k][:, t] = v * live[:, t]
        G = torch.where(live[:, t], a[:, t] * new_G, G)
        EG = torch.where(live[:, t], a[:, t] * (new_E + off_a[:, t] * new_G), EG)
    per = torch.sigmoid(lam) / softplus(lam)
    # 16 tokens in order, eight waves, then fp64
    out.update({k: terms[k] for k in ("dx", "dr", "di")})
    out["dlam"] = per * ((terms["by"] + 40 * EPS32 * terms["mby"]).sum((0, 1)))
    out["drb"] = (terms["dr"] + 32 * EPS32 * terms["mr"]).sum((0, 1))
    out["dib"] = (terms["di"] + 32 * EPS32 * terms["mi"]).sum((0, 1))
    out["dstate"] = EG + EPS32 * G
    return out
