"""The mixer operators from their definitions, in fp64 on the CPU, token by token:
the short convolution, the norms with rotation, the selective scan.  Gradients
are autograd's of these definitions (test_mixer_cpu.py holds them against
differences).  The *_mag functions give the sum of the magnitudes of the terms of
each result, which rounding errors are counted against."""
from __future__ import annotations

import torch

EPS32 = 2.0 ** -24                                       # a rounding to fp32, relative
ROUND = {torch.float32: EPS32, torch.bfloat16: 2.0 ** -8}  # a rounding to the output type


def silu(x):
    return x * torch.sigmoid(x)


# ---- short convolution -------------------------------------------------------------

def conv(x, w, bias=None, silu_act=True, state=None, lengths=None):
    """x [B,T,D], w [D,W] -> y (zeros past lengths), the last W-1 rows."""
    B, T, D = x.shape
    W = w.shape[1]
    before = x.new_zeros((B, W - 1, D)) if state is None else state
    rows = torch.cat([before, x], 1)
    pre = sum(rows[:, j:j + T] * w[:, j] for j in range(W))
    if bias is not None:
        pre = pre + bias
    y = silu(pre) if silu_act else pre
    n = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    keep = torch.arange(T)[None] < torch.tensor(n)[:, None]
    last = torch.stack([rows[b, n[b]:n[b] + W - 1] for b in range(B)])
    return y * keep[..., None], last


# ---- norms and rotation -------------------------------------------------------------

def turn(y, pos, freq, pairs):
    """The rotation; y [B,T,H,d], pos [B,T]."""
    r, d = 2 * len(freq), y.shape[-1]
    if r == 0:
        return y
    ang = (pos.double()[..., None] * freq)[:, :, None]
    c, s = torch.cos(ang), torch.sin(ang)
    i = torch.arange(r // 2)
    i0, i1 = (2 * i, 2 * i + 1) if pairs else (i, i + r // 2)
    a, b = y[..., i0], y[..., i1]
    parts = torch.zeros_like(y)
    parts = parts.index_add(-1, i0, a * c - b * s).index_add(-1, i1, a * s + b * c)
    rest = torch.arange(r, d)
    return parts.index_add(-1, rest, y[..., rest])


def turn_mag(y, r, pairs):
    """|a| + |b| for both coordinates of a rotated pair; y >= 0."""
    i = torch.arange(r // 2)
    i0, i1 = (2 * i, 2 * i + 1) if pairs else (i, i + r // 2)
    out = y.clone()
    out[..., i0] = out[..., i1] = y[..., i0] + y[..., i1]
    return out


def norm(x, w, freq, pos, kind, eps, pairs):
    """x [B,T,H,d] -> [B,H,T,d]; kind 0 none, 1 rms, 2 l2."""
    y = x
    if kind:
        ss = x.square().mean(-1, keepdim=True) if kind == 1 else x.square().sum(-1, keepdim=True)
        y = x / torch.sqrt(ss + eps)
    if w is not None:
        y = y * w
    return turn(y, pos, freq, pairs).transpose(1, 2)


# ---- selective scan -------------------------------------------------------------------

def softplus(z):
    return torch.where(z > 40, z, torch.log1p(torch.exp(z.clamp(max=40))))


def scan(x, dt, A, Bm, Cm, D=None, bias=None, soft=True, state=None, lengths=None):
    """x [B,T,H,P], dt [B,T,H], Bm and Cm [B,T,G,N] -> y (zeros past lengths), state [B,H,N,P]."""
    B, T, H, P = x.shape
    per = H // Bm.shape[2]
    z = dt if bias is None else dt + bias
    step = softplus(z) if soft else z
    Bh, Ch = Bm.repeat_interleave(per, 2), Cm.repeat_interleave(per, 2)
    S = x.new_zeros((B, H, Bm.shape[3], P)) if state is None else state
    n = [T] * B if lengths is None else [min(max(int(v), 0), T) for v in lengths]
    ys = []
    for t in range(T):
        live = torch.tensor([t < m for m in n])[:, None, None, None]
        new = (S * torch.exp(step[:, t] * A)[..., None, None]
               + (step[:, t, :, None] * Bh[:, t])[..., None] * x[:, t, :, None])
        S = torch.where(live, new, S)
        y = (Ch[:, t, :, None] @ S)[:, :, 0]
        if D is not None:
            y = y + D[:, None] * x[:, t]
        ys.append(torch.where(live[..., 0], y, torch.zeros_like(y)))
    return torch.stack(ys, 1), S


def scan_mag(x, dt, A, Bm, Cm, D, bias, soft, state, lengths):
    """Sums of magnitudes of y's and the state's terms."""
    z = dt if bias is None else dt + bias
    step = softplus(z) if soft else z
    ab = lambda t: None if t is None else t.abs()  # noqa: E731
    y, S = scan(x.abs(), step.abs(), torch.where(step.mean((0, 1)) < 0, -A, A), Bm.abs(), Cm.abs(),
                ab(D), None, False, ab(state), lengths)
    return y, S


def scan_grads(x, dt, A, Bm, Cm, D, bias, dy, soft=True):
    """Gradients by autograd, in the order x, dt, A, Bm, Cm, D, bias."""
    leaf = [None if t is None else t.clone().requires_grad_() for t in (x, dt, A, Bm, Cm, D, bias)]
    y, _ = scan(*leaf, soft=soft)
    live = [t for t in leaf if t is not None]
    got = iter(torch.autograd.grad(y, live, dy))
    return [None if t is None else next(got) for t in leaf]


def scan_grads_mag(x, dt, A, Bm, Cm, D, bias, dy, soft=True):
    """Sums of magnitudes: the gradients of sum |dy| y for the magnitudes of all inputs, each
    term positive (the decay enters with its own size: a step's direct and decay terms add
    up).  For steps > 0 and A < 0."""
    z = (dt if bias is None else dt + bias).double()
    step = (softplus(z) if soft else z).clone().requires_grad_()
    gate = torch.sigmoid(z) if soft else torch.ones_like(z)
    xa, Ba, Ca = (t.abs().clone().requires_grad_() for t in (x, Bm, Cm))
    log = (step.detach() * A).requires_grad_()  # log a_t, an input of its own
    per = x.shape[2] // Bm.shape[2]
    Bh, Ch = Ba.repeat_interleave(per, 2), Ca.repeat_interleave(per, 2)
    S = x.new_zeros((x.shape[0], x.shape[2], Bm.shape[3], x.shape[3]))
    y = torch.zeros_like(x)
    ys = []
    for t in range(x.shape[1]):
        S = (S * torch.exp(log[:, t])[..., None, None]
             + (step[:, t, :, None] * Bh[:, t])[..., None] * xa[:, t, :, None])
        y = (Ch[:, t, :, None] @ S)[:, :, 0]
        ys.append(y if D is None else y + D.abs()[:, None] * xa[:, t])
    y = torch.stack(ys, 1)
    gx, gs, gl, gB, gC = torch.autograd.grad(y, (xa, step, log, Ba, Ca), dy.abs())
    ddt = (gs + gl * A.abs()) * gate
    return (gx, ddt, (gl * step).sum((0, 1)), gB, gC, (x * dy).abs().sum((0, 1, 3)),
            ddt.sum((0, 1)))
