"""Timed cases of the operators of a mixer's layer in 8 bits: the root-mean-square norm
with the residual's addition (its output in the activations' type or in e4m3 with a scale
for each 128 columns), the quantiser to e4m3 with block scales, the matrix product of such
operands, and the gated linear recurrence, each in the directions and forms that a program
calls.

    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU, from the seed alone
    run(state)          one pass: plain torch operations, or the library's entry points
    work(case)          bytes and operations that one pass cannot do without
    exact(case, seed)   the outputs of run() in 64 bits, from the definitions

Where `own` is false, run() computes in 32 bits (long sums of gradients in 64) and rounds
each output once.  Codes of 8 bits are returned as float8 tensors: as their values.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
C = 8.0       # the recurrence's decay exponent
BLOCK = 128   # columns (and rows) of a scale
TOP = 448.0   # e4m3's largest value
LOW = 2.0 ** -126
F8 = torch.float8_e4m3fn


def _api():
    import paper_2607_17419_amd as kata
    return kata


# ---- cases ----------------------------------------------------------------------

def _norm(kind, M, D, dtype):
    return {"op": "norm", "kind": kind, "M": M, "D": D, "dtype": dtype}


def _quant(M, K, rows, dtype):
    return {"op": "quant", "kind": "quant", "M": M, "K": K, "rows": rows, "dtype": dtype}


def _gemm(M, N, K, rows, out):
    return {"op": "gemm", "kind": "gemm", "M": M, "N": N, "K": K, "rows": rows, "dtype": out}


def _recur(kind, B, T, D, dtype, lens=False):
    return {"op": "recur", "kind": kind, "B": B, "T": T, "D": D, "dtype": dtype, "lens": lens}


def listed():
    named = {
        # one token for each of 256 sequences in serving, before an 8-bit projection
        "norm_step": _norm("f8", 256, 1024, "bf16"),
        # the norm of a training step of 8 sequences of 4096 tokens, forward and gradients
        "norm_train": _norm("train", 32768, 1024, "bf16"),
        # a master weight in 32 bits to the 128 x 128 blocks of forward and gradient products
        "quant_weight": _quant(4096, 1024, 128, "f32"),
        # a training step's activations, as rows and transposed for the weight's gradient
        "quant_train": _quant(32768, 1024, 1, "bf16"),
        # eight sequences' tokens in serving: the weight is read once
        "gemm_step": _gemm(8, 8192, 4096, 128, "bf16"),
        # a prompt of odd length, a width that fills no block
        "gemm_prompt": _gemm(1999, 1152, 1000, 128, "bf16"),
        # a large projection
        "gemm_large": _gemm(8192, 8192, 8192, 128, "bf16"),
        # a weight's gradient over 32768 tokens, in 32 bits
        "gemm_weight_grad": _gemm(1152, 1024, 32768, 1, "f32"),
        # one token for each of 256 sequences
        "recur_step": _recur("step", 256, 1, 1024, "bf16"),
        # four prompts of unequal length in one padded batch, states kept for decoding
        "recur_prompt": _recur("fwd", 4, 2000, 1152, "bf16", lens=True),
        # one long sequence
        "recur_long": _recur("fwd", 1, 131072, 1024, "bf16"),
        # one layer's training step, forward and gradients
        "recur_train": _recur("train", 8, 4096, 1024, "bf16"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Half of them whole blocks of 64, the others as they come."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(("norm", "quant", "gemm", "gemm", "recur", "recur"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        D = _width(rng, 64, 8192)
        return _norm(rng.choice(("f8", "plain", "train")), _log_int(rng, 1, 33000000 // D), D, dtype)
    if op == "quant":
        K = _width(rng, 64, 8192)
        rows = rng.choice((1, 128))
        return _quant(_log_int(rng, 1 if rows == 1 else 64, 33000000 // K), K, rows, dtype)
    if op == "gemm":
        if rng.random() < 0.3:
            return _gemm(_width(rng, 64, 2048), _width(rng, 64, 2048), _log_int(rng, 256, 32768),
                         1, "f32")
        return _gemm(_log_int(rng, 1, 8192), _width(rng, 64, 8192), _width(rng, 64, 8192), 128,
                     dtype)
    kind = rng.choice(("step", "fwd", "train"))
    D = _width(rng, 64, 4096)
    if kind == "step":
        return _recur(kind, _log_int(rng, 1, 512), 1, D, dtype)
    n = (130 if kind == "fwd" else 33) * 10 ** 6 // (1 if dtype == "bf16" else 2)
    T = min(_log_int(rng, 2, 131072 if kind == "fwd" else 8192), n // D)
    B = max(1, min(_log_int(rng, 1, 8), n // (D * T)))
    return _recur(kind, B, T, D, dtype, lens=kind == "fwd" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------

def _blocks(n):
    return -(-n // BLOCK)


def _codes(x, rows):
    """x [M, K] in fp32 as codes and scales of blocks of rows x 128, in plain operations."""
    M, K = x.shape
    mb, kb = -(-M // rows), _blocks(K)
    padded = torch.nn.functional.pad(x, (0, kb * BLOCK - K, 0, mb * rows - M))
    cut = padded.view(mb, rows, kb, BLOCK)
    scale = (cut.abs().amax((1, 3)) / TOP).clamp(min=LOW)
    q = (cut * (1 / scale)[:, None, :, None]).clamp(-TOP, TOP).to(F8)
    return q.view(mb * rows, kb * BLOCK)[:M, :K], scale


def _values(q, scale, rows):
    """The fp32 values of codes [M, K] with scales of blocks of rows x 128."""
    M, K = q.shape
    wide = scale.repeat_interleave(rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]
    return q.float() * wide


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=DEV) * std

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=gen, device=DEV) * (hi - lo) + lo

    s = {"case": {k: v for k, v in case.items() if k != "name"}, "dtype": dtype}
    if case["op"] == "norm":
        M, D = case["M"], case["D"]
        s["x"], s["res"] = normal(M, D).to(dtype), normal(M, D, std=2.0).to(dtype)
        s["w"] = 1 + normal(D, std=0.1)
        if case["kind"] == "train":
            s["dy"], s["dsum"] = (normal(M, D, std=0.1).to(dtype) for _ in range(2))
        return s
    if case["op"] == "quant":
        M, K = case["M"], case["K"]
        # rows of different size, as activations and gradients have them
        s["x"] = (normal(M, K) * torch.exp(normal(M, 1))).to(dtype)
        return s
    if case["op"] == "gemm":
        M, N, K, rows = (case[k] for k in ("M", "N", "K", "rows"))

        def operand(n, rows, std):
            # rows start at multiples of 16 bytes, as the quantisers lay them out
            q, scale = _codes(normal(n, K, std=std) * torch.exp(0.5 * normal(n, 1)), rows)
            wide = torch.zeros((n, -(-K // 16) * 16), dtype=torch.uint8, device=DEV)
            wide[:, :K] = q.view(torch.uint8)
            return wide.view(F8)[:, :K], scale

        s["a"], s["sa"] = operand(M, 1, 1.0)
        s["b"], s["sb"] = operand(N, rows, 1 / math.sqrt(K))
        return s
    B, T, D = case["B"], case["T"], case["D"]
    lead = (B,) if case["kind"] == "step" else (B, T)
    wide = normal(*lead, 3 * D).to(dtype)  # one projection's output: x and both gates
    s["x"], s["r"], s["i"] = wide[..., :D], wide[..., D:2 * D], wide[..., 2 * D:]
    # decays of 0.9 to 0.999 a token where the gate is fully open
    decay = -torch.log(uniform(0.9, 0.999, D)) / C
    s["lam"] = torch.log(torch.expm1(decay))
    s["rb"], s["ib"] = normal(D, std=0.1), normal(D, std=0.1)
    if case["kind"] == "step" or case["lens"]:
        s["h"] = normal(B, D)
    if case["lens"]:
        # lengths of a padded batch: the longest fills it, none is shorter than one token
        n = (uniform(0.2, 1.0, B) * T).long().clamp(1, T)
        n[0] = T
        s["lengths"] = n.int()
        s["y"] = torch.zeros((B, T, D), dtype=dtype, device=DEV)
    if case["kind"] == "train":
        s["dy"] = normal(B, T, D, std=0.1).to(dtype)
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    how = {"norm": _run_norm, "quant": _run_quant, "gemm": _run_gemm, "recur": _run_recur}
    return how[s["case"]["op"]](s, s["case"]["kind"])


def _run_norm(s, kind):
    x, res, w = s["x"], s["res"], s["w"]
    if own:
        kata = _api()
        if kind == "f8":
            q, scale, total = kata.add_norm_f8_fwd(x, w, res, eps=EPS)
            return {"q": q, "scale": scale, "sum": total}
        y, total = kata.add_norm_fwd(x, w, res, eps=EPS)
        if kind == "plain":
            return {"y": y, "sum": total}
        dx, dw = kata.add_norm_bwd(total, w, s["dy"], s["dsum"], eps=EPS)
        return {"y": y, "sum": total, "dx": dx, "dw": dw}
    total = (x.float() + res.float()).to(x.dtype)
    t32 = total.float()
    inv = 1 / torch.sqrt((t32 * t32).mean(-1, keepdim=True) + EPS)
    hat = t32 * inv
    y = hat * w
    if kind == "f8":
        q, scale = _codes(y, 1)
        return {"q": q, "scale": scale, "sum": total}
    if kind == "plain":
        return {"y": y.to(x.dtype), "sum": total}
    dy = s["dy"].float()
    g = dy * w
    dx = s["dsum"].float() + inv * (g - hat * (g * hat).mean(-1, keepdim=True))
    dw = (dy * hat).sum(0, dtype=torch.float64).float()
    return {"y": y.to(x.dtype), "sum": total, "dx": dx.to(x.dtype), "dw": dw}


def _run_quant(s, kind):
    x, rows = s["x"], s["case"]["rows"]
    if own:
        q, scale, qt, scale_t = _api().f8_quant(x, rows=rows, transposed=True)
        return {"q": q, "scale": scale, "qt": qt, "scale_t": scale_t}
    x32 = x.float()
    q, scale = _codes(x32, rows)
    qt, scale_t = _codes(x32.t(), rows)
    return {"q": q, "scale": scale, "qt": qt, "scale_t": scale_t}


def _run_gemm(s, kind):
    if own:
        return {"c": _api().f8_gemm(s["a"], s["sa"], s["b"], s["sb"], dtype=s["dtype"])}
    a, b = _values(s["a"], s["sa"], 1), _values(s["b"], s["sb"], s["case"]["rows"])
    return {"c": torch.matmul(a, b.t()).to(s["dtype"])}


def _sigmoid(z):
    return 1 / (1 + torch.exp(-z))


def _softplus(z):
    return torch.where(z > 20, z, torch.log1p(torch.exp(z.clamp(max=20))))


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, by doubling."""
    step = 1
    while step < a.shape[1]:
        b = torch.cat([b[:, :step], a[:, step:] * b[:, :-step] + b[:, step:]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _run_recur(s, kind):
    x, r, i, lam, rb, ib = (s[k] for k in ("x", "r", "i", "lam", "rb", "ib"))
    if own:
        kata = _api()
        if kind == "step":
            return {"y": kata.recur_step(s["h"], x, r, i, lam, rb, ib, c=C), "h": s["h"]}
        if kind == "train":
            y, starts = kata.recur_fwd_train(x, r, i, lam, rb, ib, c=C)
            grads = kata.recur_bwd(x, r, i, lam, rb, ib, s["dy"], starts, c=C)
            return {"y": y, **dict(zip(("dx", "dr", "di", "dlam", "drb", "dib"), grads))}
        if s["case"]["lens"]:
            y, h = kata.recur_fwd(x, r, i, lam, rb, ib, c=C, state=s["h"], lengths=s["lengths"],
                                  y=s["y"], final_state=True)
            return {"y": y, "h": h}
        return {"y": kata.recur_fwd(x, r, i, lam, rb, ib, c=C)}
    x32 = x.float()
    soft = _softplus(lam)
    gate, take = _sigmoid(r.float() + rb), _sigmoid(i.float() + ib)
    rate = C * soft * gate
    a, room = torch.exp(-rate), -torch.expm1(-2 * rate)
    beta, u = torch.sqrt(room), take * x32
    if kind == "step":
        s["h"].mul_(a).add_(beta * u)
        return {"y": s["h"].to(x.dtype), "h": s["h"]}
    b = beta * u
    if s["case"]["lens"]:
        n = s["lengths"].long()
        there = (torch.arange(x.shape[1], device=DEV) < n[:, None])[..., None]
        first = torch.cat([a[:, :1] * s["h"][:, None] + b[:, :1], b[:, 1:]], 1)
        h = _scan(a, first)
        last = torch.take_along_dim(h, (n - 1)[:, None, None], 1)[:, 0]
        return {"y": torch.where(there, h.to(x.dtype), s["y"]), "h": last}
    h = _scan(a, b)
    if kind == "fwd":
        return {"y": h.to(x.dtype)}
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    G = _scan(after.flip(1), s["dy"].float().flip(1)).flip(1)
    dlog = G * (a * before - u * a * a / beta)
    by_rate = rate * dlog
    dr, du = by_rate * (gate - 1), G * beta
    di = du * u * (1 - take)
    # d softplus(lam) / softplus(lam)
    dlam = -(by_rate.sum((0, 1), dtype=torch.float64) * (_sigmoid(lam) / soft)).float()
    return {"y": h.to(x.dtype), "dx": (du * take).to(x.dtype), "dr": dr.to(x.dtype),
            "di": di.to(x.dtype), "dlam": dlam,
            "drb": dr.sum((0, 1), dtype=torch.float64).float(),
            "dib": di.sum((0, 1), dtype=torch.float64).float()}


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if case["op"] == "norm":
        M, D = case["M"], case["D"]
        n = M * D
        if kind == "train":  # x, res and sum, y; dy, dsum and dx (the sum is at hand)
            return {"bytes": 7 * n * e + 8 * D, "flops": 18 * n}
        out = n + 4 * M * _blocks(D) if kind == "f8" else n * e
        return {"bytes": 3 * n * e + out + 4 * D, "flops": 6 * n}
    if case["op"] == "quant":
        M, K, rows = case["M"], case["K"], case["rows"]
        scales = -(-M // rows) * _blocks(K) + -(-K // rows) * _blocks(M)
        return {"bytes": M * K * (e + 2) + 4 * scales, "flops": 4 * M * K}
    if case["op"] == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        scales = (M + -(-N // case["rows"])) * _blocks(K)
        return {"bytes": (M + N) * K + 4 * scales + M * N * e, "flops": 2 * M * N * K}
    B, T, D = case["B"], case["T"], case["D"]
    n, state = B * T * D, 4 * B * D
    if kind == "step":
        return {"bytes": 4 * n * e + 2 * state + 12 * D, "flops": 30 * n}
    if kind == "train":  # x and both gates read once for both directions
        return {"bytes": 8 * n * e + 24 * D, "flops": 90 * n}
    return {"bytes": 4 * n * e + (2 * state if case["lens"] else 0) + 12 * D, "flops": 30 * n}


# ---- the definitions in 64 bits -----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    how = {"norm": _exact_norm, "quant": _exact_quant, "gemm": _exact_gemm,
           "recur": _exact_recur}
    return how[case["op"]](s, case["kind"])


def _exact_codes(x, rows):
    """Codes' values and scales, one column block after the other, in 64 bits."""
    M, K = x.shape
    q, scales = torch.empty_like(x), []
    for k in range(0, K, BLOCK):
        part = x[:, k:k + BLOCK]
        top = part.abs().amax(1)
        if rows > 1:
            top = torch.stack([t.amax() for t in top.split(rows)])
        scale = torch.clamp(top / TOP, min=LOW)
        v = part / scale.repeat_interleave(rows)[:M, None]
        # a value of 2^(e-1) .. 2^e has steps of 2^(e-4), down to 2^-9
        step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1].clamp(min=-5) - 4)
        q[:, k:k + BLOCK] = (torch.round(v / step) * step).clamp(-TOP, TOP)
        scales.append(scale)
    return q, torch.stack(scales, 1)


def _exact_norm(s, kind):
    w = s["w"].double()
    whole = s["x"].double() + s["res"].double()
    t = (s["x"].float() + s["res"].float()).to(s["dtype"]).double()  # the norm's input
    if kind == "train":
        t.requires_grad_()
        w.requires_grad_()
    y = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w
    if kind == "f8":
        q, scale = _exact_codes(y, 1)
        return {"q": q, "scale": scale, "sum": whole}
    if kind == "plain":
        return {"y": y, "sum": whole}
    dt, dw = torch.autograd.grad(y, (t, w), s["dy"].double())
    return {"y": y.detach(), "sum": whole, "dx": dt + s["dsum"].double(), "dw": dw}


def _exact_quant(s, kind):
    x, rows = s["x"].double(), s["case"]["rows"]
    q, scale = _exact_codes(x, rows)
    qt, scale_t = _exact_codes(x.t().contiguous(), rows)
    return {"q": q, "scale": scale, "qt": qt, "scale_t": scale_t}


def _exact_gemm(s, kind):
    rows, K = s["case"]["rows"], s["case"]["K"]
    c = torch.zeros((s["a"].shape[0], s["b"].shape[0]), dtype=torch.float64, device=DEV)
    for kb in range(_blocks(K)):
        at = slice(kb * BLOCK, min(K, (kb + 1) * BLOCK))
        a, b = (t[:, at].float().double() for t in (s["a"], s["b"]))
        sb = s["sb"][:, kb].double().repeat_interleave(rows)[:b.shape[0]]
        c.addmm_(a * s["sa"][:, kb, None].double(), (b * sb[:, None]).t())
    return {"c": c}


def _exact_recur(s, kind):
    x, r, i, lam, rb, ib = (s[k].double() for k in ("x", "r", "i", "lam", "rb", "ib"))
    if kind == "step":
        x, r, i = x[:, None], r[:, None], i[:, None]
    B, T, D = x.shape
    soft = torch.where(lam > 40, lam, torch.log1p(torch.exp(lam.clamp(max=40))))
    rate = torch.sigmoid(r + rb) * (C * soft)
    take = torch.sigmoid(i + ib)
    a, beta = torch.exp(-rate), torch.sqrt(-torch.expm1(-2 * rate))
    b = beta * take * x
    h = s["h"].double() if "h" in s else x.new_zeros((B, D))
    start = h
    y = torch.empty_like(x)
    for t in range(T):
        h = torch.addcmul(b[:, t], a[:, t], h)
        y[:, t] = h
    if kind == "step":
        return {"y": y[:, 0], "h": h}
    if kind == "fwd":
        if not s["case"]["lens"]:
            return {"y": y}
        n = s["lengths"].tolist()
        last = torch.stack([y[k, n[k] - 1] for k in range(B)])
        for k in range(B):
            y[k, n[k]:] = 0
        return {"y": y, "h": last}
    # the adjoint recurrence, token by token; G is the gradient of h_t
    G, dy = torch.zeros_like(h), s["dy"].double()
    dx, dr, di = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dlam = torch.zeros_like(lam)
    for t in reversed(range(T)):
        G = G + dy[:, t]
        before = y[:, t - 1] if t else start
        at, bt, st, it = a[:, t], beta[:, t], rate[:, t], take[:, t]
        by_rate = -st * G * (at * before - it * x[:, t] * at * at / bt)
        dr[:, t] = by_rate * (1 - st / (C * soft))
        dlam += by_rate.sum(0)
        dx[:, t] = G * bt * it
        di[:, t] = G * bt * x[:, t] * it * (1 - it)
        G = G * at
    dlam *= torch.sigmoid(lam) / soft
    return {"y": y, "dx": dx, "dr": dr, "di": di, "dlam": dlam, "drb": dr.sum((0, 1)),
            "dib": di.sum((0, 1))}
