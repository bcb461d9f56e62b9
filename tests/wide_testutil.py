"""Plain 64-bit forms of the wide layer steps, 8-bit checkpoints and label heads, with
element-by-element error bounds, for the GPU tests.

The bounds follow from the arithmetic alone. U = eps / 2 is half a step of the element type. A
product of K terms accumulated in fp32 is off by at most (K + 2) 2^-23 of the sum of the terms'
magnitudes (a whole step per addition: the matrix instructions may round downwards). The
activations have slopes of at most 1 (their derivatives of at most 5), the hardware's exp2,
reciprocal and the activation formulas are good to EF = 2^-20."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_1812_04352_amd import lp as L

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E32 = 2.0 ** -23
EF = 2.0 ** -20


def half_step(dtype: str) -> float:
    return torch.finfo(DT[dtype]).eps / 2


def tiny(dtype: str) -> float:
    """Half of the smallest step of the type (what a subnormal result may be off)."""
    return torch.finfo(DT[dtype]).smallest_normal * torch.finfo(DT[dtype]).eps / 2


def draw(gen, shape, dtype: str, std: float = 1.0):
    """A CPU tensor of the type."""
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(DT[dtype])


def gpu(t):
    """On the GPU, one element off any wider alignment (a view into a flat vector)."""
    if t is None:
        return None
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    v = flat[1:].view(t.shape)
    v.copy_(t)
    return v


def out(shape, dtype):
    """An output with a value in it that must not survive, and a guard behind it."""
    n = int(np.prod(shape))
    flat = torch.full((n + 65,), 77, dtype=dtype, device="cuda")
    return flat[1:1 + n].view(shape), flat


def guarded(flat, n: int) -> bool:
    return bool((flat[0] == 77).item() and (flat[1 + n:] == 77).all().item())


def sigma(z, act):
    if act == "tanh":
        return torch.tanh(z)
    if act == "relu":
        return z.clamp(min=0)
    if act == "smoothrelu":
        return torch.where(z.abs() <= 0.1, 2.5 * z * z + 0.5 * z + 0.025, z.clamp(min=0))
    return z


def dsigma(z, act):
    if act == "tanh":
        return 1 / torch.cosh(z) ** 2
    if act == "relu":
        return (z > 0).double()
    if act == "smoothrelu":
        return torch.where(z.abs() <= 0.1, 5 * z + 0.5, (z > 0).double())
    return torch.ones_like(z)


def preact(x, W, b):
    """z and its bound."""
    x, W = x.double(), W.double()
    z, mag = x @ W.t(), x.abs() @ W.abs().t()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    return z, (x.shape[1] + 2) * E32 * mag


def forward(x, W, b, r, act, h, dtype):
    z, ez = preact(x, W, b)
    s = h * sigma(z, act)
    y = s if r is None else s + r.double()
    err = abs(h) * (ez + EF) + 2 * E32 * (s.abs() + (0 if r is None else r.double().abs()))
    return y, err + half_step(dtype) * (y.abs() + err) + tiny(dtype)


def backward(x, W, b, dy, act, h, residual, dtype):
    """(dx, dW, db), each with its bound."""
    z, ez = preact(x, W, b)
    x, W, dy = x.double(), W.double(), dy.double()
    u = half_step(dtype)
    g = dsigma(z, act) * dy
    # g before rounding: the slope's own error; a ReLU may decide a site within ez of 0 either way
    slope = {"tanh": ez, "relu": (z.abs() <= ez).double(), "smoothrelu": 5 * ez, "identity": 0 * ez}[act]
    eg32 = dy.abs() * (slope + EF * dsigma(z, act) + E32)
    eg = eg32 + u * (g.abs() + eg32) + tiny(dtype)
    B, no = dy.shape
    dx = h * (g @ W)
    ex = abs(h) * (eg @ W.abs() + (no + 2) * E32 * ((g.abs() + eg) @ W.abs()))
    if residual:
        dx = dx + dy
    ex = ex + 2 * E32 * (dx.abs() + dy.abs().amax())
    dW = h * (g.t() @ x)
    eW = abs(h) * (eg.t() @ x.abs() + (B + 2) * E32 * ((g.abs() + eg).t() @ x.abs())) + 2 * E32 * dW.abs()
    db = h * g.sum(0)
    eb = abs(h) * (eg32.sum(0) + (B + 2) * E32 * (g.abs() + eg32).sum(0)) + 2 * E32 * db.abs()
    return [(v, e + u * (v.abs() + e) + tiny(dtype)) for v, e in ((dx, ex), (dW, eW), (db, eb))]


def loss(u, W, mu, labels, gscale, dtype):
    """J, row, du, dW, dmu, each with its bound (from finite logits)."""
    nc = W.shape[0]
    z, ez = preact(u, W, mu)
    u, W = u.double(), W.double()
    on = (labels >= 0) & (labels < nc)
    n = max(1, int(on.sum()))
    idx = torch.where(on, labels, torch.zeros_like(labels))
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    # the sum of exponentials: every term's exponent (its distance from the maximum, times 2^-23,
    # weighted by its probability) and the additions, at most 64 + 8 in a tile and nc / 2048 + 16 joins
    top = z.amax(1)
    spread = (p * (top[:, None] - z).nan_to_num(posinf=0.0)).sum(1)
    fin = torch.where(torch.isfinite(ez), ez, torch.zeros_like(ez))
    e_lse = fin.amax(1) + (spread + 96 + nc / 2048) * E32 + EF + 2 * E32 * (lse.abs() + top.abs())
    zl = z.gather(1, idx[:, None]).squeeze(1)
    row = torch.where(on, lse - zl, torch.zeros_like(lse))
    e_row = torch.where(on, e_lse + fin.gather(1, idx[:, None]).squeeze(1) + E32 * (lse.abs() + zl.abs()), 0 * lse)
    J, e_J = row.sum() / n, e_row.sum() / n + E32 * row.sum().abs() / n
    P = p.clone()
    P[torch.arange(len(idx)), idx] -= 1
    rel = fin + e_lse[:, None] + (z - lse[:, None]).abs().nan_to_num(posinf=0.0) * E32 + EF
    # a probability below 2^-126, the smallest normal fp32 value, may come out as zero: the hardware's
    # exp2 gives no subnormal results. So may a product of the sums below, which are of such terms.
    small = 2.0 ** -126
    eP32 = p * rel + E32 * P.abs() + small
    eP = eP32 + half_step(dtype) * (P.abs() + eP32) + tiny(dtype) / (16384 if dtype == "f16" else 1)
    for t in (P, eP, eP32):
        t[~on] = 0
    u = torch.where(on[:, None], u, torch.zeros_like(u))  # rows without a label take no part
    f = abs(gscale) / n
    uT = half_step(dtype)

    def done(v, e):
        e = e + 4 * E32 * v.abs() + f * max(n, nc) * small
        return v, e + uT * (v.abs() + e) + tiny(dtype)

    pieces = 8  # an fp32 sum over the pieces of the vocabulary
    du = done(gscale / n * (P @ W), f * (eP @ W.abs() + (nc + 2 + pieces) * E32 * ((P.abs() + eP) @ W.abs())))
    dW = done(gscale / n * (P.t() @ u), f * (eP.t() @ u.abs() + (n + 2) * E32 * ((P.abs() + eP).t() @ u.abs())))
    dmu = done(gscale / n * P.sum(0), f * (eP32.sum(0) + (n + 2) * E32 * (P.abs() + eP32).sum(0)))
    return (J, e_J), (row, e_row), du, dW, dmu


def check(got, ref, bound, what):
    g, r = got.detach().double().cpu(), ref.double().cpu()
    bound = bound.double().cpu() if torch.is_tensor(bound) else bound
    assert g.shape == r.shape, (what, g.shape, r.shape)
    over = ~((g - r).abs() <= bound)
    if bool(over.any()):
        worst = ((g - r).abs() / bound).nan_to_num(nan=math.inf).flatten().argmax()
        raise AssertionError(f"{what}: {int(over.sum())} of {over.numel()} beyond their bound, worst at {int(worst)}: "
                             f"{g.flatten()[worst]} for {r.flatten()[worst]}")


def pack(x):
    """The checkpoint of CPU rows x by its definition, value by value in Python's exact arithmetic."""
    emin = -24 if x.dtype == torch.float16 else -126
    B, q = x.shape
    nb = -(-q // 32)
    x8, xe = np.zeros((B, q), np.int8), np.zeros((B, nb), np.uint8)
    v = x.double().numpy()
    for k in range(B):
        for j in range(nb):
            blk = v[k, 32 * j:32 * (j + 1)]
            if not np.all(np.isfinite(blk)):
                xe[k, j] = 255
                continue
            m = float(np.max(np.abs(blk)))
            e = max(emin, math.frexp(m)[1] - 1 - 6) if m > 0 else emin
            xe[k, j] = e + 127
            x8[k, 32 * j:32 * j + len(blk)] = [max(-127, min(127, round(math.ldexp(float(t), -e)))) for t in blk]
    return torch.from_numpy(x8), torch.from_numpy(xe)


def unpack(x8, xe):
    q = x8.shape[1]
    s = torch.ldexp(torch.ones(xe.shape, dtype=torch.float64), xe.long() - 127)
    s[xe == 255] = math.nan
    return x8.double() * s.repeat_interleave(32, 1)[:, :q]


class Step:
    """One step's calls on GPU copies of CPU inputs, outputs guarded."""

    def __init__(self, dtype, act, B, ni, no, h):
        self.dtype, self.st = dtype, L.step(dtype, act, B, ni, no, h)
        self.B, self.ni, self.no = B, ni, no
        self.ws = L.alloc_step_workspace(self.st)

    def forward(self, x, W, b, r, ck=False):
        y, yf = out((self.B, self.no), DT[self.dtype])
        nb = -(-self.no // 32)
        y8, y8f = out((self.B, self.no), torch.int8)
        ye, yef = out((self.B, nb), torch.uint8)
        L.lp_step_forward(self.st, x, W, b, r, y, self.ws, *((y8, ye) if ck else ()))
        torch.cuda.synchronize()
        assert guarded(yf, y.numel()) and guarded(y8f, y8.numel()) and guarded(yef, ye.numel())
        return (y, y8, ye) if ck else y

    def backward(self, x, W, b, dy, residual, want=(True, True, True)):
        shapes = ((self.B, self.ni), (self.no, self.ni), (self.no,))
        bufs = [out(s, DT[self.dtype]) if w else (None, None) for s, w in zip(shapes, want)]
        L.lp_step_backward(self.st, x, W, b, dy, *[v for v, _ in bufs], self.ws, residual=residual)
        torch.cuda.synchronize()
        for v, f in bufs:
            assert v is None or guarded(f, v.numel())
        return [v for v, _ in bufs]
