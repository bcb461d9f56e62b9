"""Plain 64-bit forms of the layer norm, the gated layers and the orthogonalised update, with
element-by-element error bounds, for the GPU tests.

The bounds follow from the arithmetic alone, as in wide_testutil: half a step of the element type for each
rounding to it, a whole step of fp32 per addition of a sum, EF = 2^-20 for the activation formulas."""
from __future__ import annotations

import math

import torch

import wide_testutil as T
from paper_1812_04352_amd import lp as L

E32, EF = T.E32, T.EF
ACTS = ("tanh", "relu", "smoothrelu", "identity", "silu", "gelu")
# the largest second derivative of each activation (that of relu jumps, see slope_error)
BEND = {"tanh": 0.77, "smoothrelu": 5.0, "identity": 0.0, "silu": 0.5, "gelu": 0.8}


def gate(z, act):
    """The activation and its slope."""
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t + z * t * torch.sigmoid(-z)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z * math.sqrt(0.5))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return T.sigma(z, act), T.dsigma(z, act)


def gate_error(z, ez, act):
    """What the activation and its slope may be off for a z that is off by ez: slopes of 1.2 at most; the
    formulas' relative error grows with |z|, the exponent's size (by 1 / 8 of EF)."""
    s, ds = gate(z, act)
    grow = EF * (1 + z.abs() / 8)
    slope = (z.abs() <= ez).double() if act == "relu" else BEND[act] * ez
    return 1.2 * ez + grow * (s.abs() + (1.0 if act in ("tanh", "smoothrelu") else 0.0)), slope + grow * (1 + ds.abs())


def gated_forward(x, Wg, Wu, act, dtype):
    zg, eg = T.preact(x, Wg, None)
    zu, eu = T.preact(x, Wu, None)
    s, _ = gate(zg, act)
    es, _ = gate_error(zg, eg, act)
    y = s * zu
    err = s.abs() * eu + (zu.abs() + eu) * es + 2 * E32 * y.abs()
    return y, err + T.half_step(dtype) * (y.abs() + err) + T.tiny(dtype)


def gated_backward(x, Wg, Wu, dy, act, dtype):
    """(dx, dWg, dWu), each with its bound."""
    zg, eg = T.preact(x, Wg, None)
    zu, eu = T.preact(x, Wu, None)
    x, Wg, Wu, dy = x.double(), Wg.double(), Wu.double(), dy.double()
    s, ds = gate(zg, act)
    es, eds = gate_error(zg, eg, act)
    u, tiny = T.half_step(dtype), T.tiny(dtype)
    dzu, dzg = dy * s, dy * zu * ds
    eu32 = dy.abs() * es + 2 * E32 * dzu.abs()
    eg32 = dy.abs() * (zu.abs() * eds + (ds.abs() + eds) * eu) + 4 * E32 * dzg.abs()
    ezu = eu32 + u * (dzu.abs() + eu32) + tiny
    ezg = eg32 + u * (dzg.abs() + eg32) + tiny
    B, no = dy.shape
    dx = dzg @ Wg + dzu @ Wu
    ex = ezg @ Wg.abs() + ezu @ Wu.abs() + (2 * no + 66) * E32 * ((dzg.abs() + ezg) @ Wg.abs() + (dzu.abs() + ezu) @ Wu.abs())
    out = [(dx, ex)]
    for d, e in ((dzg, ezg), (dzu, ezu)):
        out.append((d.t() @ x, e.t() @ x.abs() + (B + 2) * E32 * ((d.abs() + e).t() @ x.abs())))
    return [(v, e + u * (v.abs() + e) + tiny) for v, e in out]


def norm_stats(x, eps):
    """xh, 1 / sqrt(var + eps) and their bounds. A thread adds at most 64 values of a row that its group holds (a
    1024th of a longer one), and 16 exchanges follow."""
    x = x.double()
    q = x.shape[1]
    n = 84 + q / 1024
    mean = x.mean(1, keepdim=True)
    d = x - mean
    ed = n * E32 * x.abs().mean(1, keepdim=True) + E32 * d.abs()
    var = (d * d).mean(1, keepdim=True)
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + n * E32 * var
    rstd = (var + eps) ** -0.5
    er = rstd * (0.5 * ev / (var + eps) + 4 * E32)
    xh = d * rstd
    return xh, (ed * (rstd + er) + d.abs() * er + E32 * xh.abs()), rstd, er, n


def norm_forward(x, gamma, beta, eps, dtype):
    xh, exh, *_ = norm_stats(x, eps)
    ga = 1.0 if gamma is None else gamma.double()
    y = xh * ga + (0.0 if beta is None else beta.double())
    err = exh * (ga if gamma is None else ga.abs()) + 2 * E32 * ((xh * ga).abs() + y.abs())
    return y, err + T.half_step(dtype) * (y.abs() + err) + T.tiny(dtype)


def norm_backward(x, gamma, dy, dr, eps, dtype):
    """(dx, dgamma, dbeta), each with its bound."""
    xh, exh, rstd, er, n = norm_stats(x, eps)
    dy = dy.double()
    g = dy if gamma is None else dy * gamma.double()
    B = x.shape[0]
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    e1 = n * E32 * g.abs().mean(1, keepdim=True)
    e2 = (g.abs() * exh).mean(1, keepdim=True) + (n + 3) * E32 * (g * xh).abs().mean(1, keepdim=True)
    inner = g - m1 - xh * m2
    ei = e1 + exh * m2.abs() + (xh.abs() + exh) * e2 + 3 * E32 * (g.abs() + m1.abs() + (xh * m2).abs())
    dx = rstd * inner
    ex = (rstd + er) * ei + er * inner.abs() + E32 * dx.abs()
    if dr is not None:
        dx = dx + dr.double()
        ex = ex + E32 * (dx.abs() + dr.double().abs())
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    eg = (dy.abs() * exh).sum(0) + (B + 4) * E32 * (dy * xh).abs().sum(0)
    eb = (B + 4) * E32 * dy.abs().sum(0)
    u = T.half_step(dtype)
    return [(v, e + u * (v.abs() + e) + T.tiny(dtype)) for v, e in ((dx, ex), (dgamma, eg), (dbeta, eb))]


def scribble(ws):
    """A workspace that holds NaN in every type."""
    ws.fill_(255)
    return ws


class Gated:
    """One layer's calls, outputs guarded, from a workspace full of NaN."""

    def __init__(self, dtype, act, B, ni, no):
        self.dtype, self.gd = dtype, L.gated(dtype, act, B, ni, no)
        self.B, self.ni, self.no = B, ni, no

    def forward(self, x, Wg, Wu):
        ws = scribble(L.alloc_gated_workspace(self.gd, grad=False))
        y, yf = T.out((self.B, self.no), T.DT[self.dtype])
        L.lp_gated_forward(self.gd, x, Wg, Wu, y, ws)
        torch.cuda.synchronize()
        assert T.guarded(yf, y.numel())
        return y

    def backward(self, x, Wg, Wu, dy, want=(True, True, True)):
        ws = scribble(L.alloc_gated_workspace(self.gd, grad=True))
        shapes = ((self.B, self.ni), (self.no, self.ni), (self.no, self.ni))
        bufs = [T.out(s, T.DT[self.dtype]) if w else (None, None) for s, w in zip(shapes, want)]
        L.lp_gated_backward(self.gd, x, Wg, Wu, dy, *[v for v, _ in bufs], ws)
        torch.cuda.synchronize()
        for v, f in bufs:
            assert v is None or T.guarded(f, v.numel())
        return [v for v, _ in bufs]


class Norm:
    """One norm's calls, outputs guarded, from a workspace full of NaN."""

    def __init__(self, dtype, B, q, eps=1e-5):
        self.dtype, self.nd = dtype, L.norm(dtype, B, q, eps)
        self.B, self.q = B, q

    def forward(self, x, gamma, beta):
        y, yf = T.out((self.B, self.q), T.DT[self.dtype])
        L.lp_norm_forward(self.nd, x, gamma, beta, y)
        torch.cuda.synchronize()
        assert T.guarded(yf, y.numel())
        return y

    def backward(self, x, gamma, dy, dr, want=(True, True, True)):
        ws = scribble(L.alloc_norm_workspace(self.nd))
        shapes = ((self.B, self.q), (self.q,), (self.q,))
        bufs = [T.out(s, T.DT[self.dtype]) if w else (None, None) for s, w in zip(shapes, want)]
        L.lp_norm_backward(self.nd, x, gamma, dy, dr, *[v for v, _ in bufs], ws)
        torch.cuda.synchronize()
        for v, f in bufs:
            assert v is None or T.guarded(f, v.numel())
        return [v for v, _ in bufs]


def momentum(g, m, mu, nesterov, dtype):
    """m' and v, with the error of m' (two fp32 roundings)."""
    g = g.double()
    if m is None and mu is None:
        return None, g
    mo = g if m is None else mu * m.double() + g
    return mo, (g + mu * mo if nesterov else mo)


def iterate(v, steps, coeffs, eps, keep=None):
    """The iteration on a batch of matrices; keep: a rounding made where the kernels make one."""
    a, b, c = coeffs
    keep = keep or (lambda t: t)
    X = keep(v / (torch.linalg.vector_norm(v, dim=(1, 2), keepdim=True) + eps))
    tall = v.shape[1] > v.shape[2]
    X = X.transpose(1, 2).contiguous() if tall else X
    for s in range(steps):
        A = keep(torch.matmul(X, X.transpose(1, 2).contiguous()))
        P = keep(b * A + c * torch.matmul(A, A))
        X = a * X + torch.matmul(P, X)
        if s + 1 < steps:
            X = keep(X)
    return X.transpose(1, 2) if tall else X


def rounding(dtype, shape, seed=0):
    """What the products' operands are rounded to: f16 of values times about the root of the long side (only X has
    values that small), fp32, with the products' own error, by 2^-21."""
    if dtype == "f32":
        g = torch.Generator(device="cpu").manual_seed(seed)
        return lambda t: t * (1 + (2 * torch.rand(t.shape, generator=g, dtype=torch.float64).to(t.device) - 1) * 2.0 ** -21)
    up = 2.0 ** round(0.5 * math.log2(max(shape[1:])))

    def keep(t):
        f = 1.0 if t.shape[1] == t.shape[2] and shape[1] != shape[2] else up
        return (t * f).half().double() / f
    return keep


def orth_check(W, v, r, steps, coeffs, eps, alpha, beta, dtype, what):
    """W against 64 bits: no further off than three times what the same roundings cost in 64-bit products
    (roundings that fall otherwise cost another amount of that size), in the norm of every matrix and in
    the largest element, besides those of W itself."""
    O = iterate(v, steps, coeffs, eps)
    E = iterate(v, steps, coeffs, eps, rounding(dtype, v.shape))
    ref = alpha * O + (0.0 if r is None else beta * r.to(v.device).double())
    err, em = (W.to(v.device).double() - ref).abs(), abs(alpha) * (E - O).abs()
    own = T.half_step(dtype) * ref.abs() + 3 * E32 * (ref.abs() + abs(alpha) * O.abs()) + T.tiny(dtype)
    norm = lambda t: torch.linalg.vector_norm(t, dim=(1, 2))
    size = v.shape[1] * v.shape[2]
    # (few values: one rounding decides; those of a matrix of a few values are allowed their largest step)
    slack = 4.0 if size >= 64 else 12.0
    step = 2.0 ** -21 if dtype == "f32" else 2.0 ** -11
    grow = sum(max(abs(coeffs[0]), 4.0) ** k for k in range(steps + 1))
    few = abs(alpha) * step * grow * norm(O) / math.sqrt(size) if size < 64 else 0.0
    over = norm(err) > slack * norm(em) + norm(own) + few
    assert not over.any(), (what, norm(err)[over], norm(em)[over], norm(own)[over])
    worst = (err - own).flatten(1).amax(1)
    assert (worst <= slack * em.flatten(1).amax(1) + few).all(), (what, worst, em.flatten(1).amax(1))


class Orth:
    """One update's calls, outputs guarded, from a workspace full of NaN."""

    def __init__(self, dtype, N, no, ni, **kw):
        self.dtype, self.od = dtype, L.orth(dtype, N, no, ni, **kw)
        self.shape = (N, no, ni)

    def __call__(self, g, m, mo, r, alpha, beta=1.0):
        ws = scribble(L.alloc_orth_workspace(self.od))
        W, wf = T.out(self.shape, T.DT[self.dtype])
        L.lp_orth_update(self.od, g, m, mo, r, W, ws, alpha=alpha, beta=beta)
        torch.cuda.synchronize()
        assert T.guarded(wf, W.numel())
        return W


def two_parts(t, up):
    """t times up as the sum of two f16 values."""
    f = (t * up).float()
    h = f.half()
    return (h.double() + (f - h.float()).half().double()) / up


def rest(t, up):
    """What f16 rounds off t times up, to 256ths of its last place."""
    h = (t * up).half().double()
    place = torch.exp2((torch.frexp(h)[1] - 11).clamp(min=-24).double()) / 256
    return torch.round((t * up - h) / place).clamp(-127, 127) * place / up


def iterate_kept(v, steps, coeffs, eps, dtype, noise=E32, seed=0):
    """The iteration in 64 bits with what the kernels round. Products' operands: X times 2^14 (of matrices of at most
    64 x 256, about the root of their size), A and b A + c A^2 times 2^8, to two f16 parts (fp32, and those small
    matrices in every type) or one, of which b A + c A^2 without (b + c) I in the last two steps (where |b + c| is at
    most 8). The X of a X: fp32 (small matrices), two parts too, or eight bits more but for the last two steps. Every
    product is off by a step of fp32 of its row's and column's norms."""
    a, b, c = coeffs
    gen = torch.Generator(device="cpu").manual_seed(seed)
    n, k = sorted(v.shape[1:])
    small = n <= 64 and k <= 256
    two = dtype == "f32" or small
    up = 2.0 ** round(0.5 * math.log2(n * k)) if small else 2.0 ** 14
    keep = two_parts if two else lambda t, f: (t * f).half().double() / f
    eye = torch.eye(n, dtype=torch.float64, device=v.device)

    def product(P, Q):
        size = torch.linalg.vector_norm(P, dim=2)[:, :, None] * torch.linalg.vector_norm(Q, dim=1)[:, None, :]
        u = 2 * torch.rand(size.shape, generator=gen, dtype=torch.float64).to(v.device) - 1
        return torch.matmul(P, Q.contiguous()) + noise * u * size

    X = v / (torch.linalg.vector_norm(v, dim=(1, 2), keepdim=True) + eps)
    tall = v.shape[1] > v.shape[2]
    X = X.transpose(1, 2).contiguous() if tall else X
    for s in range(steps):
        move = 0.0 if two or s + 2 < steps or abs(b + c) > 8 else b + c
        op = keep(X, up)
        A = keep(product(op, op.transpose(1, 2)), 2.0 ** 8)
        P = keep(b * A + c * product(A, A) - move * eye, 2.0 ** 8)
        own = X if small else op if two or s + 2 >= steps else op + rest(X, up)
        X = (a + move) * own + product(P, op)
    return X.transpose(1, 2) if tall else X


def orth_precise(W, r, O, E, dtype, what):
    """W = O + r, r within a step of -O: W's own rounding is one of a difference, and what W and r leave of O is off
    by no more than four times what the kernels' roundings cost in 64 bits (E: O with those), in every matrix's norm."""
    off = W.to(O.device).double() - r.to(O.device).double() - O
    own = T.half_step(dtype) * (O + r.to(O.device).double()).abs() + 3 * E32 * (O.abs() + r.to(O.device).double().abs()) + T.tiny(dtype)
    norm = lambda t: torch.linalg.vector_norm(t, dim=(1, 2))
    most = 4 * norm(E - O) + norm(own)
    assert (norm(off) <= most).all(), (what, (norm(off) / norm(O)).tolist()[:4], (most / norm(O)).tolist()[:4])


def norm_stats_sharp(x, eps):
    """norm_stats with a bound that does not grow with a row's mean: a first mean is off by D at most, the mean of what it
    leaves, d + D, is taken off that, and its square off the mean square. (x less the first mean is exact where
    both are near, else off by half a step of itself.)"""
    x = x.double()
    q = x.shape[1]
    n = 84 + q / 1024
    mean = x.mean(1, keepdim=True)
    d = x - mean
    D = n * E32 * x.abs().mean(1, keepdim=True)
    left = d.abs() + D
    ed = (n + 1) * E32 * left.mean(1, keepdim=True) + 2 * E32 * left
    var = (d * d).mean(1, keepdim=True)
    ev = (n + 4) * E32 * (left * left).mean(1, keepdim=True) + (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    er = rstd * (0.5 * ev / (var + eps) + 4 * E32)
    xh = d * rstd
    return xh, (ed * (rstd + er) + d.abs() * er + E32 * xh.abs()), rstd, er, n
