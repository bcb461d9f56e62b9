"""Operators around wide layers, as cases to measure: layer norm, gated layers, orthogonalised updates.

  norm   y = gamma (x - mean) / sqrt(var + eps) + beta over the features of every row, and its
         gradients dx (optionally with the gradient of a residual added), dgamma, dbeta
  gated  y = s(x Wg^T) (x Wu^T), the gated layer of a feed-forward block, and its gradients
  orth   W = alpha O + beta r for a batch of matrices, O the momentum v = g + mu m' (m' = mu m + g)
         orthogonalised by Newton-Schulz products: X = v / (|v| + eps), then some times
         A = X X^T, X = a X + (b A + c A^2) X

A case's types are those of its floating-point arrays ("bf16", "f16", "f32"; momentum is held in 32
bits); every sum is held in 32 bits. ``own`` selects the
library's kernels, else the operators run as elementary torch operations.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
COEFFS = (3.4445, -4.7750, 2.0315)  # a, b, c: singular values in (0, 1] go to about 1 in five steps
NORM_EPS, ORTH_EPS = 1e-5, 1e-7
MU = 0.95


def _lib():
    from paper_1812_04352_amd import lp
    return lp


# ---------------------------------------------------------------------- the cases


def _norm(back, dtype, B, q, dr=False):
    return dict(kind="norm", back=back, dtype=dtype, B=B, q=q, dr=dr)


def _gated(back, dtype, act, B, ni, no):
    return dict(kind="gated", back=back, dtype=dtype, act=act, B=B, ni=ni, no=no)


def _orth(dtype, N, no, ni, steps=5, momentum=True, residual=True):
    return dict(kind="orth", dtype=dtype, N=N, no=no, ni=ni, steps=steps, momentum=momentum, residual=residual)


def listed():
    return [
        # one token through the norm in front of a wide layer
        dict(_norm(False, "bf16", 1, 4096), name="norm one token"),
        # the states of one layer of the hyperspectral network (220 bands, batch 1000) in single precision
        dict(_norm(False, "f32", 1000, 220), name="norm bands f32"),
        # the way back through the norm of a residual layer, the residual's gradient added
        dict(_norm(True, "bf16", 8192, 4096, dr=True), name="norm backward train"),
        # odd width and ragged batch, a norm without a residual around it
        dict(_norm(True, "f16", 5003, 1111), name="norm backward ragged"),
        # one token through a gated layer: both weights are read once for one row
        dict(_gated(False, "bf16", "silu", 1, 4096, 10240), name="gated one token"),
        # a few requests answered together
        dict(_gated(False, "f16", "gelu", 24, 2048, 5120), name="gated few tokens"),
        # a training batch through a wide gated layer
        dict(_gated(False, "bf16", "silu", 8192, 4096, 10240), name="gated forward train"),
        # the way back through it
        dict(_gated(True, "bf16", "silu", 8192, 4096, 10240), name="gated backward train"),
        # the way back through a gated layer over the hyperspectral bands, odd width, single precision
        dict(_gated(True, "f32", "tanh", 1000, 220, 587), name="gated backward bands f32"),
        # the update of all layers of the deep dense network (2048 layers of width 64), single precision
        dict(_orth("f32", 2048, 64, 64), name="orth deep f32"),
        # the update of the hyperspectral network's layers
        dict(_orth("f32", 2048, 220, 220), name="orth bands f32"),
        # the update of a wide layer
        dict(_orth("bf16", 1, 4096, 4096), name="orth wide"),
    ]


MOST = 12.0 * 8192 * 4096 * 10240  # operations of the largest listed case
ACTS = ("tanh", "relu", "smoothrelu", "identity", "silu", "gelu")


def _spread(rng, lo, hi):
    """A size spread over the logarithm of lo..hi: as drawn (odd ones among them) or on a multiple of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 64 and rng.random() < 0.5:
        n = (n + 32) // 64 * 64
    return min(max(n, lo), hi)


def draw(rng):
    kind = rng.choice(("norm", "gated", "gated", "orth"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    # single precision has a sixteenth of the 16-bit rate
    most = MOST / 16 if dtype == "f32" else MOST
    while True:
        if kind == "norm":
            c = _norm(rng.random() < 0.6, dtype, _spread(rng, 1, 32768), _spread(rng, 16, 16384), rng.random() < 0.5)
            if c["B"] * c["q"] <= 1 << 26:
                return c
        elif kind == "gated":
            back = rng.random() < 0.6
            # (the slope of relu jumps: where a sum of 32 bits lies next to 0, either side is right)
            act = rng.choice(ACTS if dtype != "f32" or not back else tuple(a for a in ACTS if a != "relu"))
            c = _gated(back, dtype, act, _spread(rng, 1, 16384), _spread(rng, 32, 8192), _spread(rng, 32, 16384))
            if work(c)["flops"] <= most:
                return c
        else:
            # a layer of any depth: many small matrices or a few large ones
            c = _orth(dtype, _spread(rng, 1, 2048), _spread(rng, 8, 8192), _spread(rng, 8, 8192),
                      rng.choice((3, 5, 6)), rng.random() < 0.7, rng.random() < 0.8)
            # (the plain form holds some arrays of the batch in 32 bits)
            if work(c)["flops"] <= most / 2 and c["N"] * max(c["no"], c["ni"]) ** 2 <= 1 << 28:
                return c


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "norm":
        n, q = case["B"] * case["q"], case["q"]
        if not case["back"]:
            return dict(bytes=float(2 * n * e + 2 * q * e), flops=8.0 * n)
        return dict(bytes=float((3 + case["dr"]) * n * e + 3 * q * e), flops=18.0 * n)
    if case["kind"] == "gated":
        B, ni, no = case["B"], case["ni"], case["no"]
        if not case["back"]:
            return dict(bytes=float((B * ni + 2 * ni * no + B * no) * e), flops=4.0 * B * ni * no)
        return dict(bytes=float((2 * B * ni + 4 * ni * no + B * no) * e), flops=12.0 * B * ni * no)
    n, k = min(case["no"], case["ni"]), max(case["no"], case["ni"])
    # X X^T and A^2 are symmetric: half of each is enough
    each = e + (8 if case["momentum"] else 0) + e * (1 + case["residual"])
    return dict(bytes=float(case["N"] * n * k * each), flops=float(case["N"] * case["steps"]) * (3.0 * n * n * k + 1.0 * n ** 3))


# ---------------------------------------------------------------------- inputs


def _normal(g, shape, dtype, std):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _gradients(g, N, no, ni, dtype):
    """Gradients of weights [N][no][ni]: noise and a few strong directions, each matrix of its own size."""
    v = torch.randn((N, no, ni), generator=g, device="cuda")
    rank = min(4, no, ni)
    p = torch.randn((N, no, rank), generator=g, device="cuda")
    r = torch.randn((N, rank, ni), generator=g, device="cuda")
    v += torch.bmm(p, r)
    v *= 1e-2 * torch.randn((N, 1, 1), generator=g, device="cuda").exp()
    return v.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case=case)
    L = _lib() if own else None
    if case["kind"] == "norm":
        B, q = case["B"], case["q"]
        # rows of different size and place
        x = torch.randn((B, q), generator=g, device="cuda") * torch.randn((B, 1), generator=g, device="cuda").exp()
        s["x"] = (x + torch.randn((B, 1), generator=g, device="cuda")).to(dt)
        s["gamma"] = (1 + 0.2 * torch.randn((q,), generator=g, device="cuda")).to(dt)
        if case["back"]:
            s["dy"] = _normal(g, (B, q), dt, 0.05)
            s["dr"] = _normal(g, (B, q), dt, 0.05) if case["dr"] else None
        else:
            s["beta"] = _normal(g, (q,), dt, 0.2)
        if own:
            s["nd"] = L.norm(case["dtype"], B, q, eps=NORM_EPS)
            if case["back"]:
                s["dx"] = torch.empty((B, q), device="cuda", dtype=dt)
                s["dgamma"], s["dbeta"] = (torch.empty((q,), device="cuda", dtype=dt) for _ in range(2))
                s["ws"] = L.alloc_norm_workspace(s["nd"])
            else:
                s["y"] = torch.empty((B, q), device="cuda", dtype=dt)
        return s
    if case["kind"] == "gated":
        B, ni, no = case["B"], case["ni"], case["no"]
        s["x"] = _normal(g, (B, ni), dt, 1.0)
        s["Wg"], s["Wu"] = (_normal(g, (no, ni), dt, 1.0 / math.sqrt(ni)) for _ in range(2))
        if case["back"]:
            s["dy"] = _normal(g, (B, no), dt, 0.05)
        if own:
            s["gd"] = L.gated(case["dtype"], case["act"], B, ni, no)
            s["ws"] = L.alloc_gated_workspace(s["gd"], grad=case["back"])
            if case["back"]:
                s["dx"], s["dWg"], s["dWu"] = (torch.empty_like(s[k]) for k in ("x", "Wg", "Wu"))
            else:
                s["y"] = torch.empty((B, no), device="cuda", dtype=dt)
        return s
    N, no, ni = case["N"], case["no"], case["ni"]
    s["g"] = _gradients(g, N, no, ni, dt)
    s["m"] = _gradients(g, N, no, ni, torch.float32) if case["momentum"] else None
    s["r"] = _normal(g, (N, no, ni), dt, 1.0 / math.sqrt(ni)) if case["residual"] else None
    s["alpha"], s["beta"] = -0.02 * math.sqrt(max(1.0, no / ni)), 0.999
    if own:
        s["od"] = L.orth(case["dtype"], N, no, ni, steps=case["steps"], coeffs=COEFFS, eps=ORTH_EPS,
                         mu=MU if case["momentum"] else 0.0, nesterov=case["momentum"])
        s["ws"] = L.alloc_orth_workspace(s["od"])
        s["mo"] = torch.empty_like(s["m"]) if case["momentum"] else None
        s["W"] = torch.empty((N, no, ni), device="cuda", dtype=dt)
    return s


# ---------------------------------------------------------------------- plain forms


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    dt = s["x"].dtype
    xc = x - x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + NORM_EPS)
    xh = xc * rstd
    if not c["back"]:
        return (xh * s["gamma"].float() + s["beta"].float()).to(dt)
    dy = s["dy"].float()
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if s["dr"] is not None:
        dx = dx + s["dr"].float()
    return dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)


def _act(z, act):
    if act == "tanh":
        return torch.tanh(z)
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "smoothrelu":
        return torch.where(z.abs() <= 0.1, (2.5 * z + 0.5) * z + 0.025, torch.clamp(z, min=0.0))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _dact(z, act):
    if act == "tanh":
        t = torch.tanh(z)
        return 1.0 - t * t
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "smoothrelu":
        return torch.where(z.abs() <= 0.1, 5.0 * z + 0.5, (z > 0).to(z.dtype))
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return t * (1.0 + z * (1.0 - t))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _plain_gated(s):
    c = s["case"]
    dt = s["x"].dtype
    x, Wg, Wu = s["x"].float(), s["Wg"].float(), s["Wu"].float()
    zg, zu = x @ Wg.t(), x @ Wu.t()
    if not c["back"]:
        return (_act(zg, c["act"]) * zu).to(dt)
    dy = s["dy"].float()
    dzu = dy * _act(zg, c["act"])
    dzg = dy * zu * _dact(zg, c["act"])
    return (dzg @ Wg + dzu @ Wu).to(dt), (dzg.t() @ x).to(dt), (dzu.t() @ x).to(dt)


def _plain_orth(s):
    c = s["case"]
    g = s["g"].float()
    mo = None
    v = g
    if s["m"] is not None:
        mo = MU * s["m"] + g
        v = g + MU * mo
    n = torch.sqrt((v.double() ** 2).sum((1, 2), keepdim=True)).float()
    X = v / (n + ORTH_EPS)
    tall = c["no"] > c["ni"]
    if tall:
        X = X.transpose(1, 2).contiguous()
    a, b, d = COEFFS
    for _ in range(c["steps"]):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * A + d * torch.bmm(A, A), X)
    if tall:
        X = X.transpose(1, 2)
    W = s["alpha"] * X
    if s["r"] is not None:
        W = W + s["beta"] * s["r"].float()
    W = W.to(s["g"].dtype).contiguous()
    return W if mo is None else (W, mo)


def _plain(s):
    kind = s["case"]["kind"]
    return _plain_norm(s) if kind == "norm" else _plain_gated(s) if kind == "gated" else _plain_orth(s)


# ---------------------------------------------------------------------- the library's calls


def _own(s):
    c = s["case"]
    L = _lib()
    if c["kind"] == "norm":
        if c["back"]:
            L.lp_norm_backward(s["nd"], s["x"], s["gamma"], s["dy"], s["dr"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
            return s["dx"], s["dgamma"], s["dbeta"]
        L.lp_norm_forward(s["nd"], s["x"], s["gamma"], s["beta"], s["y"])
        return s["y"]
    if c["kind"] == "gated":
        if c["back"]:
            L.lp_gated_backward(s["gd"], s["x"], s["Wg"], s["Wu"], s["dy"], s["dx"], s["dWg"], s["dWu"], s["ws"])
            return s["dx"], s["dWg"], s["dWu"]
        L.lp_gated_forward(s["gd"], s["x"], s["Wg"], s["Wu"], s["y"], s["ws"])
        return s["y"]
    L.lp_orth_update(s["od"], s["g"], s["m"], s["mo"], s["r"], s["W"], s["ws"], alpha=s["alpha"], beta=s["beta"])
    return s["W"] if s["mo"] is None else (s["W"], s["mo"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------- 64 bits


def _sigma64(z, act):
    """The activation and its slope."""
    if act == "identity":
        return z, torch.ones_like(z)
    if act == "tanh":
        return torch.tanh(z), 1 / torch.cosh(z.clamp(-300, 300)) ** 2
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t + z * t * torch.sigmoid(-z)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    pos = (z > 0).double()
    if act == "relu":
        return z * pos, pos
    mid = z.abs() <= 0.1
    return torch.where(mid, 2.5 * z ** 2 + 0.5 * z + 0.025, z * pos), torch.where(mid, 5 * z + 0.5, pos)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        x, gamma = s["x"].double(), s["gamma"].double()
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        rstd = (var + NORM_EPS) ** -0.5
        if not case["back"]:
            return torch.addcmul(s["beta"].double(), (x - mean) * rstd, gamma)
        xh, dy = (x - mean) * rstd, s["dy"].double()
        g = dy * gamma
        along = (g * xh).sum(1, keepdim=True) / case["q"]
        dx = (g - g.sum(1, keepdim=True) / case["q"] - along * xh) * rstd
        return dx if s["dr"] is None else dx + s["dr"].double(), (xh * dy).sum(0), dy.sum(0)
    if case["kind"] == "gated":
        x, Wg, Wu = s["x"].double(), s["Wg"].double(), s["Wu"].double()
        f, df = _sigma64(torch.mm(x, Wg.t()), case["act"])
        zu = torch.mm(x, Wu.t())
        if not case["back"]:
            return f * zu
        dy = s["dy"].double()
        f *= dy
        df *= dy * zu
        return torch.addmm(torch.mm(f, Wu), df, Wg), torch.mm(df.t(), x), torch.mm(f.t(), x)
    a, b, c = COEFFS
    W, mo = [], []
    for i in range(case["N"]):  # matrix by matrix
        v = s["g"][i].double()
        if case["momentum"]:
            mo.append(v + MU * s["m"][i].double())
            v = v + MU * mo[-1]
        X = v / (torch.linalg.vector_norm(v) + ORTH_EPS)
        wide = X if case["no"] <= case["ni"] else X.t()
        for _ in range(case["steps"]):
            A = wide @ wide.t()
            P = torch.addmm(A * b, A, A, alpha=c)
            P.diagonal().add_(a)
            wide = P @ wide
        X = s["alpha"] * (wide if case["no"] <= case["ni"] else wide.t())
        W.append(X if s["r"] is None else X + s["beta"] * s["r"][i].double())
    W = torch.stack(W)
    return (W, torch.stack(mo)) if case["momentum"] else W
