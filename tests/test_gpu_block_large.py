"""Norms, gated layers and updates of arrays with more than 2^31 values, and of several streams at once: the last
rows and matrices against 64 bits. Bounds: tests/block_testutil.py."""
import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu


def filled(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * std)
    return t


def test_norm_beyond_32_bits():
    B, q = 530000, 4096
    x, dy = filled((B, q), torch.bfloat16, 1), filled((B, q), torch.bfloat16, 2, 0.1)
    gamma, beta = filled((q,), torch.bfloat16, 3), filled((q,), torch.bfloat16, 4)
    nd = L.norm("bf16", B, q)
    ws = K.scribble(L.alloc_norm_workspace(nd))
    y, (dgamma, dbeta) = torch.empty_like(x), (torch.empty_like(gamma) for _ in range(2))
    L.lp_norm_forward(nd, x, gamma, beta, y)
    rows = [slice(0, 3), slice(B - 5, B)]
    for r in rows:
        T.check(y[r], *K.norm_forward(x[r].cpu(), gamma.cpu(), beta.cpu(), 1e-5, "bf16"), "y")
    L.lp_norm_backward(nd, x, gamma, dy, None, y, dgamma, dbeta, ws)
    for r in rows:
        T.check(y[r], *K.norm_backward(x[r].cpu(), gamma.cpu(), dy[r].cpu(), None, 1e-5, "bf16")[0], "dx")
    want, mag = torch.zeros((2, q), dtype=torch.float64, device="cuda"), torch.zeros((2, q), dtype=torch.float64, device="cuda")
    for i in range(0, B, 10000):
        d = dy[i:i + 10000].double()
        c = x[i:i + 10000].double()
        c = c - c.mean(1, keepdim=True)
        p = d * c / ((c * c).mean(1, keepdim=True) + 1e-5).sqrt()
        want += torch.stack([p.sum(0), d.sum(0)])
        mag += torch.stack([p.abs().sum(0), d.abs().sum(0)])
    # a thread adds at most 2048 terms in fp32, four groups join, the rest is fp64; xh is good to 100 steps of fp32
    bound = (2048 + 4 + 100) * K.E32 * mag
    for k, a in enumerate((dgamma, dbeta)):
        T.check(a, want[k], bound[k] + T.half_step("bf16") * (want[k].abs() + bound[k]), ("dgamma", "dbeta")[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gated_beyond_32_bits(dtype):
    B, ni, no = 270000, 72, 8200
    dt = T.DT[dtype]
    x, dy = filled((B, ni), dt, 1), filled((B, no), dt, 2, 0.1)
    Wg, Wu = filled((no, ni), dt, 3, 0.15), filled((no, ni), dt, 4, 0.12)
    gd = L.gated(dtype, "silu", B, ni, no)
    ws = L.alloc_gated_workspace(gd)
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    L.lp_gated_forward(gd, x, Wg, Wu, y, ws)
    L.lp_gated_backward(gd, x, Wg, Wu, dy, dx, None, None, ws)
    for r in (slice(0, 3), slice(B - 5, B)):
        a = [t.cpu() for t in (x[r], Wg, Wu, dy[r])]
        T.check(y[r], *K.gated_forward(a[0], a[1], a[2], "silu", dtype), "y")
        T.check(dx[r], *K.gated_backward(*a, "silu", dtype)[0], "dx")


@pytest.mark.parametrize("dtype,shape", [("bf16", (560000, 60, 64)), ("f32", (560000, 60, 64)), ("bf16", (600, 1900, 1900)),
                                         ("bf16", (1 << 24, 3, 2))])
def test_orth_beyond_32_bits(dtype, shape):
    dt = T.DT[dtype]
    g = filled(shape, dt, 1, 0.01)
    m = filled(shape, torch.float32, 2, 0.01) if 1000 < shape[0] < 1 << 20 else None
    od = L.orth(dtype, *shape, steps=2, mu=0.9, nesterov=m is not None)
    W = torch.empty_like(g)
    last = slice(shape[0] - 3, shape[0])
    _, v = K.momentum(g[last], None if m is None else m[last], 0.9 if m is not None else None, m is not None, dtype)
    L.lp_orth_update(od, g, m, m, None, W, K.scribble(L.alloc_orth_workspace(od)), alpha=1.0)
    K.orth_check(W[last], v, None, 2, L.QUINTIC, 1e-7, 1.0, 0.0, dtype, "O")
    assert torch.isfinite(W[::max(1, shape[0] // 50)]).all()


def test_several_streams_at_once():
    """Calls of all kinds on four streams, each with its own arrays and workspaces, give what they give alone."""
    dtype, jobs = "bf16", []
    for k in range(4):
        B, q, m = 300 + 77 * k, 200 + 8 * k, 500 + 33 * k
        t = {n: filled(s, torch.bfloat16, 10 * k + i, d) for i, (n, s, d) in enumerate(
            (("x", (B, q), 1.0), ("gamma", (q,), 1.0), ("Wg", (m, q), 0.1), ("Wu", (m, q), 0.1), ("dp", (B, m), 0.1)))}
        nd, gd, od = L.norm(dtype, B, q), L.gated(dtype, "gelu", B, q, m), L.orth(dtype, 1, m, q)
        ws = [f(d) for f, d in ((L.alloc_norm_workspace, nd), (L.alloc_gated_workspace, gd), (L.alloc_orth_workspace, od))]
        out = {n: torch.empty_like(t[s]) for n, s in (("n", "x"), ("p", "dp"), ("dn", "x"), ("dx", "x"), ("dWg", "Wg"), ("dWu", "Wu"),
                                                      ("dg", "gamma"), ("db", "gamma"), ("O", "Wg"))}

        def run(t=t, nd=nd, gd=gd, od=od, ws=ws, o=out):
            L.lp_norm_forward(nd, t["x"], t["gamma"], None, o["n"])
            L.lp_gated_forward(gd, o["n"], t["Wg"], t["Wu"], o["p"], ws[1])
            L.lp_gated_backward(gd, o["n"], t["Wg"], t["Wu"], t["dp"], o["dn"], o["dWg"], o["dWu"], ws[1])
            L.lp_norm_backward(nd, t["x"], t["gamma"], o["dn"], o["n"], o["dx"], o["dg"], o["db"], ws[0])
            L.lp_orth_update(od, o["dWg"], None, None, None, o["O"], ws[2], alpha=1.0)

        run()
        torch.cuda.synchronize()
        want = {n: v.clone() for n, v in out.items()}
        for w in ws:
            K.scribble(w)
        jobs.append((torch.cuda.Stream(), run, out, want))
    torch.cuda.synchronize()
    for _ in range(5):
        for st, run, _, _ in jobs:
            with torch.cuda.stream(st):
                run()
    torch.cuda.synchronize()
    for _, _, out, want in jobs:
        for n in out:
            assert torch.equal(out[n], want[n]), n
