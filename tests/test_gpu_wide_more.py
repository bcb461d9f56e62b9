"""More of the wide operators on the GPU: what must not depend on what a workspace held, and forms that
the other tests' sizes do not reach. Bounds: tests/wide_testutil.py."""
import math

import pytest
import torch

import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [2, 33])
def test_what_the_workspace_held_does_not_matter(B):
    """fp32 probabilities that take their logits' place, several pieces of them: a tile's columns behind
    the last class read nothing that no kernel has written, so NaN there do not choose the instructions
    that form the tile. Weight gradients alone (nothing else writes the bytes behind the last row)."""
    q, nc = 262145, 300  # rows of W that do not start on 16 bytes, copied 256 at a time
    g = torch.Generator("cuda").manual_seed(1)
    u = torch.randn((B, q), generator=g, device="cuda")
    W = torch.randn((nc, q), generator=g, device="cuda") / 512
    lab = torch.randint(0, nc, (B,), generator=g, device="cuda")
    hd = L.label_head("f32", B, q, nc)
    ws = L.alloc_loss_labels_workspace(hd)
    J = torch.empty(1, device="cuda")
    results = []
    for fill in (0, 255):  # zeros, NaN
        ws.fill_(fill)
        dW = torch.empty_like(W)
        L.lp_loss_labels(hd, u, W, None, lab, J, ws, dW=dW)
        results.append(dW)
    assert torch.equal(*results)
    assert torch.isfinite(results[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_any_workspace_gives_the_same_bits(dtype):
    """Steps and heads over odd and whole sizes, one row to split contractions, from workspaces of zeros
    and of NaN."""
    dt = T.DT[dtype]
    g = torch.Generator().manual_seed(2)
    for B, ni, no in ((1, 33, 257), (3, 1001, 70), (24, 2049, 515), (300, 65, 513), (700, 257, 129), (4090, 130, 70)):
        x, W, b, dy = (T.draw(g, s, dtype).cuda() for s in ((B, ni), (no, ni), (no,), (B, no)))
        x8, xe = (t.cuda() for t in T.pack(x.cpu())) if B <= 300 else (None, None)
        st = L.step(dtype, "tanh", B, ni, no, 0.5)
        ws = L.alloc_step_workspace(st)
        results = []
        for fill in (0, 255):
            out = [torch.empty(s, dtype=dt, device="cuda") for s in ((B, no), (B, ni), (no, ni), (no,))]
            ws.fill_(fill)
            L.lp_step_forward(st, x, W, b, None, out[0], ws)
            for inp in ([x] if x8 is None else [x, (x8, xe)]):
                ws.fill_(fill)
                L.lp_step_backward(st, inp, W, b, dy, *out[1:], ws)
                results.append([t.clone() for t in out])
        half = len(results) // 2
        for r, s in zip(results[:half], results[half:]):
            assert all(torch.equal(a, c) for a, c in zip(r, s)), (B, ni, no)
    for B, q, nc in ((1, 65, 513), (33, 130, 1001), (300, 33, 70), (513, 260, 2050)):
        u, W, mu = (T.draw(g, s, dtype).cuda() for s in ((B, q), (nc, q), (nc,)))
        lab = torch.randint(-nc // 2 if B > 1 else 0, nc, (B,), generator=g).cuda()
        hd = L.label_head(dtype, B, q, nc)
        ws = L.alloc_loss_labels_workspace(hd)
        results = []
        for fill in (0, 255):
            out = [torch.empty(s, dtype=dt, device="cuda") for s in ((B, q), (nc, q), (nc,))]
            J, row = torch.empty(1, device="cuda"), torch.empty(B, device="cuda")
            ws.fill_(fill)
            L.lp_loss_labels(hd, u, W, mu, lab, J, ws, row=row, du=out[0], dW=out[1], dmu=out[2])
            results.append([J, row] + out)
        assert all(torch.equal(a, c) for a, c in zip(*results)), (B, q, nc)


# fp32 products are split bf16 ones, whose instruction's sums round towards minus infinity. Summed with
# one sign, sums of K positive products have a mean relative error (measured, 96000 results each) of
# -1.3e-8, -6.1e-9 and -2.1e-8 for K = 220, 1024 and 8192. The middle half is summed with the other sign,
# which cancels the error of a sum that grows evenly but for the steps of its last place (a binade's
# step is constant: for an end anywhere in its binade that leaves at most a quarter) and the unevenness
# of the quarters (7 stages at K = 220: a seventh). Limit: a third of the drift, and three standard
# deviations of the mean of N results that are off by 2^-22 at most, each on its own: 3 2^-22 / sqrt(N).
DRIFT = {220: 1.3e-8, 1024: 6.1e-9, 8192: 2.1e-8}


def sides(K, positive):
    g = torch.Generator("cuda").manual_seed(K + positive)
    a, b = (torch.randn(n, K, generator=g, device="cuda") for n in (300, 320))
    return (a.abs(), b.abs()) if positive else (a, b)


@pytest.mark.parametrize("form", ["z", "dx", "dW"])
@pytest.mark.parametrize("positive", [True, False])
@pytest.mark.parametrize("K", [220, 1024, 8192])
def test_fp32_products_do_not_drift(K, positive, form):
    """The mean error of each of a step's three products, as a part of the sum of its terms' magnitudes
    (cancelling sums stay smaller than that on the way, and so does their drift)."""
    a, b = sides(K, positive)
    M, N = len(a), len(b)
    out = torch.empty(M, N, device="cuda")
    if form == "z":
        st = L.step("f32", "identity", M, K, N)
        L.lp_step_forward(st, a, b, None, None, out, L.alloc_step_workspace(st))
    elif form == "dx":  # h g W with g = dy = a, W = b^T
        st = L.step("f32", "identity", M, N, K)
        L.lp_step_backward(st, torch.zeros(M, N, device="cuda"), b.t().contiguous(), None, a, out, None, None,
                           L.alloc_step_workspace(st))
    else:  # h g^T x with g = dy = a^T, x = b^T
        st = L.step("f32", "identity", K, N, M)
        L.lp_step_backward(st, b.t().contiguous(), torch.zeros(M, N, device="cuda"), None, a.t().contiguous(), None, out,
                           None, L.alloc_step_workspace(st))
    ref = a.double() @ b.double().t().contiguous()
    mag = a.abs().double() @ b.abs().double().t().contiguous()
    mean = float(((out.double() - ref) / mag).mean())
    assert abs(mean) <= DRIFT[K] / 3 + 3 * 2 ** -22 / math.sqrt(M * N), mean


def test_fp32_layers_have_no_common_bias():
    """Residual steps of the identity in a row: the mean relative error of their increments (the rounding
    of the state is unbiased, about 1e-6 of an increment: 5e-10 in the mean of three million)."""
    q, B, N = 220, 200, 64
    g = torch.Generator("cuda").manual_seed(3)
    st = L.step("f32", "identity", B, q, q)
    ws = L.alloc_step_workspace(st)
    u = torch.randn(B, q, generator=g, device="cuda").abs() + 0.5
    mean = []
    for _ in range(N):
        W = torch.randn(q, q, generator=g, device="cuda").abs()
        W *= 0.1 / W.sum(1).mean()
        y = torch.empty_like(u)
        L.lp_step_forward(st, u, W, None, u, y, ws)
        z = u.double() @ W.double().t().contiguous()
        mean.append(((y.double() - u.double()) / z - 1).mean())
        u = y
    assert abs(float(torch.stack(mean).mean())) <= DRIFT[220] / 3 + 5e-10


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("ni,no", [(40, 16385), (33, 20001)])
def test_one_row_to_many_outputs(dtype, ni, no):
    """More outputs than the narrower one-row kernel serves, with and without a checkpoint, and back."""
    g = torch.Generator().manual_seed(no)
    x, W, b, dy = T.draw(g, (1, ni), dtype), T.draw(g, (no, ni), dtype, 1 / math.sqrt(ni)), T.draw(g, (no,), dtype, 0.3), \
        T.draw(g, (1, no), dtype, 0.1)
    r = T.draw(g, (1, no), dtype)
    s = T.Step(dtype, "tanh", 1, ni, no, 0.5)
    dev = [T.gpu(t) for t in (x, W, b)]
    y, y8, ye = s.forward(*dev, T.gpu(r), ck=True)
    T.check(y, *T.forward(x, W, b, r, "tanh", 0.5, dtype), "y")
    e8, ee = T.pack(y.cpu())
    assert torch.equal(y8.cpu(), e8) and torch.equal(ye.cpu(), ee)
    T.check(s.forward(*dev, T.gpu(r)), *T.forward(x, W, b, r, "tanh", 0.5, dtype), "y without a checkpoint")
    got = s.backward(*dev, T.gpu(dy), False)
    for name, a, (v, e) in zip(("dx", "dW", "db"), got, T.backward(x, W, b, dy, "tanh", 0.5, False, dtype)):
        T.check(a, v, e, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_one_row_of_many_classes(dtype):
    q, nc = 64, 20001
    g = torch.Generator().manual_seed(4)
    u, W, mu = T.draw(g, (1, q), dtype), T.draw(g, (nc, q), dtype, 2 / math.sqrt(q)), T.draw(g, (nc,), dtype, 0.5)
    lab = torch.tensor([nc - 1])
    hd = L.label_head(dtype, 1, q, nc)
    ws = L.alloc_loss_labels_workspace(hd)
    out, flat = zip(*[T.out(s, T.DT[dtype]) for s in ((1, q), (nc, q), (nc,))])
    J, row = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    L.lp_loss_labels(hd, T.gpu(u), T.gpu(W), T.gpu(mu), lab.cuda(), J, ws, row=row, du=out[0], dW=out[1], dmu=out[2])
    torch.cuda.synchronize()
    assert all(T.guarded(f, o.numel()) for o, f in zip(out, flat))
    (rJ, eJ), *rest = T.loss(u, W, mu, lab, 1.0, dtype)
    T.check(J, rJ.reshape(1), eJ.reshape(1), "J")
    for name, a, (r, e) in zip(("row", "du", "dW", "dmu"), (row,) + out, rest):
        T.check(a, r, e, name)


@pytest.mark.parametrize("k", [108, 114, 122, 130])
@pytest.mark.parametrize("B", [1, 70])
def test_small_fp32_operands(k, B):
    """A value is taken as three bf16 ones, the last of which is a multiple of 2^-133 (half of it off):
    2^-134 of every other operand's value on top of the usual bound, nothing for a row alone."""
    ni, no = 64, 72
    g = torch.Generator().manual_seed(k)
    x = (torch.randn((B, ni), generator=g, dtype=torch.float64) * 2.0 ** -k).float()
    W = (torch.randn((no, ni), generator=g, dtype=torch.float64) * 2.0 ** 60).float()
    dy = (torch.randn((B, no), generator=g, dtype=torch.float64) * 2.0 ** -k).float()
    s = T.Step("f32", "identity", B, ni, no, 1.0)
    y = s.forward(T.gpu(x), T.gpu(W), None, None)
    ref, bound = T.preact(x, W, None)
    part = 2.0 ** -134
    off = 0 if B == 1 else part * (W.double().abs().sum(1)[None] + x.double().abs().sum(1)[:, None])
    T.check(y, ref, (bound + off) * (1 + 2 ** -20) + T.half_step("f32") * ref.abs() + T.tiny("f32"), "y")
    dx, dW, _ = s.backward(T.gpu(x), T.gpu(W), None, T.gpu(dy), False)
    d, w, v = dy.double(), W.double(), x.double()
    for name, got, r, mag, n, o in (
            ("dx", dx, d @ w, d.abs() @ w.abs(), no, w.abs().sum(0)[None] + d.abs().sum(1)[:, None]),
            ("dW", dW, d.t() @ v, d.abs().t() @ v.abs(), B, v.abs().sum(0)[None] + d.abs().sum(0)[:, None])):
        T.check(got, r, ((n + 2) * T.E32 * mag + part * o) * (1 + 2 ** -20) + T.half_step("f32") * r.abs() + T.tiny("f32"),
                name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,ni,no", [(2 ** 24, 3, 2), (3, 2 ** 20, 5), (2, 5, 2 ** 20), (1, 2 ** 20, 33)])
def test_steps_at_the_limits(dtype, B, ni, no):
    """The most rows, the widest input and output (64 bits on the GPU)."""
    g = torch.Generator("cuda").manual_seed(B)
    dt = T.DT[dtype]
    x, W, b, dy = (torch.randn(s, generator=g, device="cuda").mul_(f).to(dt)
                   for s, f in (((B, ni), 1.0), ((no, ni), ni ** -0.5), ((no,), 0.3), ((B, no), 0.1)))
    s = T.Step(dtype, "tanh", B, ni, no, 0.5)
    y, y8, ye = s.forward(x, W, b, None, ck=True)
    T.check(y, *T.forward(x, W, b, None, "tanh", 0.5, dtype), "y")
    back = torch.empty_like(y)
    L.lp_checkpoint_load(y8, ye, back)
    q8, qe, other = torch.empty_like(y8), torch.empty_like(ye), torch.empty_like(y)
    L.lp_checkpoint_store(y, q8, qe)
    L.lp_checkpoint_load(q8, qe, other)
    assert torch.equal(q8, y8) and torch.equal(qe, ye) and torch.equal(other, back)
    got = s.backward(x, W, b, dy, False)
    for name, a, (v, e) in zip(("dx", "dW", "db"), got, T.backward(x, W, b, dy, "tanh", 0.5, False, dtype)):
        T.check(a, v, e, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,q,nc", [(2 ** 24, 3, 2), (3, 2 ** 20, 40), (3, 4, 2 ** 24), (1, 5, 2 ** 24)])
def test_heads_at_the_limits(dtype, B, q, nc):
    """The most rows, features and classes, in norms: half a step of P and of the result, and fp32 sums
    (a probability below 2^-126 may be zero: nc 2^-126 is nothing here)."""
    g = torch.Generator("cuda").manual_seed(nc)
    dt = T.DT[dtype]
    u, W, mu = (torch.randn(s, generator=g, device="cuda").mul_(f).to(dt)
                for s, f in (((B, q), 1.0), ((nc, q), q ** -0.5), ((nc,), 0.5)))
    lab = torch.randint(0, nc, (B,), generator=g, device="cuda")
    if B > 2:
        lab[1] = -1
    hd = L.label_head(dtype, B, q, nc)
    ws = L.alloc_loss_labels_workspace(hd)
    J, row = torch.empty(1, device="cuda"), torch.empty(B, device="cuda")
    out = [torch.empty(s, dtype=dt, device="cuda") for s in ((B, q), (nc, q), (nc,))]
    L.lp_loss_labels(hd, u, W, mu, lab, J, ws, row=row, du=out[0], dW=out[1], dmu=out[2])
    on = lab >= 0
    n = int(on.sum())
    z = u.double() @ W.double().t() + mu.double()
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(B, device="cuda")
    ref = torch.where(on, lse - z[rows, lab.clamp(min=0)], 0)
    P = z.sub_(lse[:, None]).exp_()
    P[rows, lab.clamp(min=0)] -= 1
    P[~on] = 0
    refs = [(ref.sum() / n).reshape(1), ref, P @ W.double() / n, P.t() @ u.double() / n, P.sum(0) / n]
    half = 2 ** -8 if dtype == "bf16" else 2 ** -18
    for name, a, r in zip(("J", "row", "du", "dW", "dmu"), [J, row] + out, refs):
        d = float((a.double() - r).norm() / r.norm())
        assert d <= (2 ** -18 if name in ("J", "row") else half), (name, d)
