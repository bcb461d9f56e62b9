"""Norms, gated layers, layer steps, the label head and orthogonalised updates together, as a training program uses
them: residual blocks u' = u + h (s(n Wg^T) (n Wu^T)) Wd^T, n = norm(u), forward, the loss, the way back and the
update of all weights. Every array is checked against its operator's 64-bit form of the arrays that it was made of
(bounds: tests/block_testutil.py, tests/wide_testutil.py), the whole against autograd in 64 bits."""
import math

import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

EPS, H, ALPHA, KEEP, MU = 1e-5, 0.5, -0.02, 0.999, 0.9


class Network:
    """`layers` blocks of width q with m hidden features and a head over nc classes; the blocks' weights lie in one
    array a kind, so that an update takes all of them at once."""

    def __init__(self, dtype, act, B, q, m, layers, nc):
        self.dtype, self.act, self.layers, dt = dtype, act, layers, T.DT[dtype]
        e = lambda *s: torch.empty(s, dtype=dt, device="cuda")
        self.nd, self.gd = L.norm(dtype, B, q, EPS), L.gated(dtype, act, B, q, m)
        self.st, self.head = L.step(dtype, "identity", B, m, q, H), L.label_head(dtype, B, q, nc)
        self.ups = {k: L.orth(dtype, layers, *s, mu=MU, nesterov=True) for k, s in (("Wg", (m, q)), ("Wu", (m, q)), ("Wd", (q, m)))}
        self.nws, self.gws = L.alloc_norm_workspace(self.nd), L.alloc_gated_workspace(self.gd)
        self.sws, self.hws = L.alloc_step_workspace(self.st), L.alloc_loss_labels_workspace(self.head, True)
        self.ows = {k: L.alloc_orth_workspace(o) for k, o in self.ups.items()}
        self.n, self.p, self.u = e(layers, B, q), e(layers, B, m), e(layers, B, q)
        self.dn, self.dp, self.lam = e(layers, B, q), e(layers, B, m), e(layers + 1, B, q)
        self.grads = {"gamma": e(layers, q), "beta": e(layers, q), "Wg": e(layers, m, q), "Wu": e(layers, m, q), "Wd": e(layers, q, m),
                      "HW": e(nc, q)}
        self.J = torch.empty(1, device="cuda")

    def run(self, x, w, labels, mom):
        for k in range(self.layers):
            u = x if k == 0 else self.u[k - 1]
            L.lp_norm_forward(self.nd, u, w["gamma"][k], w["beta"][k], self.n[k])
            L.lp_gated_forward(self.gd, self.n[k], w["Wg"][k], w["Wu"][k], self.p[k], self.gws)
            L.lp_step_forward(self.st, self.p[k], w["Wd"][k], None, u, self.u[k], self.sws)
        g = self.grads
        L.lp_loss_labels(self.head, self.u[-1], w["HW"], None, labels, self.J, self.hws, du=self.lam[-1], dW=g["HW"])
        for k in reversed(range(self.layers)):
            u = x if k == 0 else self.u[k - 1]
            L.lp_step_backward(self.st, self.p[k], w["Wd"][k], None, self.lam[k + 1], self.dp[k], g["Wd"][k], None, self.sws)
            L.lp_gated_backward(self.gd, self.n[k], w["Wg"][k], w["Wu"][k], self.dp[k], self.dn[k], g["Wg"][k], g["Wu"][k], self.gws)
            L.lp_norm_backward(self.nd, u, w["gamma"][k], self.dn[k], self.lam[k + 1], self.lam[k], g["gamma"][k], g["beta"][k], self.nws)
        for k, o in self.ups.items():
            L.lp_orth_update(o, g[k], mom[k], mom[k], w[k], w[k], self.ows[k], alpha=ALPHA, beta=KEEP)


def inputs(dtype, B, q, m, layers, nc, seed):
    g = torch.Generator().manual_seed(seed)
    w = {"gamma": (1 + T.draw(g, (layers, q), "f32", 0.2)).to(T.DT[dtype]), "beta": T.draw(g, (layers, q), dtype, 0.1),
         "Wg": T.draw(g, (layers, m, q), dtype, 1 / math.sqrt(q)), "Wu": T.draw(g, (layers, m, q), dtype, 1 / math.sqrt(q)),
         "Wd": T.draw(g, (layers, q, m), dtype, 1 / math.sqrt(m)), "HW": T.draw(g, (nc, q), dtype, 1 / math.sqrt(q))}
    return T.draw(g, (B, q), dtype), w, torch.randint(0, nc, (B,), generator=g)


def momenta(w):
    return {k: torch.zeros(w[k].shape, dtype=torch.float32, device="cuda") for k in ("Wg", "Wu", "Wd")}


SHAPE = (70, 48, 100, 3, 50)
# a value's rounding, twice a block each way (the stream itself and what is added to it), and the sums' own in fp32
ROUNDINGS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -20}


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_training_step(dtype, act):
    B, q, m, layers, nc = SHAPE
    x, w, labels = inputs(dtype, *SHAPE, seed=1)
    net = Network(dtype, act, *SHAPE)
    before = {k: v.cuda() for k, v in w.items()}
    after, mom = {k: v.clone() for k, v in before.items()}, momenta(w)
    net.run(x.cuda(), after, labels.cuda(), mom)
    torch.cuda.synchronize()
    c = lambda t: t.cpu()
    for k in range(layers):
        u = x if k == 0 else c(net.u[k - 1])
        n, p, lam, dp, dn = c(net.n[k]), c(net.p[k]), c(net.lam[k + 1]), c(net.dp[k]), c(net.dn[k])
        T.check(n, *K.norm_forward(u, w["gamma"][k], w["beta"][k], EPS, dtype), f"n {k}")
        T.check(p, *K.gated_forward(n, w["Wg"][k], w["Wu"][k], act, dtype), f"p {k}")
        T.check(net.u[k], *T.forward(p, w["Wd"][k], None, u, "identity", H, dtype), f"u {k}")
        for name, a, (r, e) in zip(("dp", "dWd"), (net.dp[k], net.grads["Wd"][k]), T.backward(p, w["Wd"][k], None, lam, "identity", H, False, dtype)):
            T.check(a, r, e, f"{name} {k}")
        got = (net.dn[k], net.grads["Wg"][k], net.grads["Wu"][k])
        for name, a, (r, e) in zip(("dn", "dWg", "dWu"), got, K.gated_backward(n, w["Wg"][k], w["Wu"][k], dp, act, dtype)):
            T.check(a, r, e, f"{name} {k}")
        got = (net.lam[k], net.grads["gamma"][k], net.grads["beta"][k])
        for name, a, (r, e) in zip(("lam", "dgamma", "dbeta"), got, K.norm_backward(u, w["gamma"][k], dn, lam, EPS, dtype)):
            T.check(a, r, e, f"{name} {k}")
    for k in ("Wg", "Wu", "Wd"):
        g = net.grads[k].cpu()
        want, v = K.momentum(g, torch.zeros(g.shape), MU, True, dtype)
        T.check(mom[k], want, 2 * K.E32 * want.abs(), f"momentum {k}")
        K.orth_check(after[k], v.cuda(), before[k], 5, L.QUINTIC, 1e-7, ALPHA, KEEP, dtype, k)

    # the whole in 64 bits
    d = {k: v.double().requires_grad_() for k, v in w.items()}
    s = x.double().requires_grad_()
    u = s
    for k in range(layers):
        xc = u - u.mean(1, keepdim=True)
        n = xc / ((xc * xc).mean(1, keepdim=True) + EPS).sqrt() * d["gamma"][k] + d["beta"][k]
        z = n @ d["Wg"][k].t()
        a = z * torch.sigmoid(z) if act == "silu" else 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
        u = u + H * (a * (n @ d["Wu"][k].t())) @ d["Wd"][k].t()
    J = torch.nn.functional.cross_entropy(u @ d["HW"].t(), labels)
    J.backward()
    # errors in norm: at most ROUNDINGS for each of the up to 8 roundings a block and way that lie one behind the
    # other, stretched by the head's softmax and the norms, whose slopes are of the order of one here
    most = 2 * (8 * layers + 4) * ROUNDINGS[dtype]
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert abs(net.J.item() - J.item()) <= most * abs(J.item())
    assert rel(net.lam[0], s.grad) <= most
    for k, v in net.grads.items():
        assert rel(v, d[k].grad) <= most, k


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_captured_training_steps(dtype):
    """Three steps replayed from a graph, each updating the weights in place, give the eager steps' bits; eager work of
    another network runs between them."""
    x, w, labels = inputs(dtype, *SHAPE, seed=2)
    x, labels = x.cuda(), labels.cuda()
    net, other = Network(dtype, "silu", *SHAPE), Network(dtype, "silu", *SHAPE)
    a, b = ({k: v.cuda() for k, v in w.items()} for _ in range(2))
    ma, mb = momenta(w), momenta(w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        net.run(x, a, labels, ma)
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.run(x, a, labels, ma)
    other.run(x, b, labels, mb)
    losses = []
    for _ in range(3):
        graph.replay()
        other.run(x, b, labels, mb)
        torch.cuda.synchronize()
        losses.append((net.J.item(), other.J.item()))
        assert losses[-1][0] == losses[-1][1]
        for k in a:
            assert torch.equal(a[k], b[k]), k
        for k in ma:
            assert torch.equal(ma[k], mb[k]), k
