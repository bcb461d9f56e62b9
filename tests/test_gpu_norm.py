"""Layer norm and its gradients against 64-bit plain forms, at the sizes, types and values where they can
go wrong. Bounds: tests/block_testutil.py."""
import math

import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
# a value, odd widths, every width of group and its limits, rows that no group holds; one row to many workgroups
SHAPES = [(1, 1), (3, 2), (2, 3), (1, 7), (5, 33), (70, 64), (33, 65), (1000, 220), (129, 255), (40, 257), (17, 511), (9, 512),
          (300, 513), (1, 4096), (65, 1025), (1500, 1111), (1100, 2048), (37, 2050), (1029, 4096), (21, 4100), (3, 8192), (5, 8200),
          (6, 16384), (11, 16390), (2, 32769), (3, 65536), (2, 65540), (70, 70001), (5000, 20), (20011, 8)]


def inputs(seed, dtype, B, q):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, q), generator=g, dtype=torch.float64) * torch.randn((B, 1), generator=g, dtype=torch.float64).exp()
    x = (x + 2 * torch.randn((B, 1), generator=g, dtype=torch.float64)).to(T.DT[dtype])
    return (x, (1 + T.draw(g, (q,), "f32", 0.3)).to(T.DT[dtype]), T.draw(g, (q,), dtype, 0.5), T.draw(g, (B, q), dtype, 0.1),
            T.draw(g, (B, q), dtype, 0.1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(dtype, i):
    B, q = SHAPES[i]
    x, gamma, beta, _, _ = inputs(i, dtype, B, q)
    if i % 5 == 3:
        gamma = None
    if i % 7 == 4:
        beta = None
    s = K.Norm(dtype, B, q)
    y = s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta))
    T.check(y, *K.norm_forward(x, gamma, beta, 1e-5, dtype), "y")
    # the same bits on wider alignment, and in place
    z = x.cuda()
    L.lp_norm_forward(s.nd, z, None if gamma is None else gamma.cuda(), None if beta is None else beta.cuda(), z)
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(dtype, i):
    B, q = SHAPES[i]
    x, gamma, _, dy, dr = inputs(100 + i, dtype, B, q)
    if i % 5 == 2:
        gamma = None
    if i % 2:
        dr = None
    s = K.Norm(dtype, B, q)
    got = s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), T.gpu(dr))
    for name, a, (r, e) in zip(("dx", "dgamma", "dbeta"), got, K.norm_backward(x, gamma, dy, dr, 1e-5, dtype)):
        T.check(a, r, e, name)
    again = s.backward(x.cuda(), None if gamma is None else gamma.cuda(), dy.cuda(), None if dr is None else dr.cuda())
    for a, b in zip(got, again):
        assert torch.equal(a, b)
    if dr is not None:  # dr's own array takes dx
        z = T.gpu(dr)
        L.lp_norm_backward(s.nd, T.gpu(x), T.gpu(gamma), T.gpu(dy), z, z, None, None, K.scribble(L.alloc_norm_workspace(s.nd)))
        assert torch.equal(z, got[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("q", [100, 3000, 70001])
def test_wanted_gradients_alone(dtype, q):
    B = 50
    x, gamma, _, dy, dr = (T.gpu(t) for t in inputs(13, dtype, B, q))
    s = K.Norm(dtype, B, q)
    full = s.backward(x, gamma, dy, dr)
    for want in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (False, False, False)):
        for a, f, w in zip(s.backward(x, gamma, dy, dr, want), full, want):
            assert (a is None) if not w else torch.equal(a, f)


@pytest.mark.parametrize("dtype", DTYPES)
def test_empty_batch(dtype):
    for q in (33, 70001):
        s = K.Norm(dtype, 0, q)
        e = torch.empty((0, q), dtype=T.DT[dtype], device="cuda")
        assert s.forward(e, None, None).numel() == 0
        dx, dgamma, dbeta = s.backward(e, None, e, None)
        assert dx.numel() == 0 and not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_far_from_zero(dtype):
    """A mean far larger than the spread (the mean square minus the squared mean would leave nothing of it),
    rows of equal values, and infinities and NaN, which stay in their row."""
    B, q = 40, 600
    x, gamma, beta, dy, _ = inputs(5, dtype, B, q)
    far = 100.0 if dtype == "bf16" else 1000.0
    x[4] = (far + 4 * torch.randn(q, generator=torch.Generator().manual_seed(6))).to(x.dtype)
    x[6] = 3.0
    x[11, 5] = math.nan
    x[13, 599] = math.inf
    clean = torch.ones(B, dtype=torch.bool)
    clean[[11, 13]] = False
    s = K.Norm(dtype, B, q)
    y = s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)).cpu()
    T.check(y[clean], *K.norm_forward(x[clean], gamma, beta, 1e-5, dtype), "y")
    assert torch.isnan(y[~clean]).all() and torch.equal(y[6], beta)
    dx = s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), None)[0].cpu()
    T.check(dx[clean], *K.norm_backward(x[clean], gamma, dy[clean], None, 1e-5, dtype)[0], "dx")
    assert torch.isnan(dx[~clean]).all()


def test_gradients_are_differences():
    """The formula's gradients against central differences of the 64-bit form, through the library in fp32."""
    B, q, h = 4, 9, 1e-6
    x, gamma, beta, dy, _ = inputs(19, "f32", B, q)
    x = (x.double() * 0.3 + torch.randn((B, q), generator=torch.Generator().manual_seed(3), dtype=torch.float64)).float()
    got = K.Norm("f32", B, q).backward(*(T.gpu(t) for t in (x, gamma, dy)), None)

    def value(x, gamma, beta):
        return float(((K.norm_stats(x, 1e-5)[0] * gamma + beta) * dy.double()).sum())

    args = [t.double() for t in (x, gamma, beta)]
    for k, name in enumerate(("dx", "dgamma", "dbeta")):
        d = torch.zeros(args[k].shape, dtype=torch.float64)
        for j in range(d.numel()):
            v = []
            for sign in (1, -1):
                m = [t.clone() for t in args]
                m[k].view(-1)[j] += sign * h
                v.append(value(*m))
            d.view(-1)[j] = (v[0] - v[1]) / (2 * h)
        T.check(got[k], d, torch.full_like(d, 1e-5), name)


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured(dtype):
    """A graph's replays give the eager results, on new inputs too, with eager calls between them."""
    for B, q in ((300, 130), (2000, 1500), (40, 70001)):
        x, gamma, beta, dy, dr = (t.cuda() for t in inputs(23, dtype, B, q))
        nd = L.norm(dtype, B, q)
        ws = K.scribble(L.alloc_norm_workspace(nd))
        outs = [torch.empty_like(t) for t in (x, x, gamma, gamma)]

        def calls():
            L.lp_norm_forward(nd, x, gamma, beta, outs[0])
            L.lp_norm_backward(nd, x, gamma, dy, dr, *outs[1:], ws)

        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            calls()
        torch.cuda.current_stream().wait_stream(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for seed in (24, 25, 26):
            for t, v in zip((x, gamma, beta, dy, dr), inputs(seed, dtype, B, q)):
                t.copy_(v)
            calls()
            want = [t.clone() for t in outs]
            for t in outs:
                t.zero_()
            K.scribble(ws)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


# every way a row is held: lanes of a wave, waves, several pieces a thread, read again for each pass
WIDTHS = [3, 20, 223, 257, 1111, 3000, 4096, 7001, 9000, 16384, 20001, 70001]


@pytest.mark.parametrize("q", WIDTHS)
def test_rows_of_equal_values(q):
    """A sum of q equal values is rounded and so is its mean: what it is off by must not pass for a spread."""
    values = [0.1, 0.7, 3.3, 3.3e3, -1.1e-3, 12345.678]
    g = torch.Generator().manual_seed(q)
    x = torch.tensor(values).repeat(5)[:, None].repeat(1, q)
    gamma, beta = 1 + T.draw(g, (q,), "f32", 0.3), T.draw(g, (q,), "f32", 0.5)
    dy, dr = T.draw(g, x.shape, "f32", 0.1), T.draw(g, x.shape, "f32", 0.1)
    s = K.Norm("f32", *x.shape)
    assert torch.equal(s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)).cpu(), beta.expand(x.shape))
    dx, dgamma, dbeta = s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), T.gpu(dr))
    assert not dgamma.any()
    (r, e), _, (rb, eb) = K.norm_backward(x, gamma, dy, dr, 1e-5, "f32")
    ga = (dy * gamma).double()  # dx = (g - mean g) / sqrt(eps) + dr
    e = 400 * (84 + q / 1024) * K.E32 * (ga.abs().mean(1, keepdim=True) + ga.abs()) + 2 * K.E32 * dr.abs()
    T.check(dx, r, e, "dx")
    T.check(dbeta, rb, eb, "dbeta")


@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("q", WIDTHS)
def test_means_far_beyond_the_spread(q, B, monkeypatch):
    """Rows whose mean is 10^3 to 10^5 times their spread: held to a bound without the mean."""
    monkeypatch.setattr(K, "norm_stats", K.norm_stats_sharp)
    _, gamma, beta, dy, dr = inputs(q, "f32", B, q)
    g = torch.Generator().manual_seed(q)
    x = (torch.randn((B, q), generator=g) + torch.tensor([1e3, 1e4, -1e5, 3e4, 0.0])[torch.arange(B) % 5][:, None]).float()
    s = K.Norm("f32", B, q)
    T.check(s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)), *K.norm_forward(x, gamma, beta, 1e-5, "f32"), "y")
    got = s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), T.gpu(dr))
    for name, a, (r, e) in zip(("dx", "dgamma", "dbeta"), got, K.norm_backward(x, gamma, dy, dr, 1e-5, "f32")):
        T.check(a, r, e, name)


@pytest.mark.parametrize("dtype", DTYPES)
def test_equal_values_without_eps(dtype):
    """No spread and nothing added to it: NaN, and in the other rows nothing of it."""
    B, q = 12, 223
    x, gamma, beta, dy, _ = inputs(3, dtype, B, q)
    x = (torch.randn((B, q), generator=torch.Generator().manual_seed(4)) * 0.5).to(x.dtype)
    for i, v in ((1, 0.1), (4, 0.7), (7, 3.3), (11, 0.0)):
        x[i] = v
    rows = torch.ones(B, dtype=torch.bool)
    rows[[1, 4, 7, 11]] = False
    s = K.Norm(dtype, B, q, eps=0.0)
    y = s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)).cpu()
    assert torch.isnan(y[~rows]).all()
    T.check(y[rows], *K.norm_forward(x[rows], gamma, beta, 0.0, dtype), "y")
    dx = s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), None)[0].cpu()
    assert torch.isnan(dx[~rows]).all()
    T.check(dx[rows], *K.norm_backward(x[rows], gamma, dy[rows], None, 0.0, dtype)[0], "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q", WIDTHS)
def test_rows_of_equal_16_bit_values(q, dtype):
    """And rows of which a value or two differ by the last place, the least spread that the type has."""
    g = torch.Generator().manual_seed(q)
    x = torch.tensor([0.1, 0.7, 3.3, 3.3e3, -1.1e-3, 12345.678]).repeat(5)[:, None].repeat(1, q).to(T.DT[dtype])
    gamma, beta = (1 + T.draw(g, (q,), "f32", 0.3)).to(x.dtype), T.draw(g, (q,), dtype, 0.5)
    dy = T.draw(g, x.shape, dtype, 0.1)
    s = K.Norm(dtype, *x.shape)
    assert torch.equal(s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)).cpu(), beta.expand(x.shape))
    assert not s.backward(T.gpu(x), T.gpu(gamma), T.gpu(dy), None)[1].any()
    step = (x.double().abs().log2().floor().exp2() * torch.finfo(x.dtype).eps).to(x.dtype)
    x[:, 0] += step[:, 0]
    x[3:, q // 2] -= step[3:, 0]
    xd = x.double()
    d = xd - xd.mean(1, keepdim=True)
    rstd = ((d * d).mean(1, keepdim=True) + 1e-5) ** -0.5
    ref = d * rstd * gamma.double() + beta.double()
    # bf16 rows that a group holds (2^15 values forward): off by half an fp32 step of the mean; else by what sums of x - mean
    # are; fp32 steps of the values, the type's half step
    off = 2.0 ** -24 * xd.mean(1, keepdim=True).abs() if dtype == "bf16" and q <= 1 << 15 else 0.0
    n = 84 + q / 1024
    err = (off + (n + 2) * K.E32 * (d.abs().mean(1, keepdim=True) + d.abs())) * rstd * gamma.double().abs() + n * K.E32 * (ref.abs() + beta.double().abs())
    T.check(s.forward(T.gpu(x), T.gpu(gamma), T.gpu(beta)), ref, err + T.half_step(dtype) * (ref.abs() + err) + T.tiny(dtype), "y")
