"""Gated layers and their gradients against 64-bit plain forms, at the sizes, types and values where they
can go wrong. Bounds: tests/block_testutil.py."""
import math

import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
# one row to ragged tiles; widths of one value, odd ones, below, at and above blocks, tiles and stages
SHAPES = [(1, 1, 1), (1, 64, 64), (2, 7, 5), (1, 4096, 203), (1, 40, 9000), (5, 33, 1000), (16, 512, 48), (31, 256, 96),
          (64, 64, 128), (129, 130, 131), (200, 63, 257), (256, 192, 320), (300, 220, 587), (17, 1000, 33), (40, 8, 2050),
          (513, 96, 64), (1000, 24, 40), (24, 2048, 160), (70, 6000, 72)]


def inputs(seed, dtype, B, ni, no):
    g = torch.Generator().manual_seed(seed)
    return (T.draw(g, (B, ni), dtype), T.draw(g, (no, ni), dtype, 1.5 / math.sqrt(ni)), T.draw(g, (no, ni), dtype, 1 / math.sqrt(ni)),
            T.draw(g, (B, no), dtype, 0.1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(dtype, i):
    B, ni, no = SHAPES[i]
    act = K.ACTS[(i + len(dtype)) % 6]
    x, Wg, Wu, _ = inputs(i, dtype, B, ni, no)
    s = K.Gated(dtype, act, B, ni, no)
    y = s.forward(T.gpu(x), T.gpu(Wg), T.gpu(Wu))
    T.check(y, *K.gated_forward(x, Wg, Wu, act, dtype), f"y {act}")
    # rows on 16 bytes where the width allows it: the same bits
    assert torch.equal(s.forward(x.cuda(), Wg.cuda(), Wu.cuda()), y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(dtype, i):
    B, ni, no = SHAPES[i]
    act = K.ACTS[(i + len(dtype) + 1) % 6]
    x, Wg, Wu, dy = inputs(50 + i, dtype, B, ni, no)
    s = K.Gated(dtype, act, B, ni, no)
    got = s.backward(T.gpu(x), T.gpu(Wg), T.gpu(Wu), T.gpu(dy))
    for name, a, (r, e) in zip(("dx", "dWg", "dWu"), got, K.gated_backward(x, Wg, Wu, dy, act, dtype)):
        T.check(a, r, e, f"{name} {act}")
    for a, b in zip(got, s.backward(x.cuda(), Wg.cuda(), Wu.cuda(), dy.cuda())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("act", K.ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_gate(dtype, act):
    B, ni, no = 70, 40, 100
    x, Wg, Wu, dy = inputs(7, dtype, B, ni, no)
    Wg = (Wg.double() * 4).to(Wg.dtype)  # gates up to 20 or so either way
    s = K.Gated(dtype, act, B, ni, no)
    T.check(s.forward(T.gpu(x), T.gpu(Wg), T.gpu(Wu)), *K.gated_forward(x, Wg, Wu, act, dtype), "y")
    got = s.backward(T.gpu(x), T.gpu(Wg), T.gpu(Wu), T.gpu(dy))
    for name, a, (r, e) in zip(("dx", "dWg", "dWu"), got, K.gated_backward(x, Wg, Wu, dy, act, dtype)):
        T.check(a, r, e, name)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_tiles(dtype):
    """Sizes that take the largest tiles, whole and ragged ones."""
    for B, ni, no in ((4096, 128, 2048), (3001, 72, 4100)):
        x, Wg, Wu, dy = inputs(11, dtype, B, ni, no)
        s = K.Gated(dtype, "silu", B, ni, no)
        T.check(s.forward(T.gpu(x), T.gpu(Wg), T.gpu(Wu)), *K.gated_forward(x, Wg, Wu, "silu", dtype), "y")
        got = s.backward(T.gpu(x), T.gpu(Wg), T.gpu(Wu), T.gpu(dy))
        for name, a, (r, e) in zip(("dx", "dWg", "dWu"), got, K.gated_backward(x, Wg, Wu, dy, "silu", dtype)):
            T.check(a, r, e, f"{name} {B} {ni} {no}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_wanted_gradients_alone(dtype):
    B, ni, no = 90, 70, 100
    x, Wg, Wu, dy = (T.gpu(t) for t in inputs(13, dtype, B, ni, no))
    s = K.Gated(dtype, "gelu", B, ni, no)
    full = s.backward(x, Wg, Wu, dy)
    for want in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, False, False)):
        for a, f, w in zip(s.backward(x, Wg, Wu, dy, want), full, want):
            assert (a is None) if not w else torch.equal(a, f)


@pytest.mark.parametrize("dtype", DTYPES)
def test_empty_batch(dtype):
    ni, no = 33, 65
    g = torch.Generator().manual_seed(1)
    Wg, Wu = (T.gpu(T.draw(g, (no, ni), dtype)) for _ in range(2))
    s = K.Gated(dtype, "silu", 0, ni, no)
    x, y = (torch.empty((0, n), dtype=T.DT[dtype], device="cuda") for n in (ni, no))
    assert s.forward(x, Wg, Wu).numel() == 0
    dx, dWg, dWu = s.backward(x, Wg, Wu, y)
    assert dx.numel() == 0 and not dWg.any() and not dWu.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_extreme_gates(dtype):
    """Gates far out on either side, infinities and NaN stay in their row."""
    B, ni, no = 40, 16, 48
    for act in K.ACTS:
        x, Wg, Wu, dy = inputs(17, dtype, B, ni, no)
        x[3] *= 100
        x[7, 2] = math.nan
        x[9, 1] = math.inf
        s = K.Gated(dtype, act, B, ni, no)
        y = s.forward(T.gpu(x), T.gpu(Wg), T.gpu(Wu)).cpu()
        clean = torch.ones(B, dtype=torch.bool)
        clean[[7, 9]] = False
        ref, bound = K.gated_forward(x[clean], Wg, Wu, act, dtype)
        T.check(y[clean], ref, bound, act)
        assert torch.isnan(y[7]).all(), act
        dx = s.backward(T.gpu(x), T.gpu(Wg), T.gpu(Wu), T.gpu(dy))[0].cpu()
        T.check(dx[clean], *K.gated_backward(x[clean], Wg, Wu, dy[clean], act, dtype)[0], act)
        assert torch.isnan(dx[7]).all(), act


def test_gradients_are_differences():
    """The formula's gradients against central differences, through the library in fp32."""
    B, ni, no = 5, 6, 7
    for act in K.ACTS:
        x, Wg, Wu, dy = inputs(19, "f32", B, ni, no)
        s = K.Gated("f32", act, B, ni, no)
        got = s.backward(*(T.gpu(t) for t in (x, Wg, Wu, dy)))
        h = 1e-6
        for name, arr, grad in (("dx", x, got[0]), ("dWg", Wg, got[1]), ("dWu", Wu, got[2])):
            d = torch.zeros(arr.shape, dtype=torch.float64)
            for j in range(arr.numel()):
                vals = []
                for sign in (1, -1):
                    m = arr.double().clone()
                    m.view(-1)[j] += sign * h
                    a = [m if arr is t else t.double() for t in (x, Wg, Wu)]
                    vals.append(float((K.gate(a[0] @ a[1].t(), act)[0] * (a[0] @ a[2].t()) * dy.double()).sum()))
                d.view(-1)[j] = (vals[0] - vals[1]) / (2 * h)
            # differences are off by h^2 and 2^-52 / h of values of order 1; a bend of an activation
            # within h of a gate is not met by these inputs
            T.check(grad, d, torch.full_like(d, 1e-5), f"{name} {act}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_on_another_stream(dtype):
    """Calls on a side stream and their graph's replays give the eager results, on new inputs too."""
    B, ni, no = 300, 130, 200
    x, Wg, Wu, dy = (t.cuda() for t in inputs(23, dtype, B, ni, no))
    gd = L.gated(dtype, "silu", B, ni, no)
    ws = K.scribble(L.alloc_gated_workspace(gd))
    y, dx, dWg, dWu = (torch.empty_like(t) for t in (dy, x, Wg, Wu))

    def calls():
        L.lp_gated_forward(gd, x, Wg, Wu, y, ws)
        L.lp_gated_backward(gd, x, Wg, Wu, dy, dx, dWg, dWu, ws)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        calls()
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (24, 25, 26):
        for t, v in zip((x, Wg, Wu, dy), inputs(seed, dtype, B, ni, no)):
            t.copy_(v)
        calls()
        want = [t.clone() for t in (y, dx, dWg, dWu)]
        for t in (y, dx, dWg, dWu):
            t.zero_()
        K.scribble(ws)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, dx, dWg, dWu), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(1000, 220, 587), (209, 649, 649), (320, 60, 384), (2000, 256, 700), (600, 512, 1024), (40, 3000, 500), (700, 200, 400), (4600, 200, 700)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_bits_do_not_depend_on_what_else_is_wanted(dtype, shape):
    """Sizes whose gradients come from one launch where both sides are wanted, and others."""
    x, Wg, Wu, dy = (T.gpu(t) for t in inputs(29, dtype, *shape))
    s = K.Gated(dtype, "silu", *shape)
    full = s.backward(x, Wg, Wu, dy)
    for want in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True)):
        for a, f, w in zip(s.backward(x, Wg, Wu, dy, want), full, want):
            assert (a is None) if not w else torch.equal(a, f), want
