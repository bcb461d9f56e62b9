"""Orthogonalised updates against the iteration in 64 bits, at the sizes, types and values where they can go
wrong. Bounds: tests/block_testutil.py."""
import math

import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
Q = L.QUINTIC
# single values, rows and columns; wide, square and tall; odd sizes; below, at and above tiles; long sides that are split
SHAPES = [(1, 1, 1), (3, 1, 5), (2, 7, 1), (4, 8, 8), (7, 21, 36), (5, 36, 21), (3, 64, 64), (2, 65, 63), (5, 33, 130), (2, 220, 220),
          (1, 300, 1000), (1, 1000, 70), (2, 129, 257), (1, 64, 4096), (1, 4096, 40), (1, 8, 5000), (1, 520, 520), (1, 1100, 1100),
          (40, 100, 90), (9, 64, 256), (3, 256, 33), (5, 17, 129), (2, 65, 256), (3, 257, 20), (300, 3, 2)]


def gradients(seed, dtype, N, no, ni):
    """Noise and a few strong directions, on the CPU."""
    g = torch.Generator().manual_seed(seed)
    k = min(4, no, ni)
    v = torch.randn((N, no, ni), generator=g, dtype=torch.float64)
    v = v + torch.matmul(torch.randn((N, no, k), generator=g, dtype=torch.float64), torch.randn((N, k, ni), generator=g, dtype=torch.float64))
    return (v * 0.01 * torch.randn((N, 1, 1), generator=g, dtype=torch.float64).exp()).to(T.DT[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_update(dtype, i):
    N, no, ni = SHAPES[i]
    steps, nesterov = (5, 1, 2, 3)[i % 4], i % 2 == 0
    mu, alpha, beta = 0.9, -0.05, 0.99
    g, m = gradients(i, dtype, N, no, ni), gradients(50 + i, "f32", N, no, ni)
    r = T.draw(torch.Generator().manual_seed(i), (N, no, ni), dtype, 0.1)
    if i % 3 == 2:
        m = None
    s = K.Orth(dtype, N, no, ni, steps=steps, mu=mu, nesterov=nesterov)
    mo, mf = T.out((N, no, ni), torch.float32)
    W = s(T.gpu(g), T.gpu(m), mo, T.gpu(r), alpha, beta)
    assert T.guarded(mf, mo.numel())
    want, v = K.momentum(g, m, mu, nesterov, dtype)
    T.check(mo, want, 2 * K.E32 * (want.abs() + (0 if m is None else m.abs())) + T.tiny("f32"), "m'")
    K.orth_check(W, v.cuda(), r, steps, Q, 1e-7, alpha, beta, dtype, f"W {steps}")
    # other alignments, the momentum and the weights in place: the same bits
    m2 = torch.zeros_like(mo) if m is None else m.cuda()
    W2 = r.cuda()
    L.lp_orth_update(s.od, g.cuda(), None if m is None else m2, m2, W2, W2, K.scribble(L.alloc_orth_workspace(s.od)), alpha=alpha, beta=beta)
    assert torch.equal(m2, mo) and torch.equal(W2, W)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(3, 40, 70), (2, 200, 130)])
def test_plain_orthogonalisation(dtype, shape):
    """Without momentum and weights: O itself, singular values about one; with the converging coefficients an
    orthogonal matrix."""
    g = gradients(3, dtype, *shape)
    W = K.Orth(dtype, *shape)(T.gpu(g), None, None, None, 1.0)
    K.orth_check(W, g.double().cuda(), None, 5, Q, 1e-7, 1.0, 0.0, dtype, "O")
    sv = torch.linalg.svdvals(W.double())
    assert 0.6 < sv.min() and sv.max() < 1.3
    # 15/8, -10/8, 3/8: s -> 1 cubically; growth by 15/8 a step from 1/40 of the norm at least
    W = K.Orth(dtype, *shape, steps=14, coeffs=(15 / 8, -10 / 8, 3 / 8))(T.gpu(g), None, None, None, 1.0).double()
    A = torch.matmul(W, W.transpose(1, 2).contiguous()) if shape[1] <= shape[2] else torch.matmul(W.transpose(1, 2).contiguous(), W)
    off = (A - torch.eye(A.shape[1], dtype=torch.float64, device="cuda")).abs().max()
    # (W's own rounding, 2 u sqrt(1 / n) sqrt(n) at most an element, and the last product's of about the same size)
    assert off <= 8 * T.half_step("f16" if dtype == "f16" else dtype) + 2e-5, off


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 2304, 2048), (1, 2048, 2304), (1, 4096, 512), (1, 1500, 1600), (3, 1000, 1008)])
def test_large(dtype, shape):
    g = gradients(5, dtype, *shape)
    s = K.Orth(dtype, *shape)
    W = s(g.cuda(), None, None, None, 1.0)
    K.orth_check(W, g.cuda().double(), None, 5, Q, 1e-7, 1.0, 0.0, dtype, "O")


@pytest.mark.parametrize("dtype", DTYPES)
def test_batches_of_several_chunks(dtype):
    """More matrices than the workspace holds at once; each is treated by itself."""
    N, no, ni = (6100, 250, 66) if dtype == "f32" else (12200, 250, 66)
    g = gradients(6, dtype, 64, no, ni)
    s = K.Orth(dtype, N, no, ni, steps=3)
    assert L.lp_orth_workspace_bytes(L.orth(dtype, 2 * N, no, ni)) < 1.1 * L.lp_orth_workspace_bytes(s.od)
    one = K.Orth(dtype, 64, no, ni, steps=3)
    few = g.cuda()
    W = s(few.repeat(-(-N // 64), 1, 1)[:N].contiguous(), None, None, None, 1.0)
    ref = one(few, None, None, None, 1.0)
    K.orth_check(ref, g.double().cuda(), None, 3, Q, 1e-7, 1.0, 0.0, dtype, "O")
    # (another plan of products: the same values but for the order of sums)
    K.orth_check(W[-70:], g.double().repeat(3, 1, 1)[(N - 70) % 64:][:70].cuda(), None, 3, Q, 1e-7, 1.0, 0.0, dtype, "last")
    for z in range(0, N - 64, 64):
        assert torch.equal(W[z:z + 64], W[:64]), z


@pytest.mark.parametrize("dtype", DTYPES)
def test_zeros_scales_and_not_finite(dtype):
    """A matrix of zeros has none to give; a tiny, a huge and an ordinary one of the same directions give the same; NaN
    and infinity stay in their matrix."""
    no, ni = 30, 50
    g = gradients(8, dtype, 1, no, ni)[0].double()
    g = g / g.abs().max()
    small, large = (2.0 ** -10, 2.0 ** 14) if dtype == "f16" else (2.0 ** -60, 2.0 ** 100)
    batch = torch.stack([g, g * 0, g * small, g * large, g, g]).to(T.DT[dtype])
    batch[4, 3, 7] = math.nan
    batch[5, 0, 0] = math.inf
    W = K.Orth(dtype, 6, no, ni, eps=1e-30)(batch.cuda(), None, None, None, 1.0)
    assert not W[1].any() and torch.isnan(W[4]).all() and torch.isnan(W[5]).all()
    v = batch[[0, 2, 3]].double().cuda()
    K.orth_check(W[[0, 2, 3]], v, None, 5, Q, 1e-30, 1.0, 0.0, dtype, "scales")


@pytest.mark.parametrize("dtype", DTYPES)
def test_nothing_to_do(dtype):
    s = K.Orth(dtype, 0, 4, 5)
    e = torch.empty((0, 4, 5), dtype=T.DT[dtype], device="cuda")
    assert s(e, None, None, None, 1.0).numel() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured(dtype):
    """A graph's replays give the eager results, on new inputs too, with eager calls between them."""
    for shape in ((6, 64, 64), (2, 300, 700), (1, 40, 3000)):
        g, m = gradients(1, dtype, *shape).cuda(), gradients(2, "f32", *shape).cuda()
        r = T.draw(torch.Generator().manual_seed(3), shape, dtype).cuda()
        od = L.orth(dtype, *shape, mu=0.9, nesterov=True)
        ws = K.scribble(L.alloc_orth_workspace(od))
        mo, W = torch.empty_like(m), torch.empty_like(r)

        def calls():
            L.lp_orth_update(od, g, m, mo, r, W, ws, alpha=-0.1, beta=0.9)

        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            calls()
        torch.cuda.current_stream().wait_stream(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for seed in (24, 25, 26):
            g.copy_(gradients(seed, dtype, *shape))
            calls()
            want = mo.clone(), W.clone()
            mo.zero_(), W.zero_()
            K.scribble(ws)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(mo, want[0]) and torch.equal(W, want[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(70, 8, 5000), (67, 5000, 8), (130, 70, 1500), (64, 300, 20)])
def test_large_batches_of_long_matrices(dtype, shape):
    """Batches whose matrices are spread over the XCDs, with contractions that are split."""
    g, m = gradients(9, dtype, *shape), gradients(10, "f32", *shape)
    r = T.draw(torch.Generator().manual_seed(2), shape, dtype, 0.1)
    s = K.Orth(dtype, *shape, mu=0.9, nesterov=True)
    mo, mf = T.out(shape, torch.float32)
    W = s(T.gpu(g), T.gpu(m), mo, T.gpu(r), -0.05, 0.99)
    assert T.guarded(mf, mo.numel())
    _, v = K.momentum(g, m, 0.9, True, dtype)
    K.orth_check(W, v.cuda(), r, 5, Q, 1e-7, -0.05, 0.99, dtype, f"W {shape}")
