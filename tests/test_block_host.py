"""Refusals of the layer norm, the gated layers and the orthogonalised updates on the host (no GPU): every bad call returns its documented status before
any device work, the binding refuses bad tensors, and workspaces hold what they have to."""
import ctypes
import random

import pytest
import torch

from paper_1812_04352_amd import lp as L

FAKE = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(16)]  # never dereferenced
BIG = 1 << 50
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def gated(dtype="bf16", act="silu", B=8, ni=16, no=24):
    return L.gated(dtype, act, B, ni, no)


def forward(gd, x=FAKE[0], Wg=FAKE[1], Wu=FAKE[2], y=FAKE[3], ws=FAKE[4], n=BIG):
    return L.load().lp_gated_forward(ctypes.byref(gd) if gd else None, x, Wg, Wu, y, ws, n, None)


def backward(gd, x=FAKE[0], Wg=FAKE[1], Wu=FAKE[2], dy=FAKE[3], dx=FAKE[4], dWg=FAKE[5], dWu=FAKE[6], ws=FAKE[7], n=BIG):
    return L.load().lp_gated_backward(ctypes.byref(gd) if gd else None, x, Wg, Wu, dy, dx, dWg, dWu, ws, n, None)


def bad_workspaces(need):
    return (dict(ws=None), dict(ws=ctypes.c_void_p(0x1010)), dict(n=need - 1))


def test_gated_descriptor():
    assert forward(None) == L.LP_EINVAL and backward(None) == L.LP_EINVAL
    for call in (forward, backward):
        for kw in (dict(B=-1), dict(ni=0), dict(no=-3)):
            assert call(gated(**kw)) == L.LP_EINVAL, kw
        for kw in (dict(dtype="f64"), dict(B=(1 << 24) + 1), dict(ni=(1 << 20) + 1), dict(no=(1 << 20) + 1),
                   dict(B=1 << 24, ni=1 << 12), dict(ni=1 << 18, no=(1 << 17) + 1)):
            assert call(gated(**kw)) == L.LP_EUNSUPPORTED, kw
        for field, value in (("act", 6), ("act", -1), ("dtype", 9), ("abi_version", 3)):
            g = gated()
            setattr(g, field, value)
            assert call(g) == L.LP_EINVAL
            assert L.load().lp_gated_workspace_bytes(ctypes.byref(g), 1) == 0
    with pytest.raises(L.LpError):
        L.lp_gated_workspace_bytes(gated(ni=0), False)
    for n in (2 ** 31, 2 ** 32 + 8, 2 ** 63):
        for kw in (dict(B=n), dict(ni=n), dict(no=n)):
            with pytest.raises(L.LpError):
                L.lp_gated_workspace_bytes(gated(**kw), True)


def test_gated_arguments():
    g = gated()
    for kw in (dict(x=None), dict(Wg=None), dict(Wu=None), dict(y=None), dict(y=FAKE[0]), dict(y=FAKE[1]), dict(y=FAKE[2])):
        assert forward(g, **kw) == L.LP_EINVAL, kw
    for kw in (dict(x=None), dict(Wg=None), dict(Wu=None), dict(dy=None), dict(dx=FAKE[3]), dict(dx=FAKE[0]), dict(dWg=FAKE[1]),
               dict(dWu=FAKE[2]), dict(dWu=FAKE[5]), dict(dx=FAKE[6])):
        assert backward(g, **kw) == L.LP_EINVAL, kw
    for kw in bad_workspaces(L.lp_gated_workspace_bytes(g, False)):
        assert forward(g, **kw) == L.LP_EWORKSPACE, kw
    for kw in bad_workspaces(L.lp_gated_workspace_bytes(g, True)):
        assert backward(g, **kw) == L.LP_EWORKSPACE, kw
    # the step has no such gates
    assert L.load().lp_step_workspace_bytes(ctypes.byref(L.LpStep(L.LP_ABI_VERSION, L.LP_BF16, L.LP_SILU, 8, 16, 16, 1.0))) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gated_workspaces(dtype):
    """Over the whole range: what a workspace holds at least and at most."""
    rng, seen, e = random.Random(3), 0, SIZE[dtype]
    for _ in range(400):
        B, ni, no = (rng.choice((1, t, t - 1, int(2 ** rng.uniform(0, t.bit_length() - 1)))) for t in (2 ** 24, 2 ** 20, 2 ** 20))
        g = gated(dtype, B=B, ni=ni, no=no)
        if max(B * no, B * ni, no * ni) > 2 ** 35:
            with pytest.raises(L.LpError):
                L.lp_gated_workspace_bytes(g, True)
            continue
        alone, grad = (L.lp_gated_workspace_bytes(g, k) for k in (False, True))
        copies = (B + 2 * no) * ni * e
        seen += 1
        # (a contraction has at most 32 splits, each with its sums of whole tiles of 128 in fp32)
        parts = 32 * 4 * max((B + 128) * (2 * no + 128), (B + 128) * (ni + 128), (2 * no + 192) * (ni + 128))
        assert copies <= alone <= copies + 128 * (B + 2 * no) + parts and alone <= grad, (B, ni, no)
        assert copies + 2 * B * no * e <= grad <= copies + 2 * B * (no + 32) * e + 128 * (B + 2 * no) + parts, (B, ni, no)
    assert seen > 100


def norm_forward(nd, x=FAKE[0], gamma=FAKE[1], beta=FAKE[2], y=FAKE[3]):
    return L.load().lp_norm_forward(ctypes.byref(nd) if nd else None, x, gamma, beta, y, None)


def norm_backward(nd, x=FAKE[0], gamma=FAKE[1], dy=FAKE[2], dr=FAKE[3], dx=FAKE[4], dgamma=FAKE[5], dbeta=FAKE[6], ws=FAKE[7],
                  n=BIG):
    return L.load().lp_norm_backward(ctypes.byref(nd) if nd else None, x, gamma, dy, dr, dx, dgamma, dbeta, ws, n, None)


def test_norm_descriptor():
    assert norm_forward(None) == L.LP_EINVAL and norm_backward(None) == L.LP_EINVAL
    for call in (norm_forward, norm_backward):
        for d in (("bf16", -1, 8), ("bf16", 8, 0), ("f32", 8, 8, -1e-9), ("f32", 8, 8, float("nan")), ("f32", 8, 8, 1e39)):
            assert call(L.norm(*d)) == L.LP_EINVAL, d
        for d in (("f64", 8, 8), ("bf16", (1 << 24) + 1, 8), ("bf16", 8, (1 << 20) + 1), ("bf16", 1 << 24, 1 << 12)):
            assert call(L.norm(*d)) == L.LP_EUNSUPPORTED, d
        bad = L.norm("bf16", 8, 8)
        bad.abi_version = 3
        assert call(bad) == L.LP_EINVAL
    for n in (2 ** 31, 2 ** 32 + 8):
        with pytest.raises(L.LpError):
            L.lp_norm_workspace_bytes(L.norm("bf16", n, 8))
        with pytest.raises(L.LpError):
            L.lp_norm_workspace_bytes(L.norm("bf16", 8, n))


def test_norm_arguments():
    nd = L.norm("bf16", 1000, 16)
    for kw in (dict(x=None), dict(y=None), dict(y=FAKE[1]), dict(y=FAKE[2])):
        assert norm_forward(nd, **kw) == L.LP_EINVAL, kw
    for kw in (dict(x=None), dict(dy=None), dict(dx=FAKE[0]), dict(dx=FAKE[1]), dict(dx=FAKE[2]), dict(dgamma=FAKE[3]),
               dict(dbeta=FAKE[2]), dict(dgamma=FAKE[4]), dict(dbeta=FAKE[5])):
        assert norm_backward(nd, **kw) == L.LP_EINVAL, kw
    for kw in bad_workspaces(L.lp_norm_workspace_bytes(nd)):
        assert norm_backward(nd, **kw) == L.LP_EWORKSPACE, kw
    assert norm_forward(L.norm("bf16", 0, 16), None, None, None, None) == L.LP_OK


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_norm_workspaces(dtype):
    """Partial sums of few rows, however many rows there are."""
    rng, seen = random.Random(4), 0
    for _ in range(400):
        B, q = (rng.choice((1, t, t - 1, int(2 ** rng.uniform(0, t.bit_length() - 1)))) for t in (2 ** 24, 2 ** 20))
        if B * q > 2 ** 35:
            continue
        seen += 1
        assert 256 <= L.lp_norm_workspace_bytes(L.norm(dtype, B, q)) <= 8 * B + 8 * q * max(1100, B // 2048 + 1) + 512, (B, q)
    assert seen > 100


def orth(od, g=FAKE[0], m=FAKE[1], mo=FAKE[2], alpha=1.0, beta=1.0, r=FAKE[3], W=FAKE[4], ws=FAKE[5], n=BIG):
    return L.load().lp_orth_update(ctypes.byref(od) if od else None, g, m, mo, alpha, beta, r, W, ws, n, None)


def test_orth_descriptor():
    assert orth(None) == L.LP_EINVAL
    nan, inf = float("nan"), float("inf")
    for d, kw in ((("bf16", -1, 4, 4), {}), (("bf16", 2, 0, 4), {}), (("bf16", 2, 4, -1), {}), (("bf16", 2, 4, 4), dict(steps=0)),
                  (("bf16", 2, 4, 4), dict(steps=65)), (("f32", 2, 4, 4), dict(coeffs=(nan, 1, 1))),
                  (("f32", 2, 4, 4), dict(coeffs=(1, 1e39, 1))), (("f32", 2, 4, 4), dict(eps=-1.0)), (("f32", 2, 4, 4), dict(eps=inf)),
                  (("f32", 2, 4, 4), dict(mu=inf))):
        assert orth(L.orth(*d, **kw)) == L.LP_EINVAL, (d, kw)
        with pytest.raises(L.LpError):
            L.lp_orth_workspace_bytes(L.orth(*d, **kw))
    for d in (("f64", 2, 4, 4), ("bf16", (1 << 24) + 1, 4, 4), ("bf16", 1, (1 << 20) + 1, 4), ("bf16", 1, 4, (1 << 20) + 1),
              ("bf16", 1, (1 << 15) + 1, (1 << 15) + 1), ("bf16", 1 << 24, 64, 64)):
        assert orth(L.orth(*d)) == L.LP_EUNSUPPORTED, d
    for field, value in (("abi_version", 3), ("dtype", 9), ("nesterov", 2)):
        o = L.orth("bf16", 2, 4, 4)
        setattr(o, field, value)
        assert orth(o) == L.LP_EINVAL, field
    for n in (2 ** 31, 2 ** 32 + 8):
        for d in ((n, 4, 4), (1, n, 4), (1, 4, n)):
            with pytest.raises(L.LpError):
                L.lp_orth_workspace_bytes(L.orth("bf16", *d))


def test_orth_arguments():
    o = L.orth("bf16", 3, 16, 24, nesterov=True)
    for kw in (dict(g=None), dict(W=None), dict(mo=None), dict(m=None, mo=None), dict(W=FAKE[0]), dict(W=FAKE[1]), dict(W=FAKE[2]),
               dict(mo=FAKE[0]), dict(r=FAKE[2]), dict(alpha=float("nan")), dict(beta=1e39)):
        assert orth(o, **kw) == L.LP_EINVAL, kw
    for kw in bad_workspaces(L.lp_orth_workspace_bytes(o)):
        assert orth(o, **kw) == L.LP_EWORKSPACE, kw
    assert orth(L.orth("bf16", 0, 16, 24), g=None, m=None, mo=None, r=None, W=None) == L.LP_OK


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_orth_workspaces(dtype):
    """What one matrix takes at least; a batch takes no more than some or that of one."""
    rng, seen, e = random.Random(5), 0, SIZE[dtype]
    for _ in range(400):
        N, a, b = (rng.choice((1, t, t - 1, int(2 ** rng.uniform(0, t.bit_length() - 1)))) for t in (2 ** 24, 2 ** 15, 2 ** 20))
        if N * a * b > 2 ** 35:
            continue
        no, ni = (a, b) if rng.random() < 0.5 else (b, a)
        n = min(no, ni)
        seen += 1
        one, all_ = (L.lp_orth_workspace_bytes(L.orth(dtype, k, no, ni)) for k in (1, N))
        held = 2 * (no * ni + n * n) * e
        if n <= 64 and max(no, ni) <= 256:  # held by a workgroup
            assert one == all_ == 256
            continue
        assert held <= one, (no, ni)
        # (X, A and their like in rows of up to 128 bytes more; at most 32 sums of whole tiles of 128 for each product)
        rows = held + 2 * 128 * (no + n) + 8 * 128
        parts = 128 * max((n + 128) ** 2, (no + 128) * (ni + 128))
        assert all_ <= max(rows, 2 ** 30 + 16384 * 1024 + rows) + min(N, max(1, 2 ** 30 // held)) * parts + 4096, (N, no, ni, all_)
    assert seen > 60


def test_binding_refuses_tensors():
    t = torch.zeros(8, 24, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a GPU
        L.lp_gated_forward(gated(), t, t, t, t, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError):
        L.lp_gated_backward(gated(), t, t, t, t, None, None, None, None)
    with pytest.raises(ValueError):
        L.lp_norm_forward(L.norm("bf16", 8, 24), t, None, None, t)
    with pytest.raises(KeyError):
        L.gated("bf16", "swish", 1, 1, 1)
