"""Refusals of the layer steps, checkpoints and label heads on the host (no GPU): every bad call
returns its documented status before any device work, and the binding refuses bad tensors."""
import ctypes

import pytest
import torch

from paper_1812_04352_amd import lp as L

FAKE = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(16)]  # never dereferenced
BIG = 1 << 50


def forward(st, x=FAKE[0], W=FAKE[1], b=FAKE[2], r=FAKE[3], y=FAKE[4], y8=None, ye=None, ws=FAKE[5], n=BIG):
    return L.load().lp_step_forward(ctypes.byref(st) if st else None, x, W, b, r, y, y8, ye, ws, n, None)


def backward(st, x=FAKE[0], x8=None, xe=None, W=FAKE[1], b=FAKE[2], dy=FAKE[3], res=0, dx=FAKE[4], dW=FAKE[5],
             db=FAKE[6], ws=FAKE[7], n=BIG):
    return L.load().lp_step_backward(ctypes.byref(st) if st else None, x, x8, xe, W, b, dy, res, dx, dW, db, ws, n, None)


def loss(hd, u=FAKE[0], W=FAKE[1], mu=FAKE[2], lab=FAKE[3], gs=1.0, J=FAKE[4], row=FAKE[5], du=FAKE[6], dW=FAKE[7],
         dmu=FAKE[8], ws=FAKE[9], n=BIG):
    return L.load().lp_loss_labels(ctypes.byref(hd) if hd else None, u, W, mu, lab, gs, J, row, du, dW, dmu, ws, n, None)


def st(dtype="bf16", act="tanh", B=8, ni=16, no=16, h=1.0):
    return L.step(dtype, act, B, ni, no, h)


def test_step_descriptor():
    assert forward(None) == L.LP_EINVAL and backward(None) == L.LP_EINVAL
    bad = st()
    bad.abi_version = 3
    assert forward(bad) == L.LP_EINVAL and b"abi_version" in L.load().lp_last_error()
    for call in (forward, backward):
        for kw in (dict(B=-1), dict(ni=0), dict(no=-3), dict(h=float("nan")), dict(h=float("inf")), dict(h=1e39)):
            assert call(st(**kw)) == L.LP_EINVAL, kw
        for kw in (dict(dtype="f64"), dict(B=(1 << 24) + 1), dict(ni=(1 << 20) + 1), dict(no=(1 << 20) + 1),
                   dict(B=1 << 24, ni=1 << 12)):
            assert call(st(**kw)) == L.LP_EUNSUPPORTED, kw
        for field, value in (("act", 4), ("act", -1), ("dtype", 9)):
            s = st()
            setattr(s, field, value)
            assert call(s) == L.LP_EINVAL
            assert L.load().lp_step_workspace_bytes(ctypes.byref(s)) == 0
    with pytest.raises(L.LpError):
        L.lp_step_workspace_bytes(st(ni=0))


def test_forward_arguments():
    for kw in (dict(x=None), dict(W=None), dict(y=None), dict(y8=FAKE[8]), dict(ye=FAKE[8])):
        assert forward(st(), **kw) == L.LP_EINVAL, kw
    for kw in (dict(y=FAKE[0]), dict(y=FAKE[1]), dict(y=FAKE[2]), dict(r=FAKE[0], y=FAKE[0])):
        assert forward(st(), **kw) == L.LP_EINVAL, kw
    need = L.lp_step_workspace_bytes(st())
    for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x1010)), dict(n=need - 1)):
        assert forward(st(), **kw) == L.LP_EWORKSPACE, kw


def test_backward_arguments():
    for kw in (dict(x=None), dict(x8=FAKE[8], xe=FAKE[9]), dict(x=None, x8=FAKE[8]), dict(x=None, xe=FAKE[8]),
               dict(W=None), dict(dy=None), dict(res=2), dict(res=-1), dict(dx=FAKE[3]), dict(dx=FAKE[0]),
               dict(dW=FAKE[1]), dict(db=FAKE[2]), dict(dx=FAKE[5]), dict(dW=FAKE[6])):
        assert backward(st(), **kw) == L.LP_EINVAL, kw
    assert backward(st(no=24), res=1) == L.LP_EINVAL and b"ni = no" in L.load().lp_last_error()
    need = L.lp_step_workspace_bytes(st())
    for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x1010)), dict(n=need - 1)):
        assert backward(st(), **kw) == L.LP_EWORKSPACE, kw


def test_checkpoint_arguments():
    lib = L.load()
    for f in (lib.lp_checkpoint_store, lambda d, B, q, a, b, c, s: lib.lp_checkpoint_load(d, B, q, b, c, a, s)):
        assert f(L.LP_F64, 4, 4, *FAKE[:3], None) == L.LP_EUNSUPPORTED
        assert f(7, 4, 4, *FAKE[:3], None) == L.LP_EINVAL
        assert f(L.LP_BF16, -1, 4, *FAKE[:3], None) == L.LP_EINVAL
        assert f(L.LP_BF16, 4, 0, *FAKE[:3], None) == L.LP_EINVAL
        assert f(L.LP_BF16, 4, (1 << 20) + 1, *FAKE[:3], None) == L.LP_EUNSUPPORTED
        assert f(L.LP_BF16, 1 << 24, 1 << 12, *FAKE[:3], None) == L.LP_EUNSUPPORTED
        for i in range(3):
            a = list(FAKE[:3])
            a[i] = None
            assert f(L.LP_BF16, 4, 4, *a, None) == L.LP_EINVAL
        assert f(L.LP_BF16, 4, 4, FAKE[0], FAKE[0], FAKE[1], None) == L.LP_EINVAL
        assert f(L.LP_BF16, 0, 4, None, None, None, None) == L.LP_OK


def test_loss_arguments():
    hd = L.label_head("bf16", 8, 16, 100)
    assert loss(None) == L.LP_EINVAL
    for kw in (dict(u=None), dict(W=None), dict(lab=None), dict(J=None), dict(mu=None), dict(gs=float("nan")),
               dict(gs=1e39), dict(du=FAKE[0]), dict(dW=FAKE[1]), dict(dmu=FAKE[2]), dict(row=FAKE[4]),
               dict(dW=FAKE[6])):
        assert loss(hd, **kw) == L.LP_EINVAL, kw
    full, alone = L.lp_loss_labels_workspace_bytes(hd, True), L.lp_loss_labels_workspace_bytes(hd, False)
    assert alone < full
    for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x1010)), dict(n=full - 1),
               dict(du=None, dW=None, dmu=None, n=alone - 1)):
        assert loss(hd, **kw) == L.LP_EWORKSPACE, kw
    for d, status in ((("f64", 8, 16, 100), L.LP_EUNSUPPORTED), (("bf16", -1, 16, 100), L.LP_EINVAL),
                      (("bf16", 8, 0, 100), L.LP_EINVAL), (("bf16", 8, 16, 0), L.LP_EINVAL),
                      (("bf16", 8, (1 << 20) + 1, 100), L.LP_EUNSUPPORTED),
                      (("bf16", 8, 16, (1 << 24) + 1), L.LP_EUNSUPPORTED),
                      (("bf16", 1 << 24, 16, 1 << 12), L.LP_EUNSUPPORTED)):
        assert loss(L.label_head(*d)) == status, d
        with pytest.raises(L.LpError):
            L.lp_loss_labels_workspace_bytes(L.label_head(*d), True)
    bad = L.label_head("bf16", 8, 16, 100)
    bad.abi_version = 0
    assert loss(bad) == L.LP_EINVAL


def test_loss_workspace_holds_a_piece_of_the_vocabulary():
    """The workspace stays far below the logits of a training batch over a large vocabulary."""
    B, nc = 16384, 262144
    n = L.lp_loss_labels_workspace_bytes(L.label_head("bf16", B, 1024, nc), True)
    assert n < B * nc * 2 // 4


def test_other_entry_points_refuse_the_16_bit_types():
    lib = L.load()
    p = L.problem("f32", "dense", "tanh", 4, 8, 32)
    p.dtype = L.LP_BF16
    assert lib.lp_serial_forward(ctypes.byref(p), *FAKE[:3], None, None) == L.LP_EINVAL
    assert lib.lp_sgd_update(L.LP_F16, 4, 0.1, *FAKE[:2], None) == L.LP_EINVAL


def test_binding_refuses_tensors():
    s = st()
    t = torch.zeros(8, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a GPU
        L.lp_step_forward(s, t, t, t, None, t, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError):
        L.lp_step_forward(s, t, t, t, None, t, None)
    with pytest.raises(ValueError):
        L.lp_checkpoint_store(t, torch.zeros(8, 16, dtype=torch.int8), torch.zeros(8, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        L.lp_checkpoint_store(torch.zeros(4, dtype=torch.int32), None, None)
    with pytest.raises(KeyError):
        L.step("f8", "tanh", 1, 1, 1)


def test_binding_refuses_tensors_of_another_device(monkeypatch):
    """Every tensor of a call is on the current device, whose stream the call uses."""
    class Elsewhere:
        dtype, is_cuda, device = torch.bfloat16, True, "cuda:1"

        def get_device(self):
            return 1

        def is_contiguous(self):
            return True

        def numel(self):
            return 128

        def element_size(self):
            return 2

        def data_ptr(self):
            return 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = Elsewhere()
    with pytest.raises(ValueError, match="current device is cuda:0"):
        L._dev(t, 128, "x", torch.bfloat16, 0)
    with pytest.raises(ValueError, match="workspace is on cuda:1"):
        L._dev_ws(t, 0)
    with pytest.raises(ValueError, match="cuda:1"):
        L.lp_step_forward(st(), t, t, None, None, t, t)


def test_loss_workspace_with_and_without_the_logits():
    """Logits of up to 4 GiB in fp32 are kept for the gradients where there are many features;
    losses alone keep none."""
    kept, again, alone = (L.lp_loss_labels_workspace_bytes(L.label_head("bf16", B, 512, 2 ** 17), g)
                          for B, g in ((8192, True), (8193, True), (8192, False)))
    assert 2 ** 32 < kept < 2 ** 32 + 2 ** 31
    assert again < 2 ** 31 and alone < 2 ** 29
    assert L.lp_loss_labels_workspace_bytes(L.label_head("bf16", 8192, 511, 2 ** 17), True) < 2 ** 31
    # (too far apart for 32-bit offsets within a tile of rows)
    assert L.lp_loss_labels_workspace_bytes(L.label_head("f32", 256, 128, 2 ** 21), True) < 2 ** 30 + 2 ** 29
