"""The softmax cross-entropy of integer labels over large vocabularies against 64-bit plain forms.
Bounds: tests/wide_testutil.py."""
import math

import pytest
import torch

import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

# (rows, features, classes): one of each, odd sizes, below and above tiles, many classes for few rows
SHAPES = [(1, 1, 1), (1, 64, 1000), (2, 3, 2), (5, 33, 129), (16, 256, 4099), (64, 48, 128), (130, 65, 257),
          (300, 40, 700), (33, 520, 1025), (1000, 16, 90)]


def inputs(seed, dtype, B, q, nc, ignored=0.0, std=2.0):
    g = torch.Generator().manual_seed(seed)
    u = T.draw(g, (B, q), dtype)
    W = T.draw(g, (nc, q), dtype, std / math.sqrt(q))
    mu = T.draw(g, (nc,), dtype, 0.5)
    lab = torch.randint(0, nc, (B,), generator=g)
    lab[torch.rand(B, generator=g) < ignored] = -100
    return u, W, mu, lab


def run(dtype, u, W, mu, lab, gscale=1.0, want=(True, True, True), hd=None, ws=None):
    (B, q), nc = u.shape, W.shape[0]
    hd = hd or L.label_head(dtype, B, q, nc)
    grad = any(want)
    ws = ws if ws is not None else L.alloc_loss_labels_workspace(hd, grad)
    shapes = ((B, q), (nc, q), (nc,))
    bufs = [T.out(s, T.DT[dtype]) if w and not (i == 2 and mu is None) else (None, None)
            for i, (s, w) in enumerate(zip(shapes, want))]
    J, Jf = T.out((1,), torch.float32)
    row, rf = T.out((B,), torch.float32)
    L.lp_loss_labels(hd, u, W, mu, lab, J, ws, row=row, du=bufs[0][0], dW=bufs[1][0], dmu=bufs[2][0], gscale=gscale)
    torch.cuda.synchronize()
    assert T.guarded(Jf, 1) and T.guarded(rf, B)
    for v, f in bufs:
        assert v is None or T.guarded(f, v.numel())
    return [J, row] + [v for v, _ in bufs]


def compare(got, ref, what=""):
    for name, a, (r, e) in zip(("J", "row", "du", "dW", "dmu"), got, ref):
        if a is not None:
            T.check(a.reshape(-1) if name == "J" else a, r.reshape(-1) if name == "J" else r,
                    e.reshape(-1) if name == "J" else e, f"{name} {what}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_loss_and_gradients(dtype, i):
    B, q, nc = SHAPES[i]
    u, W, mu, lab = inputs(i, dtype, B, q, nc, ignored=(0.0, 0.4)[i % 2])
    if i % 3 == 2:
        mu = None
    gs = (1.0, 64.0)[i % 2]
    dev = [T.gpu(t) for t in (u, W, mu, lab)]
    got = run(dtype, *dev, gscale=gs)
    ref = T.loss(u, W, mu, lab, gs, dtype)
    compare(got, ref)
    # the losses alone
    alone = run(dtype, *dev, want=(False, False, False))
    compare(alone, ref)
    # one gradient at a time, the same bits
    for k in range(3):
        want = [j == k for j in range(3)]
        if k == 2 and mu is None:
            continue
        part = run(dtype, *dev, gscale=gs, want=want)
        assert torch.equal(part[2 + k], got[2 + k])


def test_aligned_arrays():
    for dtype in ("bf16", "f16", "f32"):
        for B, q, nc in ((130, 64, 512), (256, 128, 1000), (24, 256, 2048)):
            u, W, mu, lab = inputs(3, dtype, B, q, nc, ignored=0.2)
            compare(run(dtype, u.cuda(), W.cuda(), mu.cuda(), lab.cuda()), T.loss(u, W, mu, lab, 1.0, dtype),
                    f"{dtype} {B} {q} {nc}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_without_a_label(dtype):
    """Ignored rows may hold anything; labels outside the vocabulary (below, at and far above) are
    none; with no labelled row everything is zero."""
    B, q, nc = 150, 40, 300
    u, W, mu, lab = inputs(5, dtype, B, q, nc, ignored=0.3)
    lab[0], lab[1], lab[2], lab[149] = -1, nc, 2 ** 40, -2 ** 62
    off = (lab < 0) | (lab >= nc)
    dirty = u.clone()
    dirty[off] = math.nan
    dirty[0] = math.inf
    got = run(dtype, *[T.gpu(t) for t in (dirty, W, mu, lab)])
    compare(got, T.loss(u, W, mu, lab, 1.0, dtype))
    assert not got[1][off.cuda()].any() and not got[2][off.cuda()].any()
    compare(run(dtype, *[T.gpu(t) for t in (dirty, W, mu, lab)], want=(False,) * 3), T.loss(u, W, mu, lab, 1.0, dtype))
    none = torch.full_like(lab, -100)
    for want in ((True,) * 3, (False,) * 3):
        for a in run(dtype, *[T.gpu(t) for t in (dirty, W, mu, none)], want=want):
            assert a is None or not a.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_masked_classes(dtype):
    """Classes masked by -infinity or by the type's lowest value have probability zero; whole tiles
    of them; a label on one; every class masked."""
    B, q, nc = 70, 24, 600
    u, W, mu, lab = inputs(6, dtype, B, q, nc)
    lab = lab % 128  # labels stay in the first tile
    mu[200:] = -math.inf
    mu[5:20] = -math.inf
    ok = [k for k in range(200) if not 5 <= k < 20]
    lab[(lab >= 5) & (lab < 20)] = 3
    got = run(dtype, *[T.gpu(t) for t in (u, W, mu, lab)])
    remap = torch.full((nc,), -1, dtype=torch.long)
    remap[ok] = torch.arange(len(ok))
    ref = T.loss(u, W[ok], mu[ok], remap[lab], 1.0, dtype)
    compare(got[:3], ref[:3])
    for a, r in zip(got[3:], ref[3:]):
        T.check(a[ok], *r, "weights")
        rest = [k for k in range(nc) if k not in set(ok)]
        assert not a[rest].any()
    low = mu.clone()
    low[low == -math.inf] = torch.finfo(T.DT[dtype]).min
    compare(run(dtype, *[T.gpu(t) for t in (u, W, low, lab)])[:3], ref[:3])
    lab2 = lab.clone()
    lab2[4] = 300
    got2 = run(dtype, *[T.gpu(t) for t in (u, W, mu, lab2)])
    assert got2[1][4].item() == math.inf and torch.isfinite(got2[2]).all() and torch.isfinite(got2[3]).all()
    mu[:] = -math.inf
    assert run(dtype, *[T.gpu(t) for t in (u, W, mu, lab)])[1].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_large_logits_and_certain_rows(dtype):
    """Logits far apart (probabilities of one and of nothing), no overflow."""
    B, q, nc = 40, 64, 500
    u, W, mu, lab = inputs(8, dtype, B, q, nc, std=60.0)
    lab[:20] = (u.double() @ W.double().t() + mu.double()).argmax(1)[:20]
    compare(run(dtype, *[T.gpu(t) for t in (u, W, mu, lab)]), T.loss(u, W, mu, lab, 1.0, dtype))


def test_f16_gradients_of_a_large_vocabulary():
    """Probabilities near 1 / nc, far below f16's normal range: they must not be lost."""
    B, q, nc = 64, 32, 60000
    u, W, mu, lab = inputs(9, "f16", B, q, nc, std=0.1)
    got = run("f16", *[T.gpu(t) for t in (u, W, mu, lab)], gscale=1024.0)
    ref = T.loss(u, W, mu, lab, 1024.0, "f16")
    compare(got, ref)
    d = (got[2].double().cpu() - ref[2][0]).norm() / ref[2][0].norm()
    assert d <= 2 * T.half_step("f16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_pieces_of_the_vocabulary(dtype):
    B, q, nc = 4100, 8, 40001 if dtype == "bf16" else 20001
    u, W, mu, lab = (t.cuda() for t in inputs(10, dtype, B, q, nc, ignored=0.1))
    hd = L.label_head(dtype, B, q, nc)
    whole = B * nc * (2 if dtype == "bf16" else 4)
    assert whole > 256 << 20  # more than one piece
    got = run(dtype, u, W, mu, lab)
    assert L.lp_loss_labels_workspace_bytes(hd, True) < 2 * whole + B * (nc + 7) * 4  # (with the logits in fp32)
    with torch.device("cuda"):
        on = lab >= 0
        n = int(on.sum())
        z = u.double() @ W.double().t() + mu.double()
        lse = torch.logsumexp(z, 1)
        rows = torch.arange(B)
        row = torch.where(on, lse - z[rows, lab.clamp(min=0)], 0)
        P = torch.exp(z - lse[:, None])
        P[rows, lab.clamp(min=0)] -= 1
        P[~on] = 0
        refs = [row.sum() / n, row, P @ W.double() / n, P.t() @ u.double() / n, P.sum(0) / n]
    # norms: half a step of P and of the result, each uniform in its rounding, and fp32 sums
    lim = {"bf16": 2 ** -8, "f32": 2 ** -18}[dtype]
    for name, a, r in zip(("J", "row", "du", "dW", "dmu"), got, refs):
        d = float((a.double().reshape(-1) - r.reshape(-1)).norm() / r.norm())
        assert d <= (2 ** -18 if name in ("J", "row") else lim), (name, d)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_empty_batch(dtype):
    hd = L.label_head(dtype, 0, 20, 300)
    g = torch.Generator().manual_seed(2)
    W, mu = T.gpu(T.draw(g, (300, 20), dtype)), T.gpu(T.draw(g, (300,), dtype))
    u = torch.empty((0, 20), dtype=T.DT[dtype], device="cuda")
    lab = torch.empty((0,), dtype=torch.int64, device="cuda")
    for want in ((True,) * 3, (False,) * 3):
        got = run(dtype, u, W, mu, lab, want=want, hd=hd)
        assert all(a is None or not a.any() for a in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_streams_graphs_and_equal_bits(dtype):
    B, q, nc = 200, 72, 1500
    u, W, mu, lab = (T.gpu(t) for t in inputs(12, dtype, B, q, nc, ignored=0.3))
    dt = T.DT[dtype]
    hd = L.label_head(dtype, B, q, nc)

    def bufs():
        return dict(J=torch.zeros(1, device="cuda"), row=torch.zeros(B, device="cuda"),
                    du=torch.zeros((B, q), dtype=dt, device="cuda"), dW=torch.zeros((nc, q), dtype=dt, device="cuda"),
                    dmu=torch.zeros(nc, dtype=dt, device="cuda"), ws=L.alloc_loss_labels_workspace(hd))

    def call(o):
        L.lp_loss_labels(hd, u, W, mu, lab, o["J"], o["ws"], row=o["row"], du=o["du"], dW=o["dW"], dmu=o["dmu"])

    names = ("J", "row", "du", "dW", "dmu")
    eager, other = bufs(), bufs()
    call(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(other)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(eager[k], other[k]) for k in names)
    graphs = []
    for _ in range(2):
        o = bufs()
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr):
            call(o)
        graphs.append((gr, o))
    for it in range(4):
        # other inputs, another number of labelled rows
        g = torch.Generator("cuda").manual_seed(it)
        u.copy_(torch.randn((B, q), generator=g, device="cuda").to(dt))
        lab.copy_(torch.randint(-nc // 2 * it, nc, (B,), generator=g, device="cuda"))
        call(eager)
        torch.cuda.synchronize()
        for gr, o in graphs:
            for k in names:
                o[k].fill_(3)
            gr.replay()
        torch.cuda.synchronize()
        for gr, o in graphs:
            assert all(torch.equal(eager[k], o[k]) for k in names), it


def test_gradients_against_differences():
    B, q, nc = 30, 20, 150
    u, W, mu, lab = inputs(14, "f32", B, q, nc, ignored=0.2)
    got = run("f32", *[T.gpu(t) for t in (u, W, mu, lab)])
    g = torch.Generator().manual_seed(15)
    dirs = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (u, W, mu)]
    on = lab >= 0

    def f(e):
        z = (u.double() + e * dirs[0]) @ (W.double() + e * dirs[1]).t() + mu.double() + e * dirs[2]
        return float(-torch.log_softmax(z, 1)[on].gather(1, lab[on][:, None]).mean())

    num = (f(1e-5) - f(-1e-5)) / 2e-5
    terms = [a.double().cpu() * d for a, d in zip(got[2:], dirs)]
    ana, mag = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(num - ana) <= 1e-6 * mag + 1e-8


def on_gpu(dtype, u, W, mu, lab):
    """J, row, du, dW, dmu in 64 bits on the GPU, a slice of the rows at a time."""
    B, q = u.shape
    on = lab >= 0
    n = max(1, int(on.sum()))
    row, du = torch.zeros(B, dtype=torch.float64, device="cuda"), torch.zeros((B, q), dtype=torch.float64, device="cuda")
    dW = torch.zeros(W.shape, dtype=torch.float64, device="cuda")
    dmu = torch.zeros(W.shape[0], dtype=torch.float64, device="cuda")
    Wd = W.double()
    per = max(1, 2 ** 28 // W.shape[0])
    for k in range(0, B, per):
        at = torch.nonzero(on[k:k + per]).flatten() + k
        if not len(at):
            continue
        z = u[at].double() @ Wd.t() + (0 if mu is None else mu.double())
        lse = torch.logsumexp(z, 1)
        i = torch.arange(len(at), device="cuda")
        row[at] = lse - z[i, lab[at]]
        P = torch.exp(z - lse[:, None])
        P[i, lab[at]] -= 1
        du[at] = P @ Wd / n
        dW += P.t() @ u[at].double() / n
        dmu += P.sum(0) / n
        del z, P
    return row.sum().reshape(1) / n, row, du, dW, dmu


# norms, as in the test of several pieces: half a step of P and of the result, and fp32 sums; and half
# of the type's smallest step for each value (a mean over 7500 rows of probabilities near 1 / 131000
# leaves dW of f16 near 3e-6, below its normal range of 6.1e-5: each value may be off by 2^-25 = 3e-8,
# together 2^-25 sqrt(numel), which is 4e-4 of that norm)
NORMS = {"bf16": 2 ** -8, "f16": 2 ** -11, "f32": 2 ** -18}


def near(dtype, got, refs):
    for name, a, r in zip(("J", "row", "du", "dW", "dmu"), got, refs):
        d, n = float((a.double().reshape(-1) - r.reshape(-1)).norm()), float(r.norm())
        lim = 2 ** -18 * n if name in ("J", "row") else NORMS[dtype] * n + T.tiny(dtype) * math.sqrt(r.numel())
        assert d <= lim, (name, d, n)


@pytest.mark.parametrize("dtype,B,nc", [("f16", 8300, 131000), ("f32", 8300, 131000), ("bf16", 140, 3900001),
                                        ("f32", 140, 3900001)])
def test_logits_formed_a_second_time(dtype, B, nc):
    """Batches whose logits are too many to be kept (over 4 GiB in fp32), or too far apart."""
    u, W, mu, lab = (t.cuda() for t in inputs(12, dtype, B, 8, nc, ignored=0.1))
    hd = L.label_head(dtype, B, 8, nc)
    # (without them: the probabilities of a piece, and for each row and tile 8 bytes)
    assert L.lp_loss_labels_workspace_bytes(hd, True) < B * nc * 4
    near(dtype, run(dtype, u, W, mu, lab, gscale=1.0), on_gpu(dtype, u, W, mu, lab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 3, 70])
def test_weights_copied_in_pieces(dtype, B):
    """Rows of W that do not start on 16 bytes, and more of them than are copied at a time."""
    q, nc = 4097, 40000
    u, W, mu, lab = (t.cuda() for t in inputs(14, dtype, B, q, nc))
    assert nc * q * u.element_size() > 256 << 20
    near(dtype, run(dtype, u, W, mu, lab), on_gpu(dtype, u, W, mu, lab))
    near(dtype, run(dtype, u, W, mu, lab, want=(False,) * 3)[:2], on_gpu(dtype, u, W, mu, lab)[:2])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_many_rows(dtype):
    """More rows than a workgroup lists by itself, of one piece."""
    B, q, nc = 5003, 24, 300
    u, W, mu, lab = inputs(15, dtype, B, q, nc, ignored=0.3)
    compare(run(dtype, *[T.gpu(t) for t in (u, W, mu, lab)]), T.loss(u, W, mu, lab, 1.0, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_kept_logits_of_several_pieces(dtype):
    """Logits kept for the gradients, whose probabilities are taken a piece at a time (fp32: in place)."""
    B, q, nc = 2100, 520, 70001
    u, W, mu, lab = (t.cuda() for t in inputs(16, dtype, B, q, nc, ignored=0.2))
    hd = L.label_head(dtype, B, q, nc)
    assert B * nc * u.element_size() > 256 << 20
    assert L.lp_loss_labels_workspace_bytes(hd, True) > B * nc * 4
    near(dtype, run(dtype, u, W, mu, lab), on_gpu(dtype, u, W, mu, lab))
