"""Workspaces of the wide operators over their whole range of sizes (no GPU): the layouts' arithmetic
at the limits, and what a workspace holds at least and at most."""
import random

import pytest

from paper_1812_04352_amd import lp as L

SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def sizes(rng, *tops):
    """One size per top, over its logarithm, the ends among them."""
    return [rng.choice((1, t, t - 1, int(2 ** rng.uniform(0, t.bit_length() - 1)))) for t in tops]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_step_workspaces(dtype):
    rng, seen = random.Random(1), 0
    for _ in range(400):
        B, ni, no = sizes(rng, 2 ** 24, 2 ** 20, 2 ** 20)
        st = L.step(dtype, "tanh", B, ni, no)
        if max(B * no, B * ni, no * ni) > 2 ** 35:
            with pytest.raises(L.LpError):
                L.lp_step_workspace_bytes(st)
            continue
        n, held, seen = L.lp_step_workspace_bytes(st), (B * no + B * ni + no * ni) * SIZE[dtype], seen + 1
        # g, copies of x and W with rows of up to 128 bytes more; column partials and split sums
        assert held <= n < held + 128 * (2 * B + no) + 8 * B * no + 2 ** 31, (B, ni, no, n)
    assert seen > 100


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_label_workspaces(dtype):
    rng, seen = random.Random(2), 0
    for _ in range(400):
        B, q, nc = sizes(rng, 2 ** 24, 2 ** 20, 2 ** 24)
        hd = L.label_head(dtype, B, q, nc)
        if max(B * nc, B * q, nc * q) > 2 ** 35:
            with pytest.raises(L.LpError):
                L.lp_loss_labels_workspace_bytes(hd, True)
            continue
        alone, grad = (L.lp_loss_labels_workspace_bytes(hd, g) for g in (False, True))
        seen += 1
        assert 8 * B + B * q * SIZE[dtype] <= alone <= grad, (B, q, nc)
    assert seen > 100
