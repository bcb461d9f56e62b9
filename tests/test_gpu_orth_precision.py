"""How far orthogonalised updates are off where single rows, columns, values or directions exceed the rest: against
the iteration in 64 bits, held to what the kernels' roundings cost (tests/block_testutil.py)."""
import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
KINDS = ["noise", "row", "column", "value", "directions"]
# one workgroup's, square, wide and tall; a short side in one tile with a long one that is split
SHAPES = [(3, 64, 64), (3, 40, 200), (3, 250, 33), (2, 220, 220), (1, 300, 1000), (1, 1000, 70), (2, 65, 63)]


def matrices(kind, dtype, N, no, ni, seed=0):
    """Noise, with a row, a column or four directions 10^4 or 10^2 times as large, or a value 10^6 times."""
    g = torch.Generator().manual_seed(seed)
    v = 0.01 * torch.randn((N, no, ni), generator=g, dtype=torch.float64)
    if kind == "row":
        v[:, 3] *= 1e4
    elif kind == "column":
        v[:, :, 7] *= 1e4
    elif kind == "value":
        v[:, 3, 5] = 1e4
    elif kind == "directions":
        v = v + torch.matmul(torch.randn((N, no, 4), generator=g, dtype=torch.float64), torch.randn((N, 4, ni), generator=g, dtype=torch.float64))
    return v.to(T.DT[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_what_exceeds_the_rest(shape, kind, dtype):
    v = matrices(kind, dtype, *shape)
    O = K.iterate(v.double().cuda(), 5, L.QUINTIC, 1e-7)
    E = K.iterate_kept(v.double().cuda(), 5, L.QUINTIC, 1e-7, dtype)
    r = (-O).to(T.DT[dtype]).contiguous()
    W = K.Orth(dtype, *shape)(v.cuda(), None, None, r, 1.0)
    K.orth_precise(W, r, O, E, dtype, f"{kind} {shape}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("coeffs, steps", [((2.0, -20.0, 30.0), 2), ((2.0, -400.0, 0.0), 1), ((1.5, -0.5, 0.0), 1), ((1.5, -0.5, 0.0), 2)])
def test_other_coefficients(coeffs, steps, dtype):
    """Large ones, which small singular values allow, and iterations of one and two steps."""
    shape = (2, 220, 300)
    v = matrices("noise", dtype, *shape)
    O = K.iterate(v.double().cuda(), steps, coeffs, 1e-7)
    E = K.iterate_kept(v.double().cuda(), steps, coeffs, 1e-7, dtype)
    r = (-O).to(T.DT[dtype])
    W = K.Orth(dtype, *shape, steps=steps, coeffs=coeffs)(v.cuda(), None, None, r, 1.0)
    K.orth_precise(W, r, O, E, dtype, f"{coeffs} {steps}")
