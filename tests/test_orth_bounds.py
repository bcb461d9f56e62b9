"""What the GPU tests of orthogonalised updates hold the kernels to is less than mistakes cost that a kernel could make:
the iteration in 64 bits with such a mistake is refused, with what the kernels round it passes (CPU only)."""
import math

import pytest
import torch

import block_testutil as K
import wide_testutil as T
from paper_1812_04352_amd import lp as L
from test_gpu_orth_precision import matrices


def coarse(v, up, keep):
    """Operands and X of a X by one rounding of their own."""
    a, b, c = L.QUINTIC
    X = v / (torch.linalg.vector_norm(v, dim=(1, 2), keepdim=True) + 1e-7)
    for _ in range(5):
        X = keep(X, up)
        A = keep(torch.matmul(X, X.transpose(1, 2).contiguous()), 2.0 ** 8)
        X = a * X + torch.matmul(keep(b * A + c * torch.matmul(A, A), 2.0 ** 8), X)
    return X


def single(t, up):
    return (t * up).half().double() / up


def refused(Z, v, dtype):
    O = K.iterate(v, 5, L.QUINTIC, 1e-7)
    E = K.iterate_kept(v, 5, L.QUINTIC, 1e-7, dtype)
    r = (-O).to(T.DT[dtype])
    K.orth_precise((E + r.double()).to(T.DT[dtype]), r, O, E, dtype, "as the kernels round")
    with pytest.raises(AssertionError):
        K.orth_precise((Z + r.double()).to(T.DT[dtype]), r, O, E, dtype, "")


@pytest.mark.parametrize("kind", ["row", "column", "value"])
def test_scale_of_x(kind):
    """fp32: X in two parts, but by the root of its size."""
    v = matrices(kind, "f32", 1, 220, 220).double()
    refused(coarse(v, 2.0 ** round(math.log2(220)), K.two_parts), v, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["noise", "row", "column", "value", "directions"])
def test_low_parts_of_small_matrices(kind, dtype):
    """Matrices that a workgroup holds, with the second parts left out, in every type."""
    v = matrices(kind, dtype, 2, 40, 200).double()
    refused(coarse(v, 2.0 ** 7, single), v, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_x_of_a_x(dtype):
    """16-bit types: a X by no more bits than the products' operand has."""
    v = matrices("directions", dtype, 1, 220, 220).double()
    refused(coarse(v, 2.0 ** 14, single), v, dtype)
