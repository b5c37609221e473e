"""GPU tests of how exact fp32 results are, beside the same operators in elementary fp32 operations (no TF32): sums that a matrix
instruction cuts off instead of rounding are taken out and added often enough that no more than half as much error again is left."""
import math

import pytest
import torch

from oracle import orth_oracle as oo
from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def no_tf32():
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = before


def plain_orthogonalise(M, coefficients, eps):
    X = M.float()
    X = X / (X.square().sum(dtype=torch.float64).sqrt().float() + eps)
    X = X.t() if M.shape[0] > M.shape[1] else X
    for a, b, c in coefficients:
        A = X @ X.t()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.t() if M.shape[0] > M.shape[1] else X


@pytest.mark.parametrize("shape", [(256, 1024), (1000, 1000), (2500, 1000), (250, 1000)])
def test_orthogonalised_matrices(shape):
    errors = []
    for seed in range(4):
        g = torch.Generator(device=DEV).manual_seed(seed)
        M = torch.randn((shape[0], 8), generator=g, device=DEV) @ torch.randn((8, shape[1]), generator=g, device=DEV) / math.sqrt(8)
        M = (M * 0.5 + torch.randn(shape, generator=g, device=DEV)) * 1e-3
        out = torch.empty_like(M)
        fb.fopd_orthogonalise(fb.MatrixList([M], [out]))
        want = oo.orthogonalise(M, fb.NEWTON_SCHULZ_COEFFICIENTS)
        plain = plain_orthogonalise(M, fb.NEWTON_SCHULZ_COEFFICIENTS, 1e-7)
        errors.append([float((x.double() - want).norm() / want.norm()) for x in (out, plain)])
    here, plain = (sum(e[k] for e in errors) / len(errors) for k in range(2))
    assert here <= 1.5 * plain, (here, plain)
