"""GPU tests of fopd_orthogonalise where eps is far above a matrix's norm: X starts small and is as exact as any."""
import math

import pytest
import torch

from oracle import orth_oracle as oo
from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
FIVE = fb.NEWTON_SCHULZ_COEFFICIENTS


def matrix(m, n, seed, dtype, scale=1e-3):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((m, n), generator=g, device=DEV) + torch.randn((m, 2), generator=g, device=DEV) @ torch.randn((2, n), generator=g, device=DEV)
    return (x * scale).to(dtype)


def check(M, out, eps, coefficients=FIVE, scale=1.0):
    """Twice the played-through roundings (the oracle's planes follow the values, so they do not depend on eps), the sums' error and the
    result's own rounding, all of the result's size."""
    full = out.dtype == F32
    played, want = oo.rounding_error(M, coefficients, eps, full, exact_input=M.dtype == BF16)
    d = 4 * U * (math.ceil(max(M.shape) / 16) + 4) * (3 if full else 2)
    size = float(want.norm())
    err = float((out.double() / scale - want).norm())
    assert size > 0 and err <= 2 * played + (16 * d + (U if full else 2.0 ** -8)) * size, (err / size, played / size)


@pytest.mark.parametrize("ratio", [0.9, 0.3, 1e-2, 1e-4, 1e-6, 1e-8, 1e-12, 1e-25])
@pytest.mark.parametrize("din,dout", [(F32, F32), (BF16, BF16), (F32, BF16)])
def test_norms_below_eps(ratio, din, dout):
    Ms = [matrix(60, 90, 6, din), matrix(500, 300, 7, din), matrix(17, 40, 8, din)]
    for M in Ms:
        eps = float(torch.tensor(float(M.double().norm()) / ratio, dtype=F32))
        out = torch.empty(M.shape, device=DEV, dtype=dout)
        fb.fopd_orthogonalise(fb.MatrixList([M], [out]), eps=eps)
        check(M, out, eps)


def test_norms_of_every_size_in_one_list():
    """Scales of 10^0 to 10^-30 under one eps; the results' sizes span as much."""
    Ms = [matrix(40 + 10 * k, 200 - 9 * k, k, BF16 if k % 3 == 0 else F32, 10.0 ** -(2 * k)) for k in range(16)]
    outs = [torch.empty(M.shape, device=DEV, dtype=F32) for M in Ms]
    fb.fopd_orthogonalise(fb.MatrixList(Ms, outs, [2.0] * 16), eps=1e-7)
    eps = float(torch.tensor(1e-7, dtype=F32))
    for M, o in zip(Ms, outs):
        check(M, o, eps, scale=2.0)


@pytest.mark.parametrize("coefficients", [[(1.5, -0.5, 0.0)] * 12, [(100.0, -9.0, 5.0)], [(0.01, 2.0, -1.0)] * 2, [(-3.0, 2.0, 0.5)] * 3])
@pytest.mark.parametrize("ratio", [1e-2, 1e-5])
def test_other_coefficients(coefficients, ratio):
    """Steps that amplify more or less than their bound, and ones under which small singular values shrink."""
    M = matrix(100, 150, 9, F32)
    eps = float(torch.tensor(float(M.double().norm()) / ratio, dtype=F32))
    out = torch.empty_like(M)
    fb.fopd_orthogonalise(fb.MatrixList([M], [out]), eps=eps, coefficients=coefficients)
    c32 = [tuple(float(x) for x in torch.tensor(c, dtype=F32)) for c in coefficients]
    check(M, out, eps, c32)


def test_results_at_the_ends_of_their_range():
    """A norm 10^-60 of eps: a result below fp32's numbers is zero, and with a large factor is what it should be."""
    M = matrix(30, 50, 3, F32, 1e-30)
    small, large = torch.full_like(M, 7.0), torch.full_like(M, 7.0)
    fb.fopd_orthogonalise(fb.MatrixList([M, M], [small, large], [1.0, 1e38]), eps=1e30)
    assert (small == 0).all()
    check(M, large, float(torch.tensor(1e30, dtype=F32)), scale=float(torch.tensor(1e38, dtype=F32)))
