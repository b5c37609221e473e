"""GPU tests of fopd_orthogonalise on thin matrices with results in bf16: of A and P, as many numbers as the shorter side squared,
roundings do not average out however long the matrix is."""
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


def matrix(m, n, g, dtype, strong):
    x = torch.randn((m, n), generator=g, device=DEV)
    if strong:
        k = min(4, m)
        x = x + torch.randn((m, k), generator=g, device=DEV) @ torch.randn((k, n), generator=g, device=DEV)
    return (x * 1e-3).to(dtype)


@pytest.mark.parametrize("din", [BF16, F32])
@pytest.mark.parametrize("most,lots,longest", [(2, 2, 700), (4, 4, 1000), (8, 2, 4000), (16, 2, 4000)])
def test_thin_matrices(din, most, lots, longest):
    """A result is rounded once (2^-8 of each element); X has one plane in the last two steps and a second one before, and A and P two: what
    that leaves is played through and allowed twice, with the sums' error (4 u of the accumulator dropped for every 16 terms, in each of five
    steps' three products)."""
    g, h = torch.Generator().manual_seed(most), torch.Generator(device=DEV).manual_seed(most)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))
    for lot in range(lots):
        Ms = [matrix(pick(1, most), pick(257, longest), h, din, k % 2 == 0) for k in range(240)]
        Ms = [M.t().contiguous() if k % 3 == 0 else M for k, M in enumerate(Ms)]
        outs = [torch.empty_like(M, dtype=BF16) for M in Ms]
        fb.fopd_orthogonalise(fb.MatrixList(Ms, outs))
        for M, o in zip(Ms, outs):
            played, want = oo.rounding_error(M, FIVE, exact_input=din == BF16, square=True)
            size = float(want.norm())
            d = 4 * U * (math.ceil(max(M.shape) / 16) + 4) * 2
            err = float((o.double() - want).norm())
            assert err <= 2 * played + 16 * d * size + 2.0 ** -8 * size, (tuple(M.shape), err / size, played / size)
            assert played <= 2.0 ** -9 * size


def test_thin_matrices_among_others():
    """One list with matrices held in every way; alone each gives the same bits as in it."""
    h = torch.Generator(device=DEV).manual_seed(5)
    shapes = [(4, 1000), (3000, 3), (16, 256), (16, 257), (17, 257), (1, 2500), (100, 130), (2, 20)]
    Ms = [matrix(min(s), max(s), h, BF16 if k % 2 else F32, True) for k, s in enumerate(shapes)]
    Ms = [M.t().contiguous() if s[0] > s[1] else M for M, s in zip(Ms, shapes)]
    outs = [torch.empty_like(M, dtype=F32 if k == 5 else BF16) for k, M in enumerate(Ms)]
    fb.fopd_orthogonalise(fb.MatrixList(Ms, outs))
    for M, o in zip(Ms, outs):
        alone = torch.empty_like(o)
        fb.fopd_orthogonalise(fb.MatrixList([M], [alone]))
        assert torch.equal(alone, o)
        want = oo.orthogonalise(M, FIVE)
        assert float((o.double() - want).norm()) <= (2.0 ** -8 + 2.0 ** -10) * float(want.norm())
