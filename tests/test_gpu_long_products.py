"""GPU tests of products over very long contractions: sums are taken out of the accumulators every so often, in every pass."""
import math

import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("tall", [True, False])
def test_small_terms_of_a_long_gram_matrix(tall):
    """2^24 numbers in fp32, all 1 + 31/32 2^-11: their second plane is 31/32 2^-11 of the first, and the two products with it, 2^-10 of
    the sum together, stay exact as long as no accumulator holds more than 16,384 terms of them (31 2^-14 each, in units of the first plane
    squared; one accumulator for all 2^25 of them cuts off the last bits of each: 2.7e-4 of the result).  Sums of either kind are exact
    in fp32 then, and what is left is the rounding of A and P to 22 bits and of the polynomial's terms to 24, none above 4.78:
    2^-22 (2 (4.78 + 2 * 2.04) + 3.45 + 3 * 4.78 / 4) / 0.7 < 2^-16.5 of the result."""
    n, (a, b, c) = 1 << 24, fb.NEWTON_SCHULZ_COEFFICIENTS[0]
    value = 1 + 31 / 32 * 2.0 ** -11
    M = torch.full((n, 1) if tall else (1, n), value, device=DEV)
    out = torch.empty_like(M)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    fb.fopd_orthogonalise(fb.MatrixList([M], [out]), coefficients=[(a, b, c)], eps=0.0, status=status)
    a, b, c = (float(x) for x in torch.tensor((a, b, c)))
    want = (a + b + c) / math.sqrt(n)  # (the one singular value is 1)
    assert int(status.cpu()[0]) == 0
    assert float((out.double() / want - 1).abs().max()) <= 2.0 ** -16.5


def test_weights_gradient_of_more_rows_than_one_wait_lasts_for():
    """2^25 + 77 rows: 524,290 blocks of the contraction for each of G's planes.  Rows repeat, so that the definition is that of a
    few: sums of fp32 over 65,537 accumulators, each off by at most u of what has been added up, and G in two planes (2^-16)."""
    n, V, D, few = (1 << 25) + 77, 5, 8, 1 << 10
    g = torch.Generator(device=DEV).manual_seed(3)
    h = torch.randn((few, D), generator=g, device=DEV).bfloat16()
    w = torch.randn((V, D), generator=g, device=DEV).bfloat16()
    y = torch.randint(0, V, (few,), generator=g, device=DEV, dtype=torch.int32)
    coef = (torch.rand(few, generator=g, device=DEV) + 0.5) / n
    times = torch.full((few,), n // few, device=DEV, dtype=torch.float64)
    times[:n % few] += 1
    repeat = lambda x: x.repeat((-(-n // few),) + (1,) * (x.dim() - 1))[:n]
    z = h.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    lp = z.gather(1, y.long().unsqueeze(1)).squeeze(1) - lse
    G = torch.exp(z - lse.unsqueeze(1))
    G[torch.arange(few, device=DEV), y.long()] -= 1
    G *= (coef.double() * times).unsqueeze(1)
    d_weight = torch.full((V, D), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    fb.fopd_head_grad(repeat(h), w, repeat(y), repeat(lp.float()), repeat(lse.float()), repeat(coef), d_weight=d_weight, status=status)
    assert int(status.cpu()[0]) == 0
    size = G.abs().t() @ h.double().abs()
    err = (d_weight.double() - G.t() @ h.double()).abs()
    assert (err <= (2.0 ** -16 + 2 * 65537 * 2.0 ** -24) * size).all(), float((err / size).max())
    fb._check(fb.lib().fopd_release_device_memory(), "fopd_release_device_memory")  # (34 GB of G)
    torch.cuda.empty_cache()
