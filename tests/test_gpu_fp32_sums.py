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


@pytest.mark.parametrize("n,at_once,V,D", [(96, 1, 32000, 1024), (64, 1, 8000, 2048), (128, 128, 32000, 1024), (96, 48, 8000, 2048)])
def test_log_probs_of_few_rows(n, at_once, V, D):
    """Logits ~ N(0, 3^2), every token a likely one: its logit is near the largest.  Few rows, one at a time or all at once (elementary products
    are the more exact the fewer they are)."""
    g = torch.Generator(device=DEV).manual_seed(n)
    h = torch.randn((n, D), generator=g, device=DEV)
    w = (torch.randn((V, D), generator=g, device=DEV) * (3 / math.sqrt(D))).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    of = w[y.long()].float()
    h = (h + of * (4.0 / of.square().sum(1, keepdim=True).sqrt())).bfloat16()
    lp, plain, token = torch.empty(n, device=DEV), torch.empty(n, device=DEV), y.long().unsqueeze(1)
    for k in range(0, n, at_once):
        rows = slice(k, k + at_once)
        fb.fopd_head_logprob(h[rows], w, y[rows], lp[rows])
        z = h[rows].float() @ w.float().t()
        m = z.amax(1, keepdim=True)
        plain[rows] = (z.gather(1, token[rows]) - ((z - m).exp().sum(1, keepdim=True, dtype=torch.float64).log() + m)).squeeze(1).float()
    want = torch.log_softmax(h.double() @ w.double().t(), 1).gather(1, token).squeeze(1)
    here, plain = (float((x.double() - want).square().mean().sqrt()) for x in (lp, plain))
    assert here <= 1.5 * plain, (here, plain)
