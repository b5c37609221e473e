"""Newton-Schulz orthogonalisation in 64 bits, and the same with its intermediate roundings played through.

X = M / (|M| + eps);  X <- (a I + b A + c A^2) X with A = X X^T for every (a, b, c);  scale X.  Written from the definition."""
from __future__ import annotations

import torch


def orthogonalise(M, coefficients, eps=1e-7, scale=1.0):
    """The definition, by the Gram matrix of the shorter side."""
    X = M.double()
    X = X / (X.square().sum().sqrt() + eps)
    tall = X.shape[0] > X.shape[1]
    X = X.mT if tall else X
    one = torch.eye(X.shape[0], dtype=torch.float64, device=X.device)
    for a, b, c in coefficients:
        A = X @ X.mT
        X = (a * one + b * A + c * (A @ A)) @ X
    return scale * (X.mT if tall else X)


def _held(x, planes):
    """Rounded to 11 bits (one plane of fp16 under a scale that keeps clear of both ends of its range) or what two planes hold."""
    top = x.abs().amax().clamp(min=1e-300)
    s = torch.exp2(14 - torch.ceil(torch.log2(top)))
    y = x * s
    hi = y.half().double()
    return (hi + ((y - hi).half().double() if planes > 1 else 0.0)) / s


def rounding_error(M, coefficients, eps=1e-7, full=False, loud=32.0, exact_input=True, square=False):
    """Frobenius norm of what the roundings of X, A and P leave in the result: X has two planes while the steps ahead amplify by
    `loud` or more, A and P one (two with `square`); all have two with `full`.  The Gram matrix is that of X's first plane unless `full`."""
    want = orthogonalise(M, coefficients, eps)
    X = M.double()
    X = X / (X.square().sum().sqrt() + eps)
    X = X.mT if X.shape[0] > X.shape[1] else X
    one = torch.eye(X.shape[0], dtype=torch.float64, device=X.device)
    two, squares = 2 if full else 1, 2 if full or square else 1
    for k, (a, b, c) in enumerate(coefficients):
        ahead = 1.0
        for later in coefficients[k:]:
            ahead *= abs(later[0])
        first = X
        if k or not exact_input:
            X, first = _held(X, 2 if full or ahead >= loud else 1), _held(X, two)
        A = _held(first @ first.mT, squares)
        X = _held(a * one + b * A + c * (A @ A), squares) @ X
    X = X.mT if M.shape[0] > M.shape[1] else X
    return float((X - want).norm()), want
