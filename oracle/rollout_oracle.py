"""fp64 definitions of the rollout and clipping entry points, in plain numpy: one row, one draft at a
time.  Test infrastructure only; shares nothing with the CUDA sources."""
from __future__ import annotations

import math

import numpy as np


def as64(x):
    """A torch tensor (bf16 widened exactly) or array as fp64 numpy."""
    if hasattr(x, "detach"):
        x = x.detach().cpu().double().numpy()
    return np.asarray(x, dtype=np.float64)


def probabilities(row, temperature):
    """softmax(row / T); T = 0: all on the lowest index of the largest.  None: the row has no distribution."""
    row = as64(row)
    if np.isnan(row).any() or (row == np.inf).any() or not np.isfinite(row).any():
        return None
    if temperature == 0:
        p = np.zeros_like(row)
        p[int(np.argmax(row))] = 1.0
        return p
    w = np.exp((row - row.max()) / float(temperature))
    return w / math.fsum(w)


def invert(weights, v):
    """min { i : sum_{k <= i} w_k > v sum w }."""
    c = np.cumsum(weights)
    i = int(np.searchsorted(c, v * c[-1], side="right"))
    return i if i < len(weights) else int(np.nonzero(weights)[0][-1])


def valid_uniform(u):
    return 0.0 <= u < 1.0


def draw(row, u, temperature):
    """(token, log p), or (-1, 0) where there is none."""
    p = probabilities(row, temperature)
    if p is None or (temperature != 0 and not valid_uniform(u)):
        return -1, 0.0
    i = invert(p, u if temperature else 0.0)
    return i, math.log(p[i])


def verify(target, draft, drafted, n_draft, uniform, temperature, draft_temperature):
    """One sequence: target [K + 1, V], draft [K, V] or None, drafted [K], uniform [K + 1].
    Returns (tokens, logprobs, accepted, why) with why one of '', 'logits', 'uniform', and whether a drafted
    token out of range stopped it."""
    V = target.shape[1]
    out, lps, bad_token = [], [], False
    j = 0
    while True:
        p = probabilities(target[j], temperature)
        if p is None:
            return out, lps, j, "logits", bad_token
        if j == n_draft:
            weights = p
            break
        x = int(drafted[j])
        q = None
        if temperature != 0 and 0 <= x < V and not valid_uniform(uniform[j]):
            return out, lps, j, "uniform", bad_token
        if temperature != 0:
            if draft is None:
                q = np.zeros(V)
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                q = probabilities(draft[j], draft_temperature)
                if q is None:
                    return out, lps, j, "logits", bad_token or not 0 <= x < V
        if 0 <= x < V and (p[x] == 1.0 if temperature == 0 else uniform[j] * q[x] < p[x]):
            out.append(x)
            lps.append(math.log(p[x]))
            j += 1
            continue
        bad_token = not 0 <= x < V
        weights = p if q is None else np.maximum(p - q, 0.0)
        if not weights.sum() > 0:
            weights = p
        break
    if temperature != 0 and not valid_uniform(uniform[-1]):
        return out, lps, j, "uniform", bad_token
    y = invert(weights, uniform[-1] if temperature else 0.0)
    return out + [y], lps + [math.log(p[y])], j, "", bad_token


def clip(arrays, max_norm):
    """(norm, coef, scaled arrays)."""
    a = [as64(x) for x in arrays]
    norm = math.sqrt(math.fsum(float(np.square(x).sum()) for x in a))
    coef = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return norm, coef, [x * coef for x in a]
