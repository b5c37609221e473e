"""Measured calls of the operators that reach from hidden states to an optimiser's update: log-probs of tokens from hidden
states and the weights of the vocabulary head, the gradient behind them, and the orthogonalisation of a set of updates.

`run` makes one call, in elementary torch operations (`own` False) or through this package's entry points (`own` True).

    logprob        z = h W^T,  lse = log sum_v exp z_v,  logprob = z_y - lse, for each row whose mask is 1 (others: 0)
    grad           G_nv = coef_n (exp(z_nv - lse_n) - [v = y_n]),  d_hidden = G W,  d_weight = G^T H
    orthogonalise  X = M / (|M| + eps),  five times  X <- (a + b X X^T + c (X X^T)^2) X,  out = scale X
"""
import math

import torch

own = False

DEV = "cuda:0"
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # one sequence's next token scored against a small head: a latency
        dict(name="logprob 1 row", op="logprob", rows=1, vocab=32000, dim=1024, pad=0, masked=0.0),
        # a decoding batch against a full vocabulary: bound by reading the weights
        dict(name="logprob 48 rows", op="logprob", rows=48, vocab=151936, dim=2048, pad=0, masked=0.0),
        # a padded chunk of responses, odd sizes, rows at a pitch
        dict(name="logprob 1500 rows ragged", op="logprob", rows=1500, vocab=70001, dim=1001, pad=7, masked=0.4),
        # every row of a chunk scored
        dict(name="logprob 4096 rows", op="logprob", rows=4096, vocab=151936, dim=2048, pad=0, masked=0.0),
        # the gradient of a few tokens with a small head
        dict(name="grad 100 rows", op="grad", rows=100, vocab=32000, dim=1024, pad=0, masked=0.0, weight_grad="bf16"),
        # a padded chunk, odd sizes, the weights' gradient in fp32 (as one that chunks add to)
        dict(name="grad 1500 rows ragged fp32", op="grad", rows=1500, vocab=32003, dim=1001, pad=7, masked=0.4, weight_grad="f32"),
        # a chunk of a training step
        dict(name="grad 4096 rows", op="grad", rows=4096, vocab=151936, dim=2048, pad=0, masked=0.0, weight_grad="bf16"),
        # one small matrix: a latency
        dict(name="orthogonalise one 256 x 1024 fp32", op="orthogonalise", layout="one", rows=256, width=1024, count=1, dtype="f32"),
        # adapters: pairs of thin matrices, wide and tall
        dict(name="orthogonalise adapters", op="orthogonalise", layout="adapters", rows=64, width=1025, count=48, dtype="bf16"),
        # experts of one layer: many middling matrices
        dict(name="orthogonalise experts", op="orthogonalise", layout="experts", rows=512, width=1024, count=32, dtype="bf16"),
        # the matrices of two blocks of a model
        dict(name="orthogonalise blocks", op="orthogonalise", layout="blocks", rows=1, width=2048, count=2, dtype="bf16"),
        # the same in fp32 throughout, odd sizes
        dict(name="orthogonalise blocks fp32", op="orthogonalise", layout="blocks", rows=1, width=1000, count=1, dtype="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprob", "grad", "orthogonalise"])
    if op == "orthogonalise":
        layout = rng.choice(["one", "adapters", "experts", "blocks"])
        width = {"one": _spread(rng, 1, 3000), "adapters": _spread(rng, 33, 3000), "experts": _spread(rng, 100, 1200),
                 "blocks": _spread(rng, 100, 1500)}[layout]
        return dict(op=op, layout=layout, width=width, dtype=rng.choice(["bf16", "f32"]),
                    rows={"one": _spread(rng, 1, 3000), "adapters": rng.randint(1, 130), "experts": _spread(rng, 50, 600), "blocks": 1}[layout],
                    count={"one": 1, "adapters": _spread(rng, 1, 100), "experts": _spread(rng, 2, 32), "blocks": rng.randint(1, 2)}[layout])
    vocab = rng.choice([32000, 128256, 151936, _spread(rng, 300, 160000)])
    dim = rng.choice([1024, 2048, _spread(rng, 48, 2500)])
    most = int(4096 * 151936 * 2048 / (vocab * dim))  # rows, so that no case is larger than the largest listed ones
    case = dict(op=op, rows=_spread(rng, 1, min(most, 4096)), vocab=vocab, dim=dim, pad=rng.choice([0, rng.randint(1, 30)]),
                masked=rng.choice([0.0, 0.0, round(rng.uniform(0.1, 0.9), 2)]))
    if op == "grad":
        case["weight_grad"] = rng.choice(["bf16", "f32"])
    return case


# ---- inputs ----------------------------------------------------------------------------------------

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows(n, dim, pad, scale, g):
    """[n, dim] in bf16, N(0, scale^2), rows at a pitch of whole 16-byte vectors."""
    x = torch.empty((n, -(-(dim + pad) // 8) * 8), dtype=torch.bfloat16, device=DEV)
    for at in range(0, n, 1 << 14):
        x[at:at + (1 << 14)] = torch.randn(x[at:at + (1 << 14)].shape, generator=g, device=DEV) * scale
    return x[:, :dim]


def _shapes(case):
    """Shapes of a set of matrices."""
    r, w, n = case["rows"], case["width"], case["count"]
    if case["layout"] == "one":
        return [(r, w)]
    if case["layout"] == "adapters":
        return [(r, w) if i % 2 else (w - i % 3, r) for i in range(n)]
    if case["layout"] == "experts":
        return [(r, w) if i % 4 else (w, r) for i in range(n)]
    return [(w, w), (w // 4, w), (w // 4, w), (w, w), (2 * w + w // 2, w), (2 * w + w // 2, w), (w, 2 * w + w // 2)] * n


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    if case["op"] == "orthogonalise":
        d = _DTYPES[case["dtype"]]
        s["matrices"], s["scales"] = [], []
        for m, n in _shapes(case):  # momentum: a few strong directions and noise
            k = min(8, m, n)
            x = torch.randn((m, k), generator=g, device=DEV) @ torch.randn((k, n), generator=g, device=DEV) / math.sqrt(k)
            x = (x * 0.5 + torch.randn((m, n), generator=g, device=DEV)) * 1e-3
            s["matrices"].append(x.to(d))
            s["scales"].append(math.sqrt(max(1.0, m / n)))
        s["outs"] = [torch.empty_like(x) for x in s["matrices"]]
        if own:  # the handle that a training program keeps beside its momenta
            from paper_2605_17862_b200 import binding as fb
            s["list"] = fb.MatrixList(s["matrices"], s["outs"], scales=s["scales"])
        return s
    N, V, D = case["rows"], case["vocab"], case["dim"]
    s["hidden"] = _rows(N, D, case["pad"], 1.0, g)
    s["weight"] = _rows(V, D, case["pad"], 3.0 / math.sqrt(D), g)  # logits ~ N(0, 3^2)
    s["tokens"] = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    s["mask"] = None
    if case["masked"]:  # the rows behind the responses
        s["mask"] = (torch.rand(N, generator=g, device=DEV) >= case["masked"]).to(torch.uint8)
    # a trained policy: every other token is a likely one (its logit near the largest)
    likely = torch.arange(0, N, 2, device=DEV)
    w = s["weight"][s["tokens"][likely].long()].float()
    s["hidden"][likely] += (w * (4.0 / w.square().sum(1, keepdim=True).clamp(min=1e-6).sqrt())).bfloat16()
    s["logprob"], s["lse"] = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    if case["op"] == "logprob":
        return s
    out = _plain_logprob(s)
    s["logprob"], s["lse"] = out["logprob"], out["lse"]
    s["coef"] = torch.rand(N, generator=g, device=DEV) / N
    s["d_hidden"] = torch.empty((N, -(-D // 8) * 8), dtype=torch.bfloat16, device=DEV)[:, :D]
    s["d_weight"] = torch.empty((V, -(-D // 8) * 8), dtype=_DTYPES[case["weight_grad"]], device=DEV)[:, :D]
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    if own:
        return _RUN_OWN[s["op"]](s)
    return _RUN_PLAIN[s["op"]](s)


def _own_logprob(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_head_logprob(s["hidden"], s["weight"], s["tokens"], s["logprob"], lse=s["lse"], mask=s["mask"])
    return {"logprob": s["logprob"], "lse": s["lse"]}


def _own_grad(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_head_grad(s["hidden"], s["weight"], s["tokens"], s["logprob"], s["lse"], s["coef"], d_hidden=s["d_hidden"],
                      d_weight=s["d_weight"], mask=s["mask"])
    return {"d_hidden": s["d_hidden"], "d_weight": s["d_weight"]}


def _own_orthogonalise(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_orthogonalise(s["list"], coefficients=[COEFFICIENTS] * STEPS, eps=EPS)
    return {"outs": s["outs"]}


_RUN_OWN = {"logprob": _own_logprob, "grad": _own_grad, "orthogonalise": _own_orthogonalise}


def _logits(s):
    """Logits in 32 bits; rows that are masked out are taken as zero."""
    h = s["hidden"].float()
    if s["mask"] is not None:
        h = h * s["mask"].unsqueeze(1)
    return h, h @ s["weight"].float().t()


def _plain_logprob(s):
    _, z = _logits(s)
    m = z.amax(1, keepdim=True)
    lse = (z - m).exp().sum(1, dtype=torch.float64).log() + m.squeeze(1)
    lp = z.gather(1, s["tokens"].long().unsqueeze(1)).squeeze(1) - lse
    if s["mask"] is not None:
        lse, lp = lse * s["mask"], lp * s["mask"]
    return {"logprob": lp.float(), "lse": lse.float()}


def _plain_grad(s):
    h, G = _logits(s)
    coef = s["coef"] if s["mask"] is None else s["coef"] * s["mask"]
    G = (G - s["lse"].unsqueeze(1)).exp_()
    G.scatter_add_(1, s["tokens"].long().unsqueeze(1), torch.full_like(coef, -1.0).unsqueeze(1))
    G *= coef.unsqueeze(1)
    return {"d_hidden": (G @ s["weight"].float()).to(s["d_hidden"].dtype), "d_weight": (G.t() @ h).to(s["d_weight"].dtype)}


def _plain_orthogonalise(s):
    a, b, c = COEFFICIENTS
    outs = []
    for M, scale in zip(s["matrices"], s["scales"]):
        X = M.float()
        X = X / (X.square().sum(dtype=torch.float64).sqrt().float() + EPS)
        if X.shape[0] > X.shape[1]:
            X = X.t()
        for _ in range(STEPS):
            A = X @ X.t()
            X = a * X + (b * A + c * (A @ A)) @ X
        if M.shape[0] > M.shape[1]:
            X = X.t()
        outs.append((X * scale).to(M.dtype).contiguous())
    return {"outs": outs}


_RUN_PLAIN = {"logprob": _plain_logprob, "grad": _plain_grad, "orthogonalise": _plain_orthogonalise}


# ---- what one pass cannot do without ----------------------------------------------------------------

def work(case):
    if case["op"] == "orthogonalise":
        size = 2 if case["dtype"] == "bf16" else 4
        flops = bytes_ = 0
        for m, n in _shapes(case):
            m, n = min(m, n), max(m, n)
            flops += STEPS * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)  # two of the products are symmetric
            bytes_ += 2 * size * m * n
        return {"bytes": bytes_, "flops": flops}
    N, V, D = max(1, round(case["rows"] * (1 - case["masked"]))), case["vocab"], case["dim"]
    if case["op"] == "logprob":
        return {"bytes": 2 * D * (N + V) + 12 * case["rows"], "flops": 2 * N * V * D}
    size = 2 if case["weight_grad"] == "bf16" else 4
    return {"bytes": 2 * D * (N + V) + 2 * D * case["rows"] + size * D * V + 16 * case["rows"], "flops": 6 * N * V * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalise":
        return {"outs": [_orthogonal(M.double(), scale) for M, scale in zip(s["matrices"], s["scales"])]}
    W, y = s["weight"].double(), s["tokens"].long()
    live = torch.arange(case["rows"], device=DEV) if s["mask"] is None else s["mask"].nonzero().squeeze(1)
    out = {}
    if case["op"] == "logprob":
        out["lse"], out["logprob"] = (torch.zeros(case["rows"], dtype=torch.float64, device=DEV) for _ in range(2))
    else:
        out["d_hidden"] = torch.zeros(s["hidden"].shape, dtype=torch.float64, device=DEV)
        out["d_weight"] = torch.zeros(s["weight"].shape, dtype=torch.float64, device=DEV)
    for at in range(0, len(live), 512):
        rows = live[at:at + 512]
        H = s["hidden"][rows].double()
        Z = torch.einsum("nd,vd->nv", H, W)
        if case["op"] == "logprob":
            out["lse"][rows] = torch.logsumexp(Z, 1)
            out["logprob"][rows] = torch.log_softmax(Z, 1)[torch.arange(len(rows), device=DEV), y[rows]]
            continue
        P = torch.exp(Z - s["lse"][rows].double()[:, None])
        P[torch.arange(len(rows), device=DEV), y[rows]] -= 1
        P = P * s["coef"][rows].double()[:, None]
        out["d_hidden"][rows] = torch.einsum("nv,vd->nd", P, W)
        out["d_weight"] += torch.einsum("nv,nd->vd", P, H)
    return out


def _orthogonal(M, scale):
    """scale times the polynomial of M, by the Gram matrix of its shorter side on whichever side that is."""
    X = M / (torch.linalg.norm(M) + EPS)
    one = torch.eye(min(M.shape), dtype=torch.float64, device=M.device)
    for _ in range(STEPS):
        gram = X @ X.mT if M.shape[0] <= M.shape[1] else X.mT @ X
        poly = COEFFICIENTS[0] * one + gram @ (COEFFICIENTS[1] * one + COEFFICIENTS[2] * gram)
        X = poly @ X if M.shape[0] <= M.shape[1] else X @ poly
    return X * scale
