"""Measured calls of the operators on either side of the loss: drawing tokens from rows of logits,
verifying drafted tokens against the target's probabilities, and clipping gradients by their global norm.

`run` makes one call, in elementary torch operations (`own` False) or through this package's entry
points (`own` True).  All three take given random numbers, so both sides give the same tokens:

    draw     the lowest i with  sum_{k <= i} p_k > v sum_k p_k,   p = softmax(logits / temperature);
             temperature 0 is the lowest index of the largest logit.
    verify   draft j of a sequence is accepted while  u_j q_j(x_j) < p_j(x_j); the first one that is not is
             replaced by a draw from max(p_j - q_j, 0) (from p_j where that is zero everywhere), and a
             sequence whose drafts were all accepted gets one more token, drawn from the row behind them.
    clip     norm = sqrt(sum of all squares), coef = min(1, max_norm / norm), every gradient times coef.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---- cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of one sequence: a latency
        dict(name="draw 1 row", op="draw", rows=1, vocab=151936, pad=0, dtype="bf16", temperature=0.7, banned=0.0),
        # a decoding batch whose vocabulary fills neither its last vector nor its row pitch; banned tokens are -inf
        dict(name="draw 48 rows fp32", op="draw", rows=48, vocab=70001, pad=7, dtype="f32", temperature=1.0, banned=0.1),
        # every row of a chunk of logits
        dict(name="draw 4096 rows", op="draw", rows=4096, vocab=151936, pad=0, dtype="bf16", temperature=1.0, banned=0.0),
        # one sequence with four drafts: a latency
        dict(name="verify 1 x 4", op="verify", seqs=1, drafts=4, ragged=False, vocab=151936, pad=0, dtype="bf16",
             temperature=1.0, noise=0.5, form="rows"),
        # a rollout batch whose sequences carry up to five drafts each
        dict(name="verify 64 x 5 ragged", op="verify", seqs=64, drafts=5, ragged=True, vocab=151936, pad=0, dtype="bf16",
             temperature=0.7, noise=0.5, form="rows"),
        # a large rollout batch with a close draft
        dict(name="verify 256 x 7", op="verify", seqs=256, drafts=7, ragged=False, vocab=128256, pad=0, dtype="bf16",
             temperature=1.0, noise=0.2, form="rows"),
        # stale responses checked against the policy that has moved on: few of the rows are reached
        dict(name="verify 16 x 256 stale", op="verify", seqs=16, drafts=256, ragged=True, vocab=151936, pad=0, dtype="bf16",
             temperature=1.0, noise=0.3, form="rows"),
        # drafts looked up rather than drawn, an odd vocabulary
        dict(name="verify 24 x 10 lookup fp32", op="verify", seqs=24, drafts=10, ragged=True, vocab=32003, pad=5, dtype="f32",
             temperature=1.0, noise=0.5, form="lookup"),
        # the gradients of small adapters: many small tensors, a latency
        dict(name="clip adapters", op="clip", layout="adapters", width=1024, rows=8, count=96, dtype="bf16", max_norm=0.3, place="out"),
        # the gradients of a model: matrices in bf16 and vectors in fp32, from one element up
        dict(name="clip model", op="clip", layout="model", width=2048, rows=32000, count=10, dtype="bf16", max_norm=1.0, place="out"),
        # the gradient with respect to the logits, chunk by chunk
        dict(name="clip logits", op="clip", layout="logits", width=151936, rows=4096, count=2, dtype="bf16", max_norm=0.5, place="out"),
        # a step whose norm is below the bound, in place: the gradients stay as they are
        dict(name="clip below the bound fp32", op="clip", layout="model", width=1024, rows=32000, count=12, dtype="f32", max_norm=1e9, place="in"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["draw", "verify", "clip"])
    dtype = rng.choice(["bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    if op == "clip":
        layout = rng.choice(["adapters", "model", "logits"])
        width = {"adapters": _spread(rng, 33, 4097), "model": _spread(rng, 65, 1500), "logits": _spread(rng, 1001, 160001)}[layout]
        count = {"adapters": _spread(rng, 1, 200), "model": _spread(rng, 1, 12), "logits": rng.randint(1, 3)}[layout]
        rows = {"adapters": rng.randint(1, 64), "model": _spread(rng, 100, 40000),
                "logits": _spread(rng, 2, min(4096, int(1.1e9 / (size * width * count))))}[layout]
        place = rng.choice(["out", "out", "in"])
        return dict(op=op, layout=layout, width=width, rows=rows, count=count, dtype=dtype, place=place,
                    max_norm=1e9 if place == "in" else round(math.exp(rng.uniform(-3.0, 0.0)), 4))
    vocab = rng.choice([32000, 128256, 151936, _spread(rng, 700, 160000)])
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    temperature = rng.choice([0.0, 1.0, round(rng.uniform(0.3, 1.5), 3)])
    most = int(1.1e9 / (vocab * size))  # rows, so that no case is larger than the largest listed ones
    if op == "draw":
        return dict(op=op, rows=_spread(rng, 1, min(4096, most)), vocab=vocab, pad=pad, dtype=dtype, temperature=temperature,
                    banned=rng.choice([0.0, 0.0, 0.3]))
    drafts = _spread(rng, 1, 64)
    return dict(op=op, seqs=_spread(rng, 1, max(1, min(256, most // (2 * drafts + 1)))), drafts=drafts, ragged=rng.random() < 0.5,
                vocab=vocab, pad=pad, dtype=dtype, temperature=temperature, noise=round(rng.uniform(0.1, 1.0), 3),
                form=rng.choice(["rows", "rows", "lookup"]))


# ---- inputs ----------------------------------------------------------------------------------------

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _pitch(case):
    """Columns of a row of logits with its padding: whole 16-byte vectors, as the rows' layout wants."""
    per = 8 if case["dtype"] == "bf16" else 4
    return -(-(case["vocab"] + case["pad"]) // per) * per


def _logits(rows, case, g):
    """N(0, 3^2) with 1 % of the entries boosted by 8; the padding behind a row is left arbitrary."""
    x = torch.empty((rows, _pitch(case)), dtype=_DTYPES[case["dtype"]], device=DEV)
    for at in range(0, rows, 512):
        y = torch.randn(x[at:at + 512].shape, generator=g, device=DEV) * 3
        y += 8.0 * (torch.rand(y.shape, generator=g, device=DEV) < 0.01)
        x[at:at + 512] = y
    return x


def _tensors(case):
    """Shapes and types of a set of gradients."""
    w, r, n, d = case["width"], case["rows"], case["count"], case["dtype"]
    if case["layout"] == "adapters":  # pairs of thin matrices
        return [((r, w), d) if i % 2 else ((w - i % 3, r), d) for i in range(n)]
    if case["layout"] == "logits":  # chunks of rows, the last ones shorter
        return [((max(1, r - (r // 8 + 1) * i), w), d) for i in range(n)]
    shapes = [((r, w), d), ((1,), "f32")]
    for _ in range(n):
        shapes += [((w,), "f32"), ((w + w // 2, w), d), ((w + w // 2,), "f32"), ((w, w), d), ((w,), "f32"),
                   ((2 * (2 * w + 11), w), d), ((w, 2 * w + 11), d)]
    return shapes + [((w,), "f32"), ((r, w), d)]


def _flat(case, g):
    """The gradients as views of one buffer for each type, one after another (a tensor may start at any element)."""
    shapes = _tensors(case)
    flat = {k: torch.empty(sum(math.prod(s) for s, d in shapes if d == k), dtype=_DTYPES[k], device=DEV) for k in ("bf16", "f32")
            if any(d == k for _, d in shapes)}
    if g is not None:
        scale = math.exp(float(torch.rand((), generator=g, device=DEV)) * 2 - 7)
        for x in flat.values():
            for at in range(0, x.numel(), 1 << 26):
                x[at:at + (1 << 26)] = torch.randn(min(1 << 26, x.numel() - at), generator=g, device=DEV) * scale
    at, views = {k: 0 for k in flat}, []
    for s, d in shapes:
        views.append(flat[d][at[d]:at[d] + math.prod(s)].view(s))
        at[d] += math.prod(s)
    return flat, views


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    if case["op"] == "clip":
        s["flat"], s["grads"] = _flat(case, g)
        s["out_flat"], s["outs"] = (s["flat"], s["grads"]) if case["place"] == "in" else _flat(case, None)
        s["norm"], s["coef"] = (torch.empty(1, device=DEV) for _ in range(2))
        if own:  # the handle and the workspace that a training program keeps beside its gradients
            from paper_2605_17862_b200 import binding as fb
            s["list"] = fb.GradientList(s["grads"], None if case["place"] == "in" else s["outs"])
            s["ws"] = fb.grad_workspace(DEV)
        return s
    V = case["vocab"]
    if case["op"] == "draw":
        n = case["rows"]
        s["logits"] = _logits(n, case, g)[:, :V]
        if case["banned"]:
            s["logits"][:, torch.rand(V, generator=g, device=DEV) < case["banned"]] = -math.inf
        s["uniform"] = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
        s["tokens"], s["logprob"] = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
        return s
    B, K, T = case["seqs"], case["drafts"], case["temperature"]
    target = _logits(B * (K + 1), case, g).view(B, K + 1, -1)
    draft = torch.empty((B, K, target.shape[2]), dtype=target.dtype, device=DEV)
    tokens = torch.empty((B, K), dtype=torch.int32, device=DEV)
    for b in range(B):  # the drafting model is the target with noise; its tokens are drawn from it at the same temperature
        for at in range(0, K, 256):
            x = target[b, at:min(K, at + 256)].float()
            x += case["noise"] * torch.randn(x.shape, generator=g, device=DEV)
            draft[b, at:at + 256] = x
            z = draft[b, at:at + 256, :V].float()
            if T:
                z = z / T - torch.empty(z.shape, device=DEV).exponential_(generator=g).log_()
            tokens[b, at:at + 256] = z.argmax(-1)
    if case["form"] == "lookup":  # a looked-up token is there because the text repeats itself: the target has about even odds on it
        target.scatter_(2, torch.nn.functional.pad(tokens, (0, 1)).long().unsqueeze(2), math.log(V) + 8.0)
    s["target"], s["draft"] = target[:, :, :V], draft[:, :, :V] if case["form"] == "rows" else None
    s["draft_tokens"] = tokens
    s["n_draft"] = torch.randint(K // 2, K + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if case["ragged"] else None
    s["uniform"] = torch.rand((B, K + 1), generator=g, device=DEV, dtype=torch.float64)
    s["tokens"] = torch.empty((B, K + 1), dtype=torch.int32, device=DEV)
    s["logprob"] = torch.empty((B, K + 1), device=DEV)
    s["mask"] = torch.empty((B, K + 1), dtype=torch.uint8, device=DEV)
    s["accepted"] = torch.empty(B, dtype=torch.int32, device=DEV)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    if own:
        return _RUN_OWN[s["op"]](s)
    return _RUN_PLAIN[s["op"]](s)


def _own_draw(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_draw_tokens(s["logits"], s["uniform"], s["tokens"], logprob=s["logprob"], temperature=s["temperature"])
    return {"tokens": s["tokens"], "logprob": s["logprob"]}


def _own_verify(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_verify_draft(s["target"], s["draft"], s["draft_tokens"], s["uniform"], s["tokens"], n_draft=s["n_draft"],
                         logprob=s["logprob"], mask=s["mask"], n_accepted=s["accepted"], temperature=s["temperature"],
                         draft_temperature=s["temperature"])
    return {k: s[k] for k in ("tokens", "logprob", "mask", "accepted")}


def _own_clip(s):
    from paper_2605_17862_b200 import binding as fb
    fb.fopd_grad_clip(s["list"], s["max_norm"], s["ws"], norm=s["norm"], coef=s["coef"])
    return {"norm": s["norm"], "coef": s["coef"], "grads": s["out_flat"]}


_RUN_OWN = {"draw": _own_draw, "verify": _own_verify, "clip": _own_clip}


def _inverse(w, v):
    """The lowest index whose running sum of the weights (64 bits) passes v times their total."""
    c = w.cumsum(-1)
    return (c <= (v * c[:, -1]).unsqueeze(-1)).sum(-1).clamp(max=w.shape[-1] - 1)


def _weights64(x, T):
    x = x.double()
    return ((x - x.amax(-1, keepdim=True)) / T).exp()


def _plain_draw(s):
    x, T = s["logits"], s["temperature"]
    if T == 0:
        token = x.float().argmax(-1)
        return {"tokens": token.int(), "logprob": torch.zeros(len(token), device=x.device)}
    w = _weights64(x, T)
    token = _inverse(w, s["uniform"])
    lp = (w.gather(1, token.unsqueeze(1)).squeeze(1) / w.sum(-1)).log()
    return {"tokens": token.int(), "logprob": lp.float()}


def _log_sums(x, T):
    """Maximum and log of the sum of exponentials behind it of every row: exponentials in 32 bits, their sum in 64."""
    x = x.float()
    m = x.amax(-1, keepdim=True)
    return m.squeeze(-1).double(), ((x - m) / T).exp().sum(-1, dtype=torch.float64).log()


def _plain_verify(s):
    target, draft, drafted, T = s["target"], s["draft"], s["draft_tokens"].long(), s["temperature"]
    B, K = drafted.shape
    here = torch.arange(K + 1, device=target.device)
    n_draft = s["n_draft"].long() if s["n_draft"] is not None else torch.full((B,), K, device=target.device)
    u, v = s["uniform"][:, :K], s["uniform"][:, K]
    if T == 0:
        best = target.float().argmax(-1)
        ok = drafted == best[:, :K]
        accepted = (ok & (here[:K] < n_draft.unsqueeze(1))).int().cumprod(1).sum(1)
        new = best.gather(1, accepted.unsqueeze(1)).squeeze(1)
        row_lp = torch.zeros((B, K + 1), dtype=torch.float64, device=target.device)
        last_lp = row_lp[:, 0]
    else:
        m, z = _log_sums(target, T)
        x = target[:, :K].gather(2, drafted.unsqueeze(2)).squeeze(2).double()
        row_lp = (x - m[:, :K]) / T - z[:, :K]
        q = torch.ones_like(row_lp)
        if draft is not None:
            mq, zq = _log_sums(draft, T)
            q = ((draft.gather(2, drafted.unsqueeze(2)).squeeze(2).double() - mq) / T - zq).exp()
        ok = u * q < row_lp.exp()
        accepted = (ok & (here[:K] < n_draft.unsqueeze(1))).int().cumprod(1).sum(1)
        seq = torch.arange(B, device=target.device)
        p = _weights64(target[seq, accepted], T)
        p = p / p.sum(-1, keepdim=True)
        at = accepted.clamp(max=K - 1)
        if draft is not None:
            q = _weights64(draft[seq, at], T)
            q = q / q.sum(-1, keepdim=True)
        else:
            q = torch.zeros_like(p).scatter_(1, drafted[seq, at].unsqueeze(1), 1.0)
        rest = (p - q).clamp(min=0)
        from_rest = (accepted < n_draft) & (rest.sum(-1) > 0)
        new = _inverse(torch.where(from_rest.unsqueeze(1), rest, p), v)
        last_lp = p.gather(1, new.unsqueeze(1)).squeeze(1).log()
        row_lp = torch.cat([row_lp, torch.zeros_like(row_lp[:, :1])], 1)
    a = accepted.unsqueeze(1)
    kept, last = here < a, here == a
    tokens = torch.cat([drafted, torch.zeros_like(drafted[:, :1])], 1)
    tokens = torch.where(kept, tokens, torch.where(last, new.unsqueeze(1), -1))
    lp = torch.where(kept, row_lp, torch.where(last, last_lp.unsqueeze(1), 0.0))
    return {"tokens": tokens.int(), "logprob": lp.float(), "mask": (kept | last).to(torch.uint8), "accepted": accepted.int()}


def _plain_clip(s):
    sums = torch.stack([x.float().square().sum(dtype=torch.float64) for x in s["grads"]])
    norm = sums.sum().sqrt()
    coef = (s["max_norm"] / norm).clamp(max=1.0).float()
    [o.copy_(x.float() * coef) for x, o in zip(s["grads"], s["outs"])]
    return {"norm": norm.float().reshape(1), "coef": coef.reshape(1), "grads": s["out_flat"]}


_RUN_PLAIN = {"draw": _plain_draw, "verify": _plain_verify, "clip": _plain_clip}


# ---- what one pass cannot do without ----------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "clip":
        n = sum(math.prod(s) for s, _ in _tensors(case))
        e = sum(math.prod(s) * (2 if d == "bf16" else 4) for s, d in _tensors(case))
        return {"bytes": e if case["place"] == "in" else 2 * e, "flops": 2 * n if case["place"] == "in" else 3 * n}
    V = case["vocab"]
    if case["op"] == "draw":
        return {"bytes": case["rows"] * (V * size + 16), "flops": 3 * case["rows"] * V}
    # A draft is accepted with probability 1 - TV(p, q).  For the target's logits with noise N(0, s^2) / T on top that is
    # 1 - erf(s / (2 sqrt 2 T)); a looked-up one with its own probability, about one half.  Rows behind the first rejection
    # are not needed, nor a draft's rows at temperature 0.
    K, T = case["drafts"], case["temperature"]
    K = 0.75 * K if case["ragged"] else K
    if case["form"] == "lookup" or T == 0:
        a = 0.5 if T else 0.9 if case["form"] == "lookup" else max(0.0, 1 - 0.6 * case["noise"])
    else:
        a = 1 - math.erf(case["noise"] / (2 * math.sqrt(2) * T))
    reached = (1 - a ** (K + 1)) / (1 - a)
    drafts = (1 - a ** K) / (1 - a) if case["form"] == "rows" and T else 0.0
    B = case["seqs"]
    return {"bytes": B * ((reached + drafts) * V * size + (case["drafts"] + 1) * 21), "flops": 3 * B * (reached + drafts) * V}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _pick(prob, v):
    """Inverse of the distribution function of one row of probabilities."""
    c = torch.cumsum(prob, 0)
    return min(int(torch.searchsorted(c, v * c[-1:], right=True)), prob.numel() - 1)


def _prob(row, T):
    """Probabilities of one row of logits: softmax at a temperature, all on the first largest where that is 0."""
    row = row.double()
    if T == 0:
        p = torch.zeros_like(row)
        p[int((row == row.max()).nonzero()[0])] = 1.0
        return p
    return torch.softmax(row / T, 0)


def exact(case, seed):
    s = prepare(case, seed)
    T = case.get("temperature")
    if case["op"] == "draw":
        if case["rows"] > 8192:
            return None
        tokens, lps = [], []
        for row, v in zip(s["logits"], s["uniform"]):
            p = _prob(row, T)
            tokens.append(_pick(p, v))
            lps.append(p[tokens[-1]].log())
        return {"tokens": torch.tensor(tokens, dtype=torch.int32), "logprob": torch.stack(lps)}
    if case["op"] == "verify":
        B, K = s["draft_tokens"].shape
        out = {"tokens": torch.full((B, K + 1), -1, dtype=torch.int32), "logprob": torch.zeros((B, K + 1), dtype=torch.float64),
               "mask": torch.zeros((B, K + 1), dtype=torch.uint8), "accepted": torch.zeros(B, dtype=torch.int32)}
        for b in range(B):
            n = int(s["n_draft"][b]) if s["n_draft"] is not None else K
            j = 0
            while True:
                p = _prob(s["target"][b, j], T)
                if j == n:
                    rest = p
                    break
                x = int(s["draft_tokens"][b, j])
                if s["draft"] is not None:
                    q = _prob(s["draft"][b, j], T)
                else:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                # (a greedy target: p is 0 or 1 and the draft's own probability decides nothing)
                if not bool(s["uniform"][b, j] * q[x] < p[x]):
                    rest = torch.clamp(p - q, min=0)
                    if not bool(rest.sum() > 0):
                        rest = p
                    break
                out["tokens"][b, j], out["logprob"][b, j] = x, p[x].log().cpu()
                j += 1
            y = _pick(rest, s["uniform"][b, K])
            out["tokens"][b, j], out["logprob"][b, j], out["accepted"][b] = y, p[y].log().cpu(), j
            out["mask"][b, :j + 1] = 1
        return out
    total = sum(x[at:at + (1 << 26)].double().pow(2).sum() for x in s["flat"].values() for at in range(0, x.numel(), 1 << 26))
    norm = torch.sqrt(total)
    coef = min(1.0, case["max_norm"] / float(norm))
    return {"norm": norm.reshape(1), "coef": torch.tensor([coef], dtype=torch.float64),
            "grads": {k: x.double() * coef for k, x in s["flat"].items()}}
