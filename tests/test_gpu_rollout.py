"""GPU tests of fopd_draw_tokens and fopd_verify_draft against the fp64 definitions in
oracle/rollout_oracle.py.  Tokens, masks and counts are compared exactly.

Log-probabilities: log p = (x - max) / T - log Z with the first term in fp64 and Z from the fp32 sweep, whose
relative error is at most 7.5e-6 (three roundings in an exponent above -24, ex2, 69 additions: 3.1e-6 + 0.3e-6 + 4.1e-6);
the result is rounded to fp32 once, 2^-24 |log p|."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2605_17862_b200 import binding as fb
from paper_2605_17862_b200 import pipeline as pl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
TOP = 1 - 2.0 ** -53


def lp_tol(lp):
    return 7.5e-6 + 2.0 ** -24 * np.abs(lp)


def rows_of(shape, V, dtype, seed, pad=None, scale=3.0):
    """N(0, scale^2) logits at a pitch of whole vectors; what lies behind V is NaN."""
    per = 8 if dtype == BF16 else 4
    pitch = -(-(V + (pad or 0)) // per) * per
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.full((*shape, pitch), math.nan, device=DEV, dtype=dtype)
    x[..., :V] = torch.randn((*shape, V), generator=g, device=DEV) * scale
    return x[..., :V]


def uniforms(shape, seed):
    return torch.rand(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV, dtype=torch.float64)


def run_draw(x, u, T, vocab=None):
    n = x.shape[0]
    tokens = torch.full((n,), 77, dtype=torch.int32, device=DEV)
    lp = torch.full((n,), 77.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    fb.fopd_draw_tokens(x, u, tokens, logprob=lp, temperature=T, vocab=vocab, status=status)
    return tokens, lp, int(status.cpu()[0])


def check_draw(x, u, T, bits=0):
    tokens, lp, got_bits = run_draw(x, u, T)
    want = [ro.draw(r, float(v), T) for r, v in zip(x.cpu(), u.cpu())]
    assert got_bits == bits
    assert tokens.cpu().tolist() == [w[0] for w in want]
    wl = np.array([w[1] for w in want])
    assert np.all(np.abs(lp.cpu().numpy() - wl) <= lp_tol(wl))
    return tokens


def run_verify(target, draft, drafted, u, *, n_draft=None, T=1.0, Td=1.0):
    B, W = target.shape[:2]
    out = dict(tokens=torch.full((B, W), 77, dtype=torch.int32, device=DEV), logprob=torch.full((B, W), 77.0, device=DEV),
               mask=torch.full((B, W), 77, dtype=torch.uint8, device=DEV),
               n_accepted=torch.full((B,), 77, dtype=torch.int32, device=DEV))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tokens = out["tokens"]
    fb.fopd_verify_draft(target, draft, drafted, u, tokens, n_draft=n_draft, logprob=out["logprob"], mask=out["mask"],
                         n_accepted=out["n_accepted"], temperature=T, draft_temperature=Td, status=status)
    return {k: v.cpu().numpy() for k, v in out.items()}, int(status.cpu()[0])


def check_verify(target, draft, drafted, u, *, n_draft=None, T=1.0, Td=1.0):
    got, bits = run_verify(target, draft, drafted, u, n_draft=n_draft, T=T, Td=Td)
    B, W = target.shape[:2]
    K = W - 1
    t, d = target.cpu(), None if draft is None else draft.cpu()
    xs, us = drafted.cpu().numpy(), u.cpu().numpy()
    want_bits = 0
    for b in range(B):
        n = K if n_draft is None else int(n_draft[b])
        if not 0 <= n <= K:
            n = min(max(n, 0), K)
            want_bits |= 8
        tokens, lps, acc, why, bad_token = ro.verify(t[b], None if d is None else d[b], xs[b], n, us[b], T, Td)
        want_bits |= {"": 0, "logits": 32, "uniform": 64}[why] | (1 if bad_token else 0)
        m = len(tokens)
        assert got["n_accepted"][b] == acc, b
        assert got["tokens"][b].tolist() == tokens + [-1] * (W - m), b
        assert got["mask"][b].tolist() == [1] * m + [0] * (W - m), b
        assert np.all(np.abs(got["logprob"][b, :m] - np.array(lps)) <= lp_tol(np.array(lps))), b
        assert np.all(got["logprob"][b, m:] == 0)
    assert bits == want_bits
    return got


def drafts_from(draft, Td, seed):
    """Tokens drawn from the draft's rows (its distribution decides how many are accepted)."""
    B, K, V = draft.shape
    z = draft.float()
    if Td:
        g = torch.Generator(device=DEV).manual_seed(seed)
        z = z / Td - torch.empty(z.shape, device=DEV).exponential_(generator=g).log()
    return z.argmax(-1).int()


# ---- draws ----

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 33, 257, 1023, 1025, 2047, 2049, 4099, 20001])
def test_draw_odd_vocabularies(V, dtype):
    for T in (1.0, 0.3, 0.0):
        check_draw(rows_of((19,), V, dtype, V, pad=V % 11), uniforms(19, V + 1), T)


@pytest.mark.parametrize("V,dtype,n", [(151936, BF16, 40), (128256, F32, 12), (70001, BF16, 1)])
def test_draw_large_vocabularies(V, dtype, n):
    x = rows_of((n,), V, dtype, 5)
    x[:, ::101] += 8
    for T in (0.7, 1.0, 1.6):
        check_draw(x, uniforms(n, 9), T)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_draw_flat_rows_where_no_probability_exceeds_the_sum_error(dtype):
    """All probabilities near 1/V: the fp32 running sums do not decide any of these."""
    V = 151936
    x = rows_of((24,), V, dtype, 3, scale=0.02)
    check_draw(x, uniforms(24, 4), 1.0)
    # exactly even weights: a running sum that equals v times the total is not passed yet
    even = torch.full((5, 4096), 1.5, device=DEV, dtype=dtype)
    u = torch.tensor([0.0, 0.25, 0.25 - 2.0 ** -40, 4095 / 4096, TOP], device=DEV, dtype=torch.float64)
    assert check_draw(even, u, 1.0).tolist() == [0, 1024, 1023, 4095, 4095]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_draw_at_the_ends_of_the_unit_interval_and_at_boundaries(dtype):
    V = 5003
    x = rows_of((6,), V, dtype, 11)
    u = torch.tensor([0.0, 1e-300, 1e-12, 0.5, 1 - 1e-12, TOP], device=DEV, dtype=torch.float64)
    check_draw(x, u, 1.0)
    # just below and just above a boundary of the fp64 distribution function (by 1e-11, a thousand times its error)
    row = x[:1].expand(8, V).contiguous()
    per = -(-V // 8) * 8
    wide = torch.zeros(8, per, device=DEV, dtype=dtype)
    wide[:, :V] = row
    c = np.cumsum(ro.probabilities(row[0].cpu(), 1.0))
    ids = [10, 999, 2500, 4444]
    u = torch.tensor([c[i] + s for i in ids for s in (-1e-11, 1e-11)], device=DEV, dtype=torch.float64)
    check_draw(wide[:, :V], u, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_draw_masked_logits(dtype):
    low = torch.finfo(dtype).min
    V, n = 3001, 10
    x = rows_of((n,), V, dtype, 21)
    x[0, :] = -math.inf
    x[0, 2999] = 3.0            # one token left
    x[1, :2998] = -math.inf     # everything but the end
    x[2, 5:] = -math.inf        # everything but the beginning
    x[3, ::2] = -math.inf
    x[4, :] = low               # the lowest value everywhere is an even row
    x[5, 1:] = low              # ... and no weight beside a real one
    x[6, ::3] = low
    x[7, :] = -300.0
    x[8, :] += 5000.0
    x[9, 7] = 90.0              # all the weight on one token
    for T in (1.0, 0.5, 0.0):
        check_draw(x, uniforms(n, 22), T)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1.0, 0.0])
def test_draw_rows_without_a_distribution(dtype, T):
    x = rows_of((6,), 2500, dtype, 31)
    x[0, 2400] = math.nan
    x[1, 3] = math.inf
    x[2, :] = -math.inf
    x[4, :] = -math.inf
    x[4, 70] = math.nan
    check_draw(x, uniforms(6, 32), T, bits=32)
    y = rows_of((4,), 100, dtype, 33)
    u = torch.tensor([-1e-9, 1.0, math.nan, 0.5], device=DEV, dtype=torch.float64)
    check_draw(y, u, T, bits=64 if T else 0)


def test_draw_vocab_argument_no_rows_and_optional_outputs():
    x = rows_of((3,), 64, F32, 41)
    tokens, lp, bits = run_draw(x, uniforms(3, 42), 1.0, vocab=10)
    assert bits == 0 and [ro.draw(r[:10], float(v), 1.0)[0] for r, v in zip(x.cpu(), uniforms(3, 42).cpu())] == tokens.tolist()
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    fb.fopd_draw_tokens(x[:0], uniforms(0, 1), none)
    fb.fopd_draw_tokens(x, uniforms(3, 42), tokens)


def test_draw_rows_behind_the_32_bit_offsets():
    """16,400 rows of 151,936: the last ones start beyond 2^31 elements."""
    n, V = 16400, 151936
    x = torch.zeros((n, V), device=DEV, dtype=BF16)
    tail = rows_of((8,), V, BF16, 51)
    x[-8:] = tail
    u = uniforms(n, 52)
    tokens, lp, bits = run_draw(x, u, 1.0)
    assert bits == 0
    want = [ro.draw(r, float(v), 1.0)[0] for r, v in zip(tail.cpu(), u[-8:].cpu())]
    assert tokens[-8:].tolist() == want
    # even rows: token = floor(v V)
    assert torch.equal(tokens[:-8].long(), (u[:-8] * V).floor().long())


# ---- verification ----

@pytest.mark.parametrize("dtype,V", [(BF16, 9), (F32, 9), (BF16, 2050), (F32, 1030), (BF16, 32000)])
@pytest.mark.parametrize("form", ["rows", "certain", "best"])
@pytest.mark.parametrize("K", [1, 3, 8])
def test_verify_forms(dtype, V, form, K):
    B, T = 12, 0.8
    target = rows_of((B, K + 1), V, dtype, V + K, pad=5)
    draft = rows_of((B, K), V, dtype, 1, pad=13)
    draft += target[:, :K] - 0.6 * draft  # near the target's
    Td = 0.0 if form == "best" else 1.2
    drafted = drafts_from(draft, Td, 7)
    if form == "certain":
        drafted[:, ::2] = target[:, :K].argmax(-1).int()[:, ::2]
    n_draft = torch.randint(0, K + 1, (B,), device=DEV, dtype=torch.int32)
    n_draft[0], n_draft[1] = 0, K
    d = None if form == "certain" else draft
    got = check_verify(target, d, drafted, uniforms((B, K + 1), 8), n_draft=n_draft, T=T, Td=Td)
    check_verify(target, d, drafted, uniforms((B, K + 1), 9), T=T, Td=Td)
    assert got["n_accepted"].max() <= K


def test_verify_large_vocabulary():
    B, K, V = 6, 5, 151936
    target = rows_of((B, K + 1), V, BF16, 61)
    target[:, :, ::97] += 8
    draft = (target[:, :K].float() + 0.4 * rows_of((B, K), V, F32, 62, scale=1.0)).to(BF16)
    got = check_verify(target, draft, drafts_from(draft, 1.0, 63), uniforms((B, K + 1), 64))
    assert 0 < got["n_accepted"].sum() < B * K


def test_verify_temperature_zero_takes_the_best_tokens():
    B, K, V = 9, 4, 700
    target = rows_of((B, K + 1), V, BF16, 71)
    best = target[:, :K].argmax(-1).int()
    for k in range(K):
        best[k, k] = (best[k, k] + 1) % V
    u = torch.full((B, K + 1), math.nan, device=DEV, dtype=torch.float64)  # not needed
    got = check_verify(target, None, best, u, T=0.0)
    assert got["n_accepted"].tolist() == [0, 1, 2, 3] + [4] * (B - 4)
    nan = torch.full((B, K, V + 4), math.nan, device=DEV, dtype=BF16)[:, :, :V]  # neither are the draft's rows
    assert np.array_equal(check_verify(target, nan, best, u, T=0.0, Td=0.0)["tokens"], got["tokens"])


def test_verify_ties_and_equal_rows():
    """u q = p exactly is a rejection; a draft equal to the target is always accepted; a drafted token that neither
    can give leaves no residual and the token comes from p."""
    V = 4096
    even = torch.zeros((5, 2, V), device=DEV, dtype=F32)
    draft = torch.zeros((5, 1, V), device=DEV, dtype=F32)
    draft[:4, :, V // 2:] = -math.inf  # q = 2 / V on the lower half: accepted below u = 1/2
    draft[4] = even[4, :1]
    drafted = torch.tensor([[5], [5], [5], [V - 1], [17]], device=DEV, dtype=torch.int32)
    u = torch.tensor([[0.5, 0.0], [0.5 - 2.0 ** -40, 0.5], [0.5, TOP], [TOP, 0.3], [TOP, 0.9]], device=DEV, dtype=torch.float64)
    got = check_verify(even, draft, drafted, u)
    assert got["n_accepted"].tolist() == [0, 1, 0, 1, 1]
    assert got["tokens"][0, 0] == V // 2 and got["tokens"][2, 0] == V - 1
    target = rows_of((3, 2), 999, BF16, 81)
    target[:, 0, 300:] = -math.inf
    d = target[:, :1].contiguous()
    wide = torch.zeros((3, 1, 1000), device=DEV, dtype=BF16)
    wide[:, :, :999] = d
    got = check_verify(target, wide[:, :, :999], torch.full((3, 1), 500, dtype=torch.int32, device=DEV), uniforms((3, 2), 82))
    assert got["n_accepted"].tolist() == [0, 0, 0] and got["tokens"][:, 0].max() < 300


def test_verify_rows_that_are_not_reached_may_hold_anything():
    B, K, V = 4, 6, 1500
    target, draft = rows_of((B, K + 1), V, F32, 91), rows_of((B, K), V, F32, 92)
    drafted = drafts_from(draft, 1.0, 93)
    u = uniforms((B, K + 1), 94)
    first = check_verify(target, draft, drafted, u)
    assert first["n_accepted"].max() < K - 1  # unrelated drafts are soon rejected
    for b in range(B):
        a = int(first["n_accepted"][b])
        target[b, a + 1:] = math.nan
        draft[b, a + 1:] = math.inf
        drafted[b, a + 1:] = -5
        u[b, a + 1:K] = math.nan
    again, bits = run_verify(target, draft, drafted, u)
    assert bits == 0 and all(np.array_equal(first[k], again[k]) for k in first)


def test_verify_bad_rows_numbers_tokens_and_lengths():
    B, K, V = 12, 3, 777
    target, draft = rows_of((B, K + 1), V, F32, 101), rows_of((B, K), V, F32, 102)
    draft[:] = target[:, :K]  # everything is accepted where nothing is wrong
    drafted = drafts_from(draft, 1.0, 103)
    u = uniforms((B, K + 1), 104)
    n_draft = torch.full((B,), K, dtype=torch.int32, device=DEV)
    target[0, 1, 5] = math.nan
    target[1, 3, 700] = math.inf
    draft[2, 2, 9] = math.nan
    draft[3, 0, :] = -math.inf
    u[4, 1] = 1.0
    u[5, K] = -0.5
    drafted[6, 1] = V
    drafted[7, 0] = -1
    n_draft[8], n_draft[9] = -2, K + 4
    got = check_verify(target, draft, drafted, u, n_draft=n_draft)
    assert got["n_accepted"].tolist() == [1, 3, 2, 0, 1, 3, 1, 0, 0, 3, 3, 3]
    check_verify(target, None, drafted, u, n_draft=n_draft)
    check_verify(target, draft, drafted, u, n_draft=n_draft, Td=0.0)
    check_verify(target, draft, drafted, u, n_draft=n_draft, T=0.0)


def test_verify_without_drafts_is_a_draw():
    x, u = rows_of((7, 1), 3333, BF16, 111), uniforms((7, 1), 112)
    got = check_verify(x, None, torch.empty((7, 0), dtype=torch.int32, device=DEV), u)
    assert got["tokens"][:, 0].tolist() == run_draw(x[:, 0], u[:, 0].contiguous(), 1.0)[0].tolist()


@pytest.mark.parametrize("B,K,V,close", [(3, 300, 520, 0.05), (2, 1000, 130, 0.005), (40, 64, 2100, 0.1)])
def test_verify_long_drafts(B, K, V, close):
    target = rows_of((B, K + 1), V, BF16, K)
    draft = (target[:, :K].float() + close * torch.randn((B, K, V), device=DEV)).to(BF16)
    per = -(-V // 8) * 8
    wide = torch.zeros((B, K, per), device=DEV, dtype=BF16)
    wide[:, :, :V] = draft
    got = check_verify(target, wide[:, :, :V], drafts_from(draft, 1.0, 3), uniforms((B, K + 1), 4))
    assert got["n_accepted"].max() > 3


def test_verify_strides():
    """Sequences interleaved with each other, rows within a wider buffer, one draft row for all sequences."""
    B, K, V = 5, 4, 300
    big = rows_of((K + 1, 2 * B, 3), V, F32, 121)
    target = big[:, ::2, 1].transpose(0, 1)
    assert target.shape == (B, K + 1, V) and not target.is_contiguous()
    draft = rows_of((1, K), V, F32, 122).expand(B, K, V)
    drafted = drafts_from(draft, 1.0, 123)
    check_verify(target, draft, drafted, uniforms((B, K + 1), 124), T=2.0, Td=1.5)


def test_rollout_calls_on_a_side_stream_in_a_graph_and_at_the_same_time():
    B, K, V = 6, 4, 30001
    target, draft = rows_of((B, K + 1), V, BF16, 131), rows_of((B, K), V, BF16, 132)
    draft += target[:, :K] * 0.9 - draft * 0.6
    drafted, u = drafts_from(draft, 1.0, 133), uniforms((B, K + 1), 134)
    want, _ = run_verify(target, draft, drafted, u)
    rows = rows_of((300,), V, BF16, 135)
    ur = uniforms(300, 136)
    want_rows = run_draw(rows, ur, 1.0)[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for k in range(12):
        s = streams[k % 3]
        with torch.cuda.stream(s):
            t = torch.empty((B, K + 1), dtype=torch.int32, device=DEV)
            r = torch.empty(300, dtype=torch.int32, device=DEV)
            fb.fopd_verify_draft(target, draft, drafted, u, t, stream=s)
            fb.fopd_draw_tokens(rows, ur, r, stream=s)
            outs.append((t, r))
    torch.cuda.synchronize()
    for t, r in outs:
        assert np.array_equal(t.cpu().numpy(), want["tokens"]) and torch.equal(r, want_rows)
    # captured once, replayed on new inputs; two graphs whose temporaries must not be each other's
    t1, t2 = (torch.empty((B, K + 1), dtype=torch.int32, device=DEV) for _ in range(2))
    r1 = torch.empty(300, dtype=torch.int32, device=DEV)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        fb.fopd_verify_draft(target, draft, drafted, u, t1)
    with torch.cuda.graph(g2):
        fb.fopd_draw_tokens(rows, ur, r1)
        fb.fopd_verify_draft(target, draft, drafted, u, t2)
    u.copy_(uniforms((B, K + 1), 137))
    want2, _ = run_verify(target, draft, drafted, u)
    with torch.cuda.stream(streams[0]):
        g1.replay()
    with torch.cuda.stream(streams[1]):
        g2.replay()
    torch.cuda.synchronize()
    for t in (t1, t2):
        assert np.array_equal(t.cpu().numpy(), want2["tokens"])
    assert torch.equal(r1, want_rows)


# ---- every way a call is cut up: one launch or two, clusters of one to eight CTAs, slots of several parts ----

@pytest.mark.parametrize("n,V,dtype", [(8, 9001, BF16), (60, 4001, F32), (140, 9001, F32), (200, 9001, BF16), (700, 3001, BF16)])
def test_draw_many_rows_that_fp32_does_not_decide(n, V, dtype):
    """Flat rows: with all probabilities near 1/V a number close to a boundary is the rule; numbers 1e-9 beside one."""
    x = rows_of((n,), V, dtype, n, scale=0.01)
    u = uniforms(n, n + 1)
    for r in range(0, n, 3):
        c = np.cumsum(ro.probabilities(x[r].cpu(), 1.0))
        u[r] = float(c[(r * 37) % (V - 1)]) + (1e-9 if r % 2 else -1e-9)
    tokens = check_draw(x, u, 1.0)
    assert len(set(tokens.tolist())) > n // 3


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_draw_and_verify_rows_of_millions(dtype):
    V = 5_000_003
    x = rows_of((2,), V, dtype, 301, scale=1.0)
    x[1, 4_999_990] = 25.0
    for T in (1.0, 0.0):
        check_draw(x, torch.tensor([0.999999, 0.999], device=DEV, dtype=torch.float64), T)
    check_draw(x, uniforms(2, 302), 2.0)
    draft = (x[:1].float() + 0.1).to(dtype)
    wide = torch.zeros((1, 1, x.stride(0)), device=DEV, dtype=dtype)
    wide[0, 0, :V] = draft[0]
    wide[0, 0, 77] = 30.0  # the draft is sure of a token that the target hardly has
    check_verify(x.view(1, 2, V) if x.is_contiguous() else x.unsqueeze(0), wide[:, :, :V],
                 torch.tensor([[77]], dtype=torch.int32, device=DEV), uniforms((1, 2), 303))


def test_draw_many_rows_with_slots_of_several_parts():
    n, V = 640, 540_001
    x = torch.zeros((n, V + 7), device=DEV, dtype=BF16)[:, :V]
    some = [0, 1, 311, 638, 639]
    rows = rows_of((len(some),), V, BF16, 311)
    for k, r in enumerate(some):
        x[r] = rows[k]
    u = uniforms(n, 312)
    tokens, lp, bits = run_draw(x, u, 1.0)
    want = {r: ro.draw(rows[k].cpu(), float(u[r]), 1.0)[0] for k, r in enumerate(some)}
    assert bits == 0 and {r: int(tokens[r]) for r in some} == want
    even = torch.ones(n, dtype=torch.bool, device=DEV)
    even[some] = False
    assert torch.equal(tokens[even].long(), (u[even] * V).floor().long())  # even rows: floor(v V)


@pytest.mark.parametrize("B,K", [(3, 2), (50, 2), (100, 30)])
@pytest.mark.parametrize("form", ["rows", "certain"])
def test_verify_decisions_next_to_equality(B, K, form):
    """u q within 1e-9 of p, on both sides: fp32 leaves these open.  (B, K) such that a position has a cluster, the
    finish is cut in two launches, or clusters stay."""
    V = 1300
    target, draft = rows_of((B, K + 1), V, BF16, 321 + B, scale=1.0), rows_of((B, K), V, BF16, 322, scale=1.0)
    drafted = torch.zeros((B, K), dtype=torch.int32, device=DEV)
    u = uniforms((B, K + 1), 323)
    for b in range(B):
        for j in range(min(K, 3)):
            p = ro.probabilities(target[b, j].cpu(), 1.0)
            q = ro.probabilities(draft[b, j].cpu(), 1.0) if form == "rows" else np.ones(V)
            x = int(np.argmax(q - p)) if form == "rows" else int(np.argmax(p))
            drafted[b, j] = x
            u[b, j] = float(p[x] / q[x]) * (1 + (1e-9 if (b + j) % 3 == 0 else -1e-9))
    got = check_verify(target, draft if form == "rows" else None, drafted, u)
    assert got["n_accepted"].min() == 0 and got["n_accepted"].max() >= 2


@pytest.mark.parametrize("form,T", [("rows", 1.0), ("certain", 0.7), ("best", 1.0), ("rows", 0.0)])
@pytest.mark.parametrize("B,K,V", [(45, 6, 1501), (1, 3000, 70), (300, 9, 333), (33, 100, 129)])
def test_verify_forms_at_every_cut(form, T, B, K, V):
    target = rows_of((B, K + 1), V, F32, 331 + B, scale=2.0)
    draft = rows_of((B, K), V, F32, 332, scale=0.3)
    draft += target[:, :K]
    Td = 0.0 if form == "best" else 1.0
    drafted = drafts_from(draft if T else target[:, :K], Td if T else 0.0, 333)
    if form == "certain":
        drafted = target[:, :K].argmax(-1).int()
    u = uniforms((B, K + 1), 334) * 0.9
    n_draft = torch.randint(K // 2, K + 1, (B,), generator=torch.Generator(device=DEV).manual_seed(B), device=DEV,
                            dtype=torch.int32)
    got = check_verify(target, None if form == "certain" else draft, drafted, u, n_draft=n_draft, T=T, Td=Td)
    if T == 0:
        assert got["n_accepted"].tolist() == n_draft.tolist()
    again, _ = run_verify(target, None if form == "certain" else draft, drafted, u, n_draft=n_draft, T=T, Td=Td)
    assert all(np.array_equal(got[k], again[k]) for k in got)  # whatever order the clusters came in


@pytest.mark.parametrize("B,V,offset", [(400, 2600, 0.0), (400, 9, 0.0), (20, 2600, 3.0e6)])
def test_verify_many_sequences_without_a_residual(B, V, offset):
    """A drafted token that neither row can give, and equal rows: p - q is zero everywhere and one fp64 search comes right
    behind another (in the second launch, and in the whole kernel where logits are out of the reach of fp32)."""
    target = rows_of((B, 2), V, F32, 347)
    target += offset
    target[:, 0, V - 1] = -math.inf
    draft = rows_of((B, 1), V, F32, 348)
    draft[:] = target[:, :1]
    drafted, u = torch.full((B, 1), V - 1, dtype=torch.int32, device=DEV), uniforms((B, 2), 349)
    got = check_verify(target, draft, drafted, u)
    assert got["n_accepted"].max() == 0
    for _ in range(30):
        again, bits = run_verify(target, draft, drafted, u)
        assert bits == 0 and all(np.array_equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("T", [1.0, 0.0])
def test_small_clusters_that_start_while_the_gpu_is_full(T):
    """Rows so short that most CTAs of a cluster have nothing to read and exchange their sums as soon as they run, beside
    work on another stream that takes the places where the others are to start."""
    V, B, K, R = 5, 4, 2, 40
    x, u = rows_of((6,), V, F32, 341), uniforms(6, 342)
    target, draft = rows_of((B, K + 1), V, BF16, 343), rows_of((B, K), V, BF16, 344)
    drafted, uv = drafts_from(draft, 1.0, 345), uniforms((B, K + 1), 346)
    want, want_v = check_draw(x, u, T), check_verify(target, draft, drafted, uv, T=T)["tokens"]
    tokens = torch.zeros((R, 6), dtype=torch.int32, device=DEV)
    out = torch.zeros((R, B, K + 1), dtype=torch.int32, device=DEV)
    a = torch.randn(4096, 4096, device=DEV, dtype=BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for r in range(R):
        a @ a
        with torch.cuda.stream(side):
            fb.fopd_draw_tokens(x, u, tokens[r], temperature=T)
            fb.fopd_verify_draft(target, draft, drafted, uv, out[r], temperature=T)
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in tokens)
    assert all(np.array_equal(t, want_v) for t in out.cpu().numpy())


@pytest.mark.parametrize("V,dtype,scale,T", [(32000, BF16, 3.0, 1.0), (32003, F32, 1.0, 0.3), (9001, BF16, 0.05, 0.7), (50001, F32, 5.0, 1.7)])
def test_thousands_of_draws_against_torch_in_64_bits(V, dtype, scale, T):
    n = 6000
    x, u = rows_of((n,), V, dtype, V, scale=scale), uniforms(n, V + 1)
    tokens, lp, bits = run_draw(x, u, T)
    assert bits == 0
    for at in range(0, n, 1000):
        y = x[at:at + 1000].double() / T
        c = torch.softmax(y, -1).cumsum(-1)
        want = torch.searchsorted(c, (u[at:at + 1000] * c[:, -1]).unsqueeze(1), right=True).squeeze(1)
        assert torch.equal(tokens[at:at + 1000].long(), want)
        wl = (y.gather(1, want.unsqueeze(1)).squeeze(1) - y.logsumexp(-1)).cpu().numpy()
        assert np.all(np.abs(lp[at:at + 1000].cpu().numpy() - wl) <= lp_tol(wl))


@pytest.mark.parametrize("n,V,dtype,offset", [(400, 3001, F32, 1.0e5), (400, 3001, F32, -2.0e5), (300, 9001, BF16, 900.0),
                                              (40, 70001, F32, 7.0e4), (60, 3001, F32, 3.0e6)])
def test_many_draws_from_logits_far_from_zero(n, V, dtype, offset):
    """The rounding of max c grows with the logits' offset; sums and elements have to agree on it."""
    x = rows_of((n,), V, dtype, n + V, scale=1.0)
    x.add_(offset)
    check_draw(x, uniforms(n, 351), 1.0)
    target, draft = x.as_strided((n // 4, 2, V), (4 * x.stride(0), x.stride(0), 1)), x[2::4].unsqueeze(1)
    check_verify(target, draft, drafts_from(draft, 1.0, 352), uniforms((n // 4, 2), 353))
    check_verify(target, None, drafts_from(draft, 1.0, 354), uniforms((n // 4, 2), 355))


def test_logits_far_from_zero_and_small_temperatures():
    for dtype, offset in ((BF16, 3000.0), (F32, -3.0e4), (F32, 2.0e8), (F32, -3.0e38)):
        x = rows_of((6,), 2500, dtype, 341)
        x.add_(offset) if offset > -1e38 else x.fill_(offset)
        check_draw(x, uniforms(6, 342), 1.0)
    x = rows_of((20,), 2500, BF16, 343)
    for T in (2.0 ** -10, 0.02, 1024.0):
        check_draw(x, uniforms(20, 344), T)


# ---- together, as a training program uses them ----

@pytest.mark.parametrize("dtype,T", [(F32, 1.0), (BF16, 1.0)])
def test_draw_verify_loss_and_clip_in_one_run(dtype, T):
    """Drafts are drawn from one policy, verified against the one that has moved on, graded by a teacher; the rows
    that came out are a chunk of the loss, whose gradient is clipped by its norm.  Each stage against its fp64
    definition."""
    import _parity as par
    from oracle import fopd_oracle as orc

    B, K, V = 6, 9, 1201
    W = K + 1
    target, teacher, draft = (rows_of(s, V, dtype, k, pad=3) for k, s in ((201, (B, W)), (202, (B, W)), (203, (B, K))))
    draft[:] = target[:, :K] + 0.3 * draft
    teacher += target - 0.7 * teacher
    flat = draft.as_strided((B * K, V), (draft.stride(1), 1))
    drafted = torch.empty(B * K, dtype=torch.int32, device=DEV)
    fb.fopd_draw_tokens(flat, uniforms(B * K, 204), drafted, temperature=T)
    assert drafted.tolist() == [ro.draw(r, float(v), T)[0] for r, v in zip(flat.cpu(), uniforms(B * K, 204).cpu())]
    drafted = drafted.view(B, K)
    u = uniforms((B, W), 205)
    out = pl.verify_rollout(target, draft, drafted, u, pl.Rollout.alloc(B, K, DEV), temperature=T, draft_temperature=T)
    want = check_verify(target, draft, drafted, u, T=T, Td=T)
    assert np.array_equal(out.tokens.cpu().numpy(), want["tokens"])

    sid = torch.arange(B, dtype=torch.int32, device=DEV)
    chunk = pl.rollout_chunk(target, teacher, out, sid)
    n = B * W
    dl_buf = torch.zeros((n, target.stride(1)), dtype=dtype, device=DEV)
    dlogits = dl_buf[:, :V]
    tau = torch.tensor([0, 1, 0, 2, 0, 1], dtype=torch.int32, device=DEV)
    H = torch.full((B,), W, dtype=torch.int32, device=DEV)
    p = fb.params(**par.PARAMS)

    def run(clip):
        buf, rows = pl.BatchBuffers(B, DEV), [pl.RowOutputs.alloc(n, DEV)]
        pl.step([chunk], [dlogits], buf, tau, H, None, p, rows, clip=clip)
        assert fb.fopd_check_status(buf.status) == 0
        return buf, dlogits.clone()

    buf, plain = run(None)
    # the behaviour policy is the current one: ratio 1, no rollout drift, freshness 1 / (tau + 1)
    assert np.allclose(buf.f.cpu().numpy(), 1.0 / (tau.cpu().numpy() + 1), rtol=1e-4)
    assert buf.acc[:, 0].cpu().tolist() == (out.n_accepted + 1).cpu().tolist()
    wide = lambda t: t.as_strided((n, t.stride(1)), (t.stride(1), 1))  # the loss on these rows against its own oracle
    ch = dict(student=wide(target), teacher=wide(teacher), tokens=chunk.tokens, behav_logprob=chunk.behav_logprob,
              mask=chunk.mask, sample_id=chunk.sample_id)
    par.compare([ch], B, tau.cpu().numpy(), H.cpu().numpy(), vocab=V)
    assert torch.equal(plain[chunk.mask == 0], torch.zeros_like(plain[chunk.mask == 0]))
    norm, coef, scaled = ro.clip([plain], 0.01)
    assert coef < 1
    clip = pl.GradientClip([dlogits], 0.01)
    _, clipped = run(clip)
    assert abs(float(clip.norm) - norm) <= 2.0 ** -23 * norm and abs(float(clip.coef) - coef) <= 2.0 ** -23 * coef
    got = clipped.cpu().double().numpy()
    step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert np.all(np.abs(got - scaled[0]) <= np.abs(scaled[0]) * (step * 1.001 + 2.0 ** -22) + 1e-38)
    _, again = run(None)
    assert torch.equal(again, plain)  # without clipping a step is what it was


# ---- numbers on and next to a boundary ----

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,n", [(7, 1), (9000, 1), (9000, 60), (70001, 1), (1531, 700)])
def test_draw_even_rows_by_neighbours_of_a_boundary(V, n, dtype):
    """Even rows have whole sums, so that the token of a number v is floor(v V) to the last bit of v: with V beyond a power
    of two, v V rounds to a boundary from below it, too."""
    from fractions import Fraction

    x = rows_of((n,), V, dtype, 8)
    x.fill_(-1.5)
    k = np.random.RandomState(9).permutation(V - 1)[:200] + 1
    v = np.concatenate([f(k / V) for f in (lambda y: y, lambda y: np.nextafter(y, 0), lambda y: np.nextafter(y, 1))])
    want = [math.floor(Fraction(float(y)) * V) for y in v]
    assert any(y * V == i + 1 for y, i in zip(v, want))  # numbers whose product rounds up to the next boundary
    if n == 1:
        got = [run_draw(x, torch.tensor([y], device=DEV), 1.0)[0].tolist()[0] for y in v]
    else:
        v, want = np.resize(v, -(-len(v) // n) * n), np.resize(want, -(-len(v) // n) * n).tolist()
        got = sum((run_draw(x, torch.tensor(v[i:i + n], device=DEV), 1.0)[0].tolist() for i in range(0, len(v), n)), [])
    assert got == want


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("form", ["rows", "certain"])
@pytest.mark.parametrize("B", [1, 40, 900])
def test_verify_even_rows_by_neighbours_of_equality(B, form, dtype):
    """Even rows of a target with a tokens and of a draft with fewer, b: a draft is accepted while u a < b, to the last
    bit of u (b = 1 where it was certain)."""
    from fractions import Fraction

    V, rng = 6007, np.random.RandomState(10)
    target, draft = rows_of((B, 2), V, dtype, 11), rows_of((B, 1), V, dtype, 12)
    calls = 60 if B == 1 else 1
    wrong = 0
    for call in range(calls):
        a = rng.randint(2, V + 1, B)
        b = np.array([rng.randint(1, x) for x in a]) if form == "rows" else np.ones(B, dtype=int)
        column = torch.arange(V, device=DEV)
        even = lambda n: torch.where(column < torch.tensor(n, device=DEV).unsqueeze(1), 0.25, -math.inf).to(dtype)
        target[:, 0], draft[:, 0] = even(a), even(b)
        u = uniforms((B, 2), 13 + call)
        at = b / a
        first = np.stack([at, np.nextafter(at, 0), np.nextafter(at, 1)])[(np.arange(B) + call) % 3, np.arange(B)]
        u[:, 0] = torch.tensor(first)
        drafted = torch.zeros((B, 1), dtype=torch.int32, device=DEV)
        got, bits = run_verify(target, draft if form == "rows" else None, drafted, u)
        want = [int(Fraction(float(y)) * int(n) < int(m)) for y, n, m in zip(first, a, b)]
        wrong += sum(int(y * (1 / m) < 1 / n) != w for y, n, m, w in zip(first, a, b, want))
        assert bits == 0 and got["n_accepted"].tolist() == want
    assert wrong > 0  # some of which two rounded probabilities would decide otherwise


# ---- weights at the cut: below 2^-900 of their row's largest they are zero ----

GAPS = (890.0, 896.0, 899.0, 901.0, 905.0, 908.0, 912.0, 1000.0, 1100.0)  # bits below the largest


def at_the_cut(x, T):
    """Rows as the definition sees them: what lies below the cut is banned.  None of the tests' logits lies on the cut
    itself (exponents are rounded to sixteenths there)."""
    y = x.double()
    bits = (y.amax(-1, keepdim=True) - y) / T / math.log(2)
    assert not bool(((bits > 899.9) & (bits < 900.1)).any())
    return torch.where(bits > 900.0, torch.full_like(x, -math.inf), x)


def below(gap, T, dtype):
    """A logit `gap` bits below 0, as far as the type has it."""
    return float(torch.tensor(-gap * T * math.log(2), dtype=torch.float64).to(dtype))


@pytest.mark.parametrize("dtype,T", [(BF16, 1.0), (F32, 0.01)])
@pytest.mark.parametrize("V", [9001, 151936])
def test_draws_where_only_tiny_weights_pass(V, dtype, T):
    """A run of columns far below the rest and numbers that pass as soon as there is a weight: each alone among fewer
    elements and more, in calls of one row (eight CTAs), of some (two launches) and of many (a CTA to a row)."""
    heads = (1, 9, 300, V // 8, V - 1)
    x = rows_of((2 * len(GAPS) * len(heads),), V, dtype, 1)
    x.fill_(0.0)
    for i in range(len(x)):
        x[i, :heads[i // 2 % len(heads)]] = below(GAPS[i // 2 // len(heads)], T, dtype)
    u = torch.zeros(len(x), dtype=torch.float64, device=DEV)
    u[1::2] = 0.3
    want = [ro.draw(r, float(v), T) for r, v in zip(at_the_cut(x, T).cpu(), u.cpu())]
    wt, wl = [w[0] for w in want], np.array([w[1] for w in want])
    assert len(set(wt[::2])) > 4  # the first column, and those behind the heads
    tokens, lp, bits = run_draw(x, u, T)
    assert tokens.tolist() == wt and bits == 0
    assert np.all(np.abs(lp.cpu().numpy() - wl) <= lp_tol(wl))
    for i in range(len(x)):
        tokens, lp, bits = run_draw(x[i:i + 1], u[i:i + 1], T)
        assert tokens.tolist() == wt[i:i + 1] and bits == 0 and abs(float(lp) - wl[i]) <= lp_tol(wl[i])
    if V < 100000:
        whole = x.as_strided((len(x), x.stride(0)), (x.stride(0), 1))
        tokens, lp, bits = run_draw(whole.repeat(8, 1)[:, :V], u.repeat(8), T)
        assert tokens.tolist() == wt * 8 and bits == 0


@pytest.mark.parametrize("B", [1, 60, 700])
@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("dtype,T", [(BF16, 0.1), (F32, 1.0)])
def test_residual_of_a_greedy_draft_at_the_cut(dtype, T, bad, B):
    """The target is nearly certain of the draft's best token and the drafted one is banned (or no token): what is left
    has the whole of its weight around the cut, in a few columns or in all."""
    V = 9001
    target, draft = rows_of((B, 2), V, dtype, 2), rows_of((B, 1), V, dtype, 3, scale=0.1)
    drafted = torch.full((B, 1), V + 3 if bad else 5, dtype=torch.int32, device=DEV)
    for b in range(B):
        few = b // len(GAPS) % 3
        target[b, 0] = below(GAPS[b % len(GAPS)], T, dtype) if few == 0 else -math.inf
        if few == 1:
            target[b, 0, 7000:7009] = below(GAPS[b % len(GAPS)], T, dtype)
        if few == 2:
            target[b, 0, 4100] = below(GAPS[b % len(GAPS)], T, dtype)
        target[b, 0, 5] = -math.inf
        target[b, 0, 77], draft[b, 0, 77] = 0.0, 9.0
    u = uniforms((B, 2), 4)
    u[::2, 1] = 0.0
    got, bits = run_verify(target, draft, drafted, u, T=T, Td=0.0)
    cut = at_the_cut(target, T).cpu()
    for b in range(min(B, 3 * len(GAPS) * 2)):
        out, lps, acc, why, was_bad = ro.verify(cut[b], draft[b].cpu(), drafted[b].cpu().numpy(), 1, u[b].cpu().numpy(), T, 0.0)
        assert why == "" and acc == 0 and was_bad == bad
        assert got["tokens"][b].tolist() == [out[0], -1] and got["mask"][b].tolist() == [1, 0] and got["n_accepted"][b] == 0
        assert abs(got["logprob"][b, 0] - lps[0]) <= lp_tol(lps[0])
    assert (got["mask"] == [1, 0]).all() and (got["tokens"][:, 0] >= 0).all() and (got["tokens"][:, 1] == -1).all()
    assert bits == (1 if bad else 0)


@pytest.mark.parametrize("B", [1, 60, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_residual_of_rows_that_differ_at_the_cut(dtype, B):
    """p and q are equal but for one element with a tiny p and no q; the drafted token is banned in both."""
    V = 5003
    target, draft = rows_of((B, 2), V, dtype, 5, scale=0.5), rows_of((B, 1), V, dtype, 6)
    target[:, 0, 3] = -math.inf
    target[:, 0, 9] = 4.0
    draft.copy_(target[:, :1])
    draft[:, 0, 4444] = -math.inf
    for b in range(B):
        target[b, 0, 4444] = float(torch.tensor(4.0 + below(GAPS[b % len(GAPS)], 1.0, F32), dtype=torch.float64).to(dtype))
    u = uniforms((B, 2), 7)
    drafted = torch.full((B, 1), 3, dtype=torch.int32, device=DEV)
    got, bits = run_verify(target, draft, drafted, u)
    assert bits == 0 and (got["mask"] == [1, 0]).all()
    cut, seen = at_the_cut(target, 1.0).cpu(), set()
    for b in range(min(B, 60)):
        out, lps, acc, _, _ = ro.verify(cut[b], draft[b].cpu(), [3], 1, u[b].cpu().numpy(), 1.0, 1.0)
        assert got["tokens"][b].tolist() == [out[0], -1] and abs(got["logprob"][b, 0] - lps[0]) <= lp_tol(lps[0])
        seen.add(out[0] == 4444)
    assert len(seen) == min(B, 2)


@pytest.mark.parametrize("T", [1.0, 0.7, 0.0])
def test_a_fresh_rollout_at_any_temperature_is_fresh(T):
    """Sampled at T, a rollout's own log-probs are those of softmax(x / T); with the policy's at its tokens the ratio is 1
    and there is no drift."""
    B, K, V = 5, 4, 1203
    target, teacher, draft = (rows_of(s, V, F32, k) for k, s in ((401, (B, K + 1)), (402, (B, K + 1)), (403, (B, K))))
    draft.copy_(target[:, :K])
    drafted = drafts_from(draft, T, 404)
    out = pl.verify_rollout(target, draft, drafted, uniforms((B, K + 1), 405), pl.Rollout.alloc(B, K, DEV), temperature=T,
                            draft_temperature=T)
    assert int(out.status[0]) == 0 and out.temperature == T
    sid = torch.arange(B, dtype=torch.int32, device=DEV)
    if T == 1.0:
        chunk = pl.rollout_chunk(target, teacher, out, sid)
    else:
        with pytest.raises(AssertionError):
            pl.rollout_chunk(target, teacher, out, sid)
        lp = torch.zeros((B, K + 1), device=DEV)
        first = pl.rollout_chunk(target, None, out, sid, behav_logprob=lp)
        own = torch.zeros_like(lp)
        fb.fopd_token_stats_student(first, B, torch.zeros((B, 4), dtype=torch.float64, device=DEV), lp_s=own)
        chunk = pl.rollout_chunk(target, teacher, out, sid, behav_logprob=own)
    at = out.tokens.clamp(min=0).long().unsqueeze(2)
    want = target.double().log_softmax(-1).gather(2, at).squeeze(2)
    kept = out.mask.bool()
    assert torch.allclose(chunk.behav_logprob.view(B, K + 1)[kept].double(), want[kept], rtol=1e-5, atol=1e-5)
    buf, rows = pl.BatchBuffers(B, DEV), [pl.RowOutputs.alloc(B * (K + 1), DEV)]
    pl.measure([chunk], buf, rows)
    tau, H = torch.zeros(B, dtype=torch.int32, device=DEV), torch.full((B,), K + 1, dtype=torch.int32, device=DEV)
    pl.freshness(buf, tau, H, None, fb.params())
    assert fb.fopd_check_status(buf.status) == 0
    assert torch.allclose(buf.f, torch.ones_like(buf.f), rtol=1e-4)


def test_a_temporary_that_does_not_fit_is_this_calls_error_alone():
    """4.2 G positions take 168 GB beside 67 GB of arguments: the call says so before it launches anything, and the next ones
    (here and in torch) run."""
    B, K, V = 4000, (1 << 20) - 1, 8
    try:
        target = torch.zeros((K + 1, V), device=DEV, dtype=BF16).expand(B, K + 1, V)
        drafted, tokens = (torch.empty((B, K + w), device=DEV, dtype=torch.int32) for w in (0, 1))
        u = torch.empty((B, K + 1), device=DEV, dtype=torch.float64)
        with pytest.raises(fb.FopdError) as e:
            fb.fopd_verify_draft(target, None, drafted, u, tokens)
        assert e.value.code == -6
    finally:
        target = drafted = tokens = u = None
        torch.cuda.empty_cache()
    ws, x, norm = fb.grad_workspace(DEV), torch.full((9,), 2.0, device=DEV), torch.zeros(1, device=DEV)
    fb.fopd_grad_norm(fb.GradientList([x]), ws, norm=norm)
    assert float(norm) == 6.0 and float((x + x).sum()) == 36.0


# ---- the bound on the fp32 sums: decisions just outside it, and the log-probs it covers ----

def sum_error(V, T):
    """Relative error of an fp32 sum of exponentials and of one of them: an exponent y = x c - max c is off by the rounding
    of c = fl(log2(e) / T) and by 2^-24 |y|, with the mean of |y| at most 0.74 log2 V + 0.5 for V <= 2^18; an ex2 (2^-22) and
    six roundings (2^-24) come on top."""
    c = math.log2(math.e) / T
    return 0.6932 * (5.97e-8 + abs(float(np.float32(c)) - c) / c) * (0.74 * math.log2(V) + 0.5) + 6.2e-7


def lp_bound(V, T, lp):
    """The sum's error; its rounding to fp32; logf, within one unit of the last place of log Z <= log V; the result's rounding."""
    return sum_error(V, T) + 2.0 ** -24 + 2.0 ** -23 * max(1.0, math.log(V)) + 2.0 ** -24 * np.abs(lp)


def coarse_temperatures():
    """Temperatures whose log2(e) / T is rounded furthest, up and down, and one."""
    T = np.linspace(0.3, 1.9, 4001)
    c = math.log2(math.e) / T
    off = (c.astype(np.float32).astype(np.float64) - c) / c
    return [float(T[off.argmax()]), float(T[off.argmin()]), 1.0]


def steep(V, T, seed):
    """Logits (fp32) of the largest mean exponent: one at the top, the rest even at the distance that maximises it, in a random
    place; and the like with a spread, so that boundaries differ."""
    w = 2.0 ** -np.linspace(0.1, math.log2(V) * 1.5, 400)
    s = 1 / (1 + (V - 1) * w)
    y = -float(np.log2(w)[((1 - s) * -np.log2(w)).argmax()])
    rows = torch.full((4, V), -y * T * math.log(2), dtype=torch.float64)
    g = torch.Generator().manual_seed(seed)
    rows[2:] += torch.randn((2, V), generator=g, dtype=torch.float64) * 0.5 * T
    rows[torch.arange(4), torch.randint(0, V, (4,), generator=g)] = 0.0
    rows[1::2] += 11.3
    return rows.float()


@pytest.mark.parametrize("V", [1001, 32003, 151936])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_draws_just_outside_the_bound(V, which):
    """Numbers half to ten bounds from a boundary of the fp64 distribution, on either side: in fp32 where the bound lets a draw
    be decided there, and a bound that were too small would give the neighbour."""
    T = coarse_temperatures()[which]
    eps, base = sum_error(V, T), torch.cat([steep(V, T, 21), torch.randn((4, V), generator=torch.Generator().manual_seed(22)) * 3])
    per, per_vec = 40, 4
    x = torch.zeros((8 * per, -(-V // per_vec) * per_vec), device=DEV)[:, :V]
    x.copy_(base.to(DEV).repeat_interleave(per, 0))
    p = (x[::per].double() / T).softmax(-1)
    F = p.cumsum(-1)
    F = F / F[:, -1:]
    rng = np.random.RandomState(23 + which)
    for dist in (0.5, 1.5, 2.05, 2.5, 3.0, 4.0, 10.0):
        # half of the boundaries beside a large probability, where the neighbours are far away
        top = p.topk(20, -1).indices.cpu().numpy()
        k = np.stack([np.where(rng.rand(per) < 0.5, top[r, rng.randint(0, 20, per)] - rng.randint(0, 2, per),
                               rng.randint(0, V - 1, per)) for r in range(8)]).clip(0, V - 2)
        v = F.gather(1, torch.tensor(k, device=DEV)) + torch.tensor(rng.choice([-1, 1], k.shape), device=DEV) * dist * eps
        v = v.clamp(0, 1 - 1e-9)
        want = torch.searchsorted(F, v, right=True).clamp(max=V - 1)
        tokens, lp, bits = run_draw(x, v.view(-1).contiguous(), T)
        assert bits == 0 and torch.equal(tokens.long(), want.view(-1))
        wl = p.gather(1, want).log().view(-1).cpu().numpy()
        assert np.all(np.abs(lp.cpu().numpy() - wl) <= lp_bound(V, T, wl))


@pytest.mark.parametrize("V", [1001, 32003])
@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("form", ["rows", "certain"])
def test_acceptance_just_outside_the_bound(V, which, form):
    """u q a distance of half to twenty bounds from p, on either side, between rows of the largest mean exponent and even ones;
    the log-probs of what is accepted within the bound."""
    T, n = coarse_temperatures()[which], 96
    Td = coarse_temperatures()[(which + 1) % 3]
    eps = max(sum_error(V, T), sum_error(V, Td))
    target, draft = (torch.zeros((n, w, -(-V // 4) * 4), device=DEV)[:, :, :V] for w in (2, 1))
    a, b = steep(V, T, 31).to(DEV), steep(V, Td, 32).to(DEV)
    target[:, 0], target[:, 1], draft[:, 0] = a.repeat(n // 4, 1), a[0], b.repeat_interleave(n // 4, 0)
    draft[::3, 0] = 0.0
    p, q = (target[:, 0].double() / T).log_softmax(-1), (draft[:, 0].double() / Td).log_softmax(-1)
    if form == "certain":
        q = torch.zeros_like(q)
    rng = np.random.RandomState(33 + which)
    for dist in (0.5, 2.0, 3.9, 4.1, 5.0, 8.0, 20.0):
        x = torch.where(p < q, torch.rand(p.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(int(dist * 10))), -1.0)
        x = torch.where(torch.tensor(rng.rand(n) < 0.5, device=DEV), x.argmax(-1), torch.where(p < q, p, -math.inf).argmax(-1))
        x = x.unsqueeze(1)
        sign = torch.tensor(rng.choice([-1, 1], (n, 1)), device=DEV)
        u = uniforms((n, 2), 34)
        u[:, :1] = ((p - q).gather(1, x).exp() * (1 + sign * dist * eps)).clamp(0, 1 - 1e-9)
        want = (u[:, :1].log() + q.gather(1, x) < p.gather(1, x)).view(-1).cpu().numpy()
        assert want.any() and not want.all()
        got, bits = run_verify(target, draft if form == "rows" else None, x.int(), u, T=T, Td=Td)
        assert bits == 0 and np.array_equal(got["n_accepted"], want.astype(np.int32))
        wl = p.gather(1, x).view(-1).cpu().numpy()
        assert np.all(np.abs(got["logprob"][want, 0] - wl[want]) <= lp_bound(V, T, wl[want]))


@pytest.mark.parametrize("V,dtype,T", [(151936, BF16, 1.0), (32003, F32, 0.37), (9, F32, 1.0), (70001, BF16, 1.7)])
def test_log_probs_within_the_bound(V, dtype, T):
    x, u = rows_of((200,), V, dtype, 41), uniforms(200, 42)
    for n in (200, 1):
        tokens, lp, bits = run_draw(x[:n], u[:n], T)
        wl = (x[:n].double() / T).log_softmax(-1).gather(1, tokens.long().unsqueeze(1)).view(-1).cpu().numpy()
        assert bits == 0 and np.all(np.abs(lp.cpu().numpy() - wl) <= lp_bound(V, T, wl))


# ---- log-probs of tokens that are nearly certain ----

def near_certain(n, V, T, dtype, seed, offset):
    """Rows whose largest element, in a random place, leaves the others about 1e-9 to 0.2 of its weight together."""
    x = rows_of((n,), V, dtype, seed, scale=0.5 * T)
    rest = torch.tensor([1e-9, 1e-6, 1e-4, 1e-2, 0.05, 0.2], dtype=torch.float64)[torch.arange(n) % 6]
    x -= (T * torch.log((V - 1) / rest)).to(DEV).unsqueeze(1).to(dtype)
    x += offset
    at = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(seed + 1)).to(DEV)
    x[torch.arange(n, device=DEV), at] = offset
    assert bool((x.amax(-1) == x[torch.arange(n, device=DEV), at]).all())
    return x, at


def check_near_certain(x, at, lp, T):
    """-log(1 + rest): the rest's weights are off by their exponents (2^-24 and the rounding of log2(e) / T, relative to y), an
    ex2 (2^-22) and eight roundings on the way to an fp32 number, log1pf by two units of its last place; 1 + rest and what is
    taken out of it have been added up in fp64, some ten times.  From a rest of a quarter on the log is that of the sum."""
    n = torch.arange(len(x), device=DEV)
    z = (x.double() - x[n, at].double().unsqueeze(1)) / T
    w = z.exp()
    w[n, at] = 0.0
    rest = w.sum(-1)
    y = (w * torch.where(w > 0, -z / math.log(2), 0.0)).sum(-1) / rest
    c = math.log2(math.e) / T
    rel = 0.6932 * (5.97e-8 + abs(float(np.float32(c)) - c) / c) * y + 2.0 ** -22 + 8 * 2.0 ** -24 + 2 * 2.0 ** -23
    want = -torch.log1p(rest)
    assert float(rest.max()) < 1.0
    off = (lp.to(DEV).double() - want).abs()
    tol = torch.where(rest < 0.25, rel * want.abs() + 1.5e-15, torch.tensor(lp_bound(x.shape[1], T, want.cpu().numpy()), device=DEV))
    assert bool((off <= tol).all()), float((off / want.abs()).max())
    assert bool((lp <= 0).all())


@pytest.mark.parametrize("dtype,T,offset", [(BF16, 1.0, 0.0), (F32, 0.3577, 0.0), (F32, 1.0, 1e3), (BF16, 0.7, -64.0), (F32, 0.002, 3e4)])
@pytest.mark.parametrize("V,n", [(151936, 1), (4099, 6), (32003, 60), (1025, 700), (6, 12)])
def test_log_probs_of_drawn_tokens_that_are_nearly_certain(V, n, dtype, T, offset):
    x, at = near_certain(n, V, T, dtype, 51, offset)
    p = (x.double() / T).softmax(-1)
    middle = p.cumsum(-1).gather(1, at.unsqueeze(1)) - 0.5 * p.gather(1, at.unsqueeze(1))
    for v in (middle.view(-1).clamp(min=0.0), torch.full_like(middle.view(-1), 0.5)):
        tokens, lp, bits = run_draw(x, v.contiguous(), T)
        assert bits == 0 and torch.equal(tokens.long(), at)
        check_near_certain(x, at, lp, T)


@pytest.mark.parametrize("dtype,T,offset", [(BF16, 1.0, 0.0), (F32, 0.3577, 0.0), (F32, 1.0, 1e3)])
@pytest.mark.parametrize("V,B,K,form", [(151936, 1, 5, "certain"), (4099, 40, 2, "rows"), (1025, 300, 5, "certain"), (700, 9, 400, "rows")])
def test_log_probs_of_verified_tokens_that_are_nearly_certain(V, B, K, form, dtype, T, offset):
    x, at = near_certain(B * (K + 1), V, T, dtype, 53, offset)
    target, best = x.as_strided((B, K + 1, V), (x.stride(0) * (K + 1), x.stride(0), 1)), at.view(B, K + 1)
    u = torch.full((B, K + 1), 0.5, dtype=torch.float64, device=DEV)
    got, bits = run_verify(target, target[:, :K] if form == "rows" else None, best[:, :K].int().contiguous(), u, T=T, Td=T)
    assert bits == 0 and np.array_equal(got["tokens"], best.cpu().numpy())
    check_near_certain(x, at, torch.tensor(got["logprob"]).view(-1), T)
