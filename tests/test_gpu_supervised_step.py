"""The run of the operators together: log-probs and gradients through the head chunk by chunk, clipping, orthogonalised update, against
64 bits.  Each stage's own tolerance is that of its own test file; here the chain's result is compared in the Frobenius norm: the
weights' gradient is off by 2^-14 of its size at most (two planes of G: 2^-16, and the error of the exponentials), and what
that does to the orthogonalised update is played through in 64 bits from the gradient that came out."""
import math

import pytest
import torch

from oracle import orth_oracle as oo
from paper_2605_17862_b200 import binding as fb
from paper_2605_17862_b200 import pipeline as pl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(V, D, sizes, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    weight = (torch.randn((V, D), generator=g, device=DEV) * 2 / math.sqrt(D)).bfloat16()
    total = sum(sizes)
    chunks = []
    for k, n in enumerate(sizes):
        hidden = torch.randn((n, D), generator=g, device=DEV).bfloat16()
        tokens = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
        mask = (torch.rand(n, generator=g, device=DEV) < 0.7).to(torch.uint8) if k % 2 else None
        coef = torch.full((n,), 1.0 / total, device=DEV)
        chunks.append(pl.HeadChunk(hidden, tokens, coef, mask, torch.empty_like(hidden)))
    return weight, chunks


def definition(weight, chunks):
    w = weight.double().requires_grad_(True)
    loss, hs = 0.0, []
    for ch in chunks:
        h = ch.hidden.double().requires_grad_(True)
        lp = torch.log_softmax(h @ w.t(), 1).gather(1, ch.tokens.long().unsqueeze(1)).squeeze(1)
        on = torch.ones_like(lp) if ch.mask is None else ch.mask.double()
        loss = loss - (ch.coef.double() * on * lp).sum()
        hs.append(h)
    loss.backward()
    return float(loss.detach()), w.grad, [h.grad for h in hs]


@pytest.mark.parametrize("V,D,sizes", [(700, 128, (300, 50, 129)), (5000, 256, (1000, 700))])
@pytest.mark.parametrize("captured", [False, True])
def test_supervised_step(V, D, sizes, captured):
    weight, chunks = make(V, D, sizes, V)
    other = (torch.randn((300, 200), device=DEV) * 1e-3).bfloat16()  # another layer's gradient
    keep = other.double()
    d_weight, update = torch.empty((V, D), device=DEV), torch.empty((V, D), device=DEV, dtype=torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    clip = pl.GradientClip([d_weight, other], 1e-2)
    orth = pl.Orthogonalise([d_weight, other], [update, other], scales=[math.sqrt(V / D), 1.0])
    run = lambda: pl.supervised_step(chunks, weight, d_weight, clip=clip, update=orth, status=status)
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graph.replay()
    else:
        run()
    torch.cuda.synchronize()
    assert int(status.cpu()[0]) == 0
    loss, dw, dhs = definition(weight, chunks)
    got = -sum(float((ch.coef.double() * ch.logprob.double()).sum()) for ch in chunks)  # (masked rows have log-prob 0)
    assert abs(got - loss) <= 2.0 ** -17 * (1 + abs(loss))
    for ch, want in zip(chunks, dhs):
        assert float((ch.d_hidden.double() - want).norm()) <= 2.0 ** -7 * float(want.norm())
    norm = math.sqrt(float(dw.square().sum()) + float(keep.square().sum()))
    assert abs(float(clip.norm) - norm) <= 2.0 ** -13 * norm
    coef = min(1.0, 1e-2 / norm)
    assert coef < 1
    assert float((d_weight.double() - coef * dw).norm()) <= 2.0 ** -13 * coef * float(dw.norm())
    played, want = oo.rounding_error(d_weight, fb.NEWTON_SCHULZ_COEFFICIENTS, exact_input=False)
    err = float((update.double() / math.sqrt(V / D) - want).norm())
    assert err <= 2 * played + (2.0 ** -8 + 2.0 ** -12) * float(want.norm())
    played, want = oo.rounding_error((keep * coef).bfloat16(), fb.NEWTON_SCHULZ_COEFFICIENTS)
    assert float((other.double() - want).norm()) <= 2 * played + (2.0 ** -8 + 2.0 ** -7) * float(want.norm())


def test_log_probs_are_a_chunk_s_behaviour_log_probs():
    """fopd_head_logprob's output as fopd_chunk.behav_logprob: fresh tokens have a drift of zero against the logits of the same head."""
    V, D, B, T = 2000, 128, 4, 60
    weight, (ch,) = make(V, D, (B * T,), 3)
    fb.fopd_head_logprob(ch.hidden, weight, ch.tokens, ch.logprob)
    logits = (ch.hidden.float() @ weight.float().t()).contiguous()
    sample = torch.arange(B, device=DEV, dtype=torch.int32).repeat_interleave(T)
    chunk = fb.Chunk(logits, logits.clone(), ch.logprob, ch.tokens, torch.ones(B * T, dtype=torch.uint8, device=DEV), sample)
    buf = pl.BatchBuffers(B, DEV)
    ratio = torch.empty(B * T, device=DEV)
    fb.fopd_token_stats(chunk, B, buf.acc, ratio=ratio, status=buf.status)
    assert float((ratio.double() - 1).abs().max()) < 2.0 ** -14 and float(buf.acc[:, 1].abs().max()) < 1e-6
