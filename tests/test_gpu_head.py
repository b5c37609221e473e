"""GPU tests of fopd_head_logprob and fopd_head_grad against their definitions in 64 bits.

Tolerances.  u = 2^-24.  A product of bf16 values is exact in fp32; a matrix instruction adds 16 of them to the accumulator, and
what it drops is at most 2 u (a truncation) of each of its few partial sums, whose size is at most S_nv = sum_d |h_nd w_vd|: with
D dimensions |dz_nv| <= 4 u ceil(D / 16) S_nv.  The sum of exponentials has positive terms only: its relative error is below
2^-19 (ex2.approx 2^-22, products of the rescaled maxima, sums of 32 at a time), and lse and the log-prob carry one rounding each:
    |d lse|, |d logprob| <= 2 max_v |dz| + 2^-19 + 2 u |value|.
G is rounded to bf16 (2^-8 of each entry; to 2^-16 where two planes are kept), its own error is coef p (|dz| + |d lse| + 2^-19);
the products behind it add 4 u ceil(K / 16) of sum |G| |w| (or |h|), and a bf16 result is rounded once more (2^-8)."""
import math

import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def inputs(n, V, D, seed, pad=0, scale=3.0, masked=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows = lambda r, s: (torch.randn((r, -(-(D + pad) // 8) * 8), generator=g, device=DEV) * s).bfloat16()[:, :D]
    hidden, weight = rows(n, 1.0), rows(V, scale / math.sqrt(D))
    tokens = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    mask = (torch.rand(n, generator=g, device=DEV) >= masked).to(torch.uint8) if masked else None
    coef = (torch.rand(n, generator=g, device=DEV) - 0.25) / n
    return hidden, weight, tokens, mask, coef


def definition(hidden, weight, tokens, mask):
    """(z, lse, logprob, bound on the error of z) in 64 bits; rows that do not count as zeros."""
    h, w = hidden.double(), weight.double()
    on = torch.ones(len(h), dtype=torch.bool, device=DEV) if mask is None else mask.bool()
    on = on & (tokens >= 0) & (tokens < len(w))
    h = torch.where(on.unsqueeze(1), h, 0.0)
    z = h @ w.t()
    dz = 4 * U * math.ceil(h.shape[1] / 16) * (h.abs() @ w.abs().t())
    lse = torch.logsumexp(z, 1)
    lp = z.gather(1, tokens.long().clamp(0, len(w) - 1).unsqueeze(1)).squeeze(1) - lse
    return on, z, lse * on, lp * on, dz


def logprob(hidden, weight, tokens, mask=None, **kw):
    n = hidden.shape[0]
    lp, lse = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    fb.fopd_head_logprob(hidden, weight, tokens, lp, lse=lse, mask=mask, status=status, **kw)
    return lp, lse, int(status.cpu()[0])


def check_logprob(hidden, weight, tokens, mask=None, want_status=0):
    lp, lse, status = logprob(hidden, weight, tokens, mask)
    assert status == want_status
    on, z, lse64, lp64, dz = definition(hidden, weight, tokens, mask)
    tol = 2 * dz.amax(1) + 2.0 ** -19
    assert ((lse.double() - lse64).abs() <= (tol + 2 * U * lse64.abs()) * on).all()
    assert ((lp.double() - lp64).abs() <= (tol + 2 * U * lp64.abs()) * on).all()
    assert (lp <= 0).all()
    return lp, lse


def check_grad(hidden, weight, tokens, mask, coef, f32=False, add=False, parts=("hidden", "weight"), pad=0):
    n, D = hidden.shape
    V = weight.shape[0]
    lp, lse, _ = logprob(hidden, weight, tokens, mask)
    dt = torch.float32 if f32 else torch.bfloat16
    wide = -(-(D + pad) // 8) * 8
    dh_buf = torch.full((n, wide), 3.0, device=DEV, dtype=torch.bfloat16)
    dw_buf = torch.full((V, wide), 0.5 if add else 3.0, device=DEV, dtype=dt)
    dh, dw = dh_buf[:, :D], dw_buf[:, :D]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    fb.fopd_head_grad(hidden, weight, tokens, lp, lse, coef, d_hidden=dh if "hidden" in parts else None,
                      d_weight=dw if "weight" in parts else None, add_d_weight=add, mask=mask, status=status)
    on, z, lse64, lp64, dz = definition(hidden, weight, tokens, mask)
    h, w, c = torch.where(on.unsqueeze(1), hidden.double(), 0.0), weight.double(), coef.double() * on
    p = torch.exp(z - lse64.unsqueeze(1))
    G = p.clone()
    G[torch.arange(n, device=DEV), tokens.long().clamp(0, V - 1)] -= 1
    G *= c.unsqueeze(1)
    step = 2.0 ** -16 if f32 else 2.0 ** -8
    dG = c.abs().unsqueeze(1) * p * (dz + (2 * dz.amax(1, keepdim=True) + 2.0 ** -18 + 2 * U * lse64.abs().unsqueeze(1)))
    if "hidden" in parts:
        want, size = G @ w, G.abs() @ w.abs()
        tol = (dG + G.abs() * 2.0 ** -8) @ w.abs() * 1.01 + 4 * U * (math.ceil(V / 16) + 64) * size + 2.0 ** -8 * want.abs() + 1e-38
        err = (dh.double() - want).abs()
        assert (err <= tol).all(), float((err / tol).max())
        # (the roundings are independent: their sum is about as large as the root of the sum of their squares, which is above
        # the result's own size where its terms cancel, as a column that all weights share makes them: sum_v G_nv = 0)
        spread = (G.square() @ w.square()).sqrt().norm()
        assert float((dh.double() - want).norm()) <= 2.0 ** -8 * float(want.norm() + spread) + 1e-30
        assert (dh[~on] == 0).all()
        assert (dh_buf[:, D:] == 3).all()
    else:
        assert (dh_buf == 3).all()
    if "weight" in parts:
        want, size = G.t() @ h, G.abs().t() @ h.abs()
        tol = (dG + G.abs() * step).t() @ h.abs() * 1.01 + 4 * U * 2 * (math.ceil(n / 16) + 4) * size
        want = want + (0.5 if add else 0.0)
        tol += (2 * U if f32 else 2.0 ** -8) * (want.abs() + tol) + 1e-38
        err = (dw.double() - want).abs()
        assert (err <= tol).all(), float((err / tol).max())
        assert (dw_buf[:, D:] == (0.5 if add else 3.0)).all()
    else:
        assert (dw_buf == (0.5 if add else 3.0)).all()
    return dh, dw, int(status.cpu()[0])


SIZES = [(1, 1, 1, 0), (1, 2, 8, 0), (2, 33, 5, 3), (3, 255, 64, 0), (127, 256, 65, 7), (128, 257, 128, 0), (129, 300, 63, 0),
         (200, 1000, 100, 4), (256, 511, 256, 0), (257, 513, 1001, 7), (300, 4099, 320, 0), (513, 70001, 72, 0), (1000, 2500, 520, 8),
         (4500, 700, 96, 0)]


@pytest.mark.parametrize("n,V,D,pad", SIZES)
def test_logprob_sizes(n, V, D, pad):
    h, w, y, _, _ = inputs(n, V, D, n + V, pad)
    check_logprob(h, w, y)


@pytest.mark.parametrize("n,V,D,pad", SIZES)
@pytest.mark.parametrize("f32", [False, True])
def test_grad_sizes(n, V, D, pad, f32):
    h, w, y, _, c = inputs(n, V, D, n + V + 1, pad)
    assert check_grad(h, w, y, None, c, f32=f32, pad=pad)[2] == 0


@pytest.mark.parametrize("n,V,D,masked", [(100, 700, 72, 0.5), (129, 513, 200, 0.9), (700, 2000, 136, 0.3), (5000, 300, 64, 0.6)])
def test_masked_rows_are_not_read(n, V, D, masked):
    """Rows that do not count hold NaN, infinities, and tokens of any value; their neighbours' results do not notice."""
    h, w, y, mask, c = inputs(n, V, D, n, 0, masked=masked)
    off = mask == 0
    h[off] = float("nan")
    h[off & (torch.arange(n, device=DEV) % 3 == 0)] = float("inf")
    y[off] = torch.where(torch.arange(int(off.sum()), device=DEV) % 2 == 0, -5, 1 << 30).int()
    c[off] = float("nan")
    check_logprob(h, w, y, mask)
    clean = torch.where(mask.bool(), c, 0.0)
    for f32 in (False, True):
        lp, lse, _ = logprob(h, w, y, mask)
        a = torch.empty_like(h), torch.empty(w.shape, device=DEV, dtype=torch.float32 if f32 else torch.bfloat16)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=a[0], d_weight=a[1], mask=mask)
        b = check_grad(h, w, y, mask, clean, f32=f32)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_row_counts():
    n, V, D = 300, 700, 72
    h, w, y, _, c = inputs(n, V, D, 1)
    h[:] = float("nan")
    mask = torch.zeros(n, dtype=torch.uint8, device=DEV)
    lp, lse, status = logprob(h, w, y, mask)
    assert (lp == 0).all() and (lse == 0).all() and status == 0
    for dt in (torch.bfloat16, torch.float32):
        dh, dw = torch.full_like(h, 3.0), torch.full(w.shape, 3.0, device=DEV, dtype=dt)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, mask=mask)
        assert (dh == 0).all() and (dw == 0).all()
        dw.fill_(3.0)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, mask=mask, add_d_weight=True)
        assert (dw == 3).all()
    # no rows at all
    e = h[:0]
    z = torch.empty(0, device=DEV)
    t = torch.empty(0, dtype=torch.int32, device=DEV)
    fb.fopd_head_logprob(e, w, t, z)
    dw = torch.full(w.shape, 3.0, device=DEV, dtype=torch.bfloat16)
    fb.fopd_head_grad(e, w, t, z, z, z, d_hidden=torch.empty_like(e), d_weight=dw, add_d_weight=True)
    assert (dw == 3).all()
    fb.fopd_head_grad(e, w, t, z, z, z, d_weight=dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("n", [100, 400])
@pytest.mark.parametrize("with_mask", [False, True])
def test_tokens_out_of_range(n, with_mask):
    h, w, y, _, c = inputs(n, 515, 80, 3)
    y[3], y[50], y[n - 1] = -1, 515, 1 << 30
    mask = torch.ones(n, dtype=torch.uint8, device=DEV) if with_mask else None
    lp, lse = check_logprob(h, w, y, mask, want_status=1)
    assert float(lp[3]) == float(lse[50]) == float(lp[n - 1]) == 0
    assert check_grad(h, w, y, mask, c)[2] == 1


@pytest.mark.parametrize("n", [90, 300])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("parts", [("hidden",), ("weight",), ("hidden", "weight")])
def test_either_gradient_and_adding(n, add, f32, parts):
    h, w, y, _, c = inputs(n, 1300, 136, 5, 3)
    check_grad(h, w, y, None, c * n, f32=f32, add=add, parts=parts, pad=3)


@pytest.mark.parametrize("n", [64, 260])
def test_rows_of_coefficient_zero(n):
    h, w, y, mask, c = inputs(n, 900, 72, 8, masked=0.3)
    c[::2] = 0
    dh, _, _ = check_grad(h, w, y, None, c)
    assert (dh[::2] == 0).all()
    check_grad(h, w, y, mask, c)


def test_nearly_certain_tokens():
    """log p of -1e-4 to -1e-12 keeps its relative accuracy, and so does the gradient's entry at the token: p - 1.  One hidden
    dimension decides, so that logits are exact: z = 0 for all tokens but one."""
    n, V, D = 12, 300, 64
    w = torch.zeros((V, D), device=DEV, dtype=torch.bfloat16)
    w[17, 0] = 1.0
    h = torch.zeros((n, D), device=DEV, dtype=torch.bfloat16)
    h[:, 0] = torch.arange(8, 8 + 2 * n, 2, device=DEV).bfloat16()
    y = torch.full((n,), 17, dtype=torch.int32, device=DEV)
    lp, lse, _ = logprob(h, w, y)
    rest = (V - 1) * torch.exp(-h[:, 0].double())
    want = -torch.log1p(rest)
    assert ((lp.double() - want).abs() <= want.abs() * (2.0 ** -20 + h[:, 0].double() * 2.0 ** -23)).all()
    # d_weight of token 17 along dimension 0 is sum_n coef (p - 1) h
    c = torch.zeros(n, device=DEV)
    for r in range(n):
        c.zero_()
        c[r] = 1.0
        dw = torch.empty((V, D), device=DEV, dtype=torch.float32)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_weight=dw)
        g = -rest[r] / (1 + rest[r]) * h[r, 0].double()
        assert abs(float(dw[17, 0]) - float(g)) <= abs(float(g)) * (2.0 ** -15 + float(h[r, 0]) * 2.0 ** -22)


@pytest.mark.parametrize("n", [70, 300])
def test_logits_far_from_zero(n):
    """All logits of a row shifted by thousands (a constant column): log-probs are those of the differences as far as fp32 holds the logits."""
    h, w, y, _, c = inputs(n, 800, 72, 12)
    w[:, 0] = 64.0
    h[:, 0] = torch.where(torch.arange(n, device=DEV) % 2 == 0, 40.0, -40.0).bfloat16()
    check_logprob(h, w, y)
    check_grad(h, w, y, None, c)


def test_pieces_and_splits_of_the_vocabulary():
    """Enough rows for several pieces (more than a GiB of logits' gradient), against torch in fp32 on a part."""
    n, V, D = 20000, 40000, 64
    h, w, y, _, c = inputs(n, V, D, 21)
    lp, lse, _ = logprob(h, w, y)
    dh, dw = torch.empty_like(h), torch.empty((V, D), device=DEV, dtype=torch.float32)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw)
    want_w = torch.zeros((V, D), dtype=torch.float64, device=DEV)
    for at in range(0, n, 2000):
        hh = h[at:at + 2000].double()
        G = torch.softmax(hh @ w.double().t(), 1)
        G[torch.arange(len(hh), device=DEV), y[at:at + 2000].long()] -= 1
        G *= c[at:at + 2000].double().unsqueeze(1)
        want = G @ w.double()
        assert float((dh[at:at + 2000].double() - want).norm()) <= 2.0 ** -8 * float(want.norm())
        want_w += G.t() @ hh
    assert float((dw.double() - want_w).norm()) <= 2.0 ** -14 * float(want_w.norm())


@pytest.mark.parametrize("masked", [0.0, 0.1, 0.6, 1.0])
def test_more_rows_than_are_kept_at_a_time(masked):
    """Log-probs of more than 32,768 rows, the count of those that matter above it, below it or zero."""
    h, w, y, mask, _ = inputs(70001, 300, 64, 22, masked=masked)
    check_logprob(h, w, y, mask)


def test_weights_of_more_than_two_to_the_31_elements():
    n, V, D = 3, 1_100_003, 2048
    g = torch.Generator(device=DEV).manual_seed(9)
    w = torch.empty((V, D), device=DEV, dtype=torch.bfloat16)
    for at in range(0, V, 1 << 16):
        w[at:at + (1 << 16)] = torch.randn(w[at:at + (1 << 16)].shape, generator=g, device=DEV) * (2 / math.sqrt(D))
    h = torch.randn((n, D), generator=g, device=DEV).bfloat16()
    y = torch.tensor([0, V - 1, V // 2], dtype=torch.int32, device=DEV)
    c = torch.tensor([1.0, -0.5, 2.0], device=DEV)
    lp, lse, status = logprob(h, w, y)
    z = torch.cat([h.double() @ w[at:at + (1 << 16)].double().t() for at in range(0, V, 1 << 16)], 1)
    lse64 = torch.logsumexp(z, 1)
    lp64 = z.gather(1, y.long().unsqueeze(1)).squeeze(1) - lse64
    assert status == 0 and float((lse.double() - lse64).abs().max()) < 1e-5 and float((lp.double() - lp64).abs().max()) < 1e-5
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw)
    G = torch.softmax(z, 1)
    G[torch.arange(n, device=DEV), y.long()] -= 1
    G *= c.double().unsqueeze(1)
    want = sum(G[:, at:at + (1 << 16)] @ w[at:at + (1 << 16)].double() for at in range(0, V, 1 << 16))
    assert float((dh.double() - want).norm()) <= 2.0 ** -8 * float(want.norm())
    for rows in (slice(0, 300), slice(V // 2 - 100, V // 2 + 100), slice(V - 300, V)):
        want = G[:, rows].t() @ h.double()
        assert float((dw[rows].double() - want).norm()) <= 2.0 ** -7 * float(want.norm())


def test_hidden_states_of_more_than_two_to_the_31_elements():
    n, V, D = 1_100_003, 200, 2048
    g = torch.Generator(device=DEV).manual_seed(10)
    h = torch.empty((n, D), device=DEV, dtype=torch.bfloat16)
    for at in range(0, n, 1 << 16):
        h[at:at + (1 << 16)] = torch.randn(h[at:at + (1 << 16)].shape, generator=g, device=DEV)
    w = (torch.randn((V, D), generator=g, device=DEV) * (2 / math.sqrt(D))).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(n, generator=g, device=DEV) / n
    lp, lse, status = logprob(h, w, y)
    dh, dw = torch.empty_like(h), torch.empty((V, D), device=DEV)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw)
    total = torch.zeros((V, D), dtype=torch.float64, device=DEV)
    for at in range(0, n, 1 << 16):
        rows = slice(at, at + (1 << 16))
        hh, yy = h[rows].double(), y[rows].long().unsqueeze(1)
        lp64 = torch.log_softmax(hh @ w.double().t(), 1)
        assert float((lp[rows].double() - lp64.gather(1, yy).squeeze(1)).abs().max()) < 1e-5
        G = lp64.exp()
        G.scatter_add_(1, yy, torch.full_like(yy, -1.0, dtype=torch.float64))
        G *= c[rows].double().unsqueeze(1)
        want = G @ w.double()
        assert float((dh[rows].double() - want).norm()) <= 2.0 ** -8 * float(want.norm())
        total += G.t() @ hh
    assert status == 0 and float((dw.double() - total).norm()) <= 2.0 ** -13 * float(total.norm())


def test_gradient_against_differences():
    """Central differences of the loss -sum coef logprob computed by the forward call itself along random directions."""
    n, V, D = 40, 500, 64
    h, w, y, _, c = inputs(n, V, D, 30, scale=1.0)
    lp, lse, _ = logprob(h, w, y)
    dh, dw = torch.empty_like(h), torch.empty((V, D), device=DEV, dtype=torch.float32)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw)
    loss = lambda hh, ww: -(c.double() * logprob(hh, ww, y)[0].double()).sum()
    g = torch.Generator(device=DEV).manual_seed(1)
    for grad, which in ((dh, 0), (dw, 1)):
        x = (h, w)[which]
        e = torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.5, -1.0, 1.0)
        up, down = (x.float() * (1 + e * 2.0 ** -6)).bfloat16(), (x.float() * (1 - e * 2.0 ** -6)).bfloat16()
        d = (up.double() - down.double())
        args = lambda v: (v, w) if which == 0 else (h, v)
        diff = float(loss(*args(up)) - loss(*args(down)))
        want = float((grad.double() * d).sum())
        # third-order term: |d|^3 sup |L'''| / 24 with |dz| <= 2^-5 |z|; and the log-probs' error
        z = (h.double() @ w.double().t()).abs().amax(1)
        third = float((c.abs().double() * (z * 2.0 ** -5) ** 3).sum()) / 4
        noise = float(c.abs().double().sum()) * 2 * 2.0 ** -18
        assert abs(diff - want) <= third + noise + 2.0 ** -8 * float((grad.double().abs() * d.abs()).sum())


def test_streams_graphs_and_repeats():
    n, V, D = 300, 2000, 136
    h, w, y, mask, c = inputs(n, V, D, 40, masked=0.4)
    lp, lse, _ = logprob(h, w, y, mask)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    run = lambda st=None: (fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=mask, stream=st),
                           fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, mask=mask, stream=st))
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in (lp, lse, dh, dw)]
    side = torch.cuda.Stream()
    for t in (lp, lse, dh, dw):
        t.zero_()
    torch.cuda.synchronize()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((lp, lse, dh, dw), want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        graphs.append(g)
    for g in graphs + graphs[::-1]:
        for t in (lp, lse, dh, dw):
            t.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((lp, lse, dh, dw), want))
    # replayed on other inputs in the same places, another mask among them
    h2, w2, y2, mask2, c2 = inputs(n, V, D, 41, masked=0.7)
    for a, b in ((h, h2), (w, w2), (y, y2), (mask, mask2), (c, c2)):
        a.copy_(b)
    graphs[0].replay()
    got = [t.clone() for t in (lp, lse, dh, dw)]
    run()
    assert all(torch.equal(a, b) for a, b in zip((lp, lse, dh, dw), got))


def test_two_streams_at_once():
    n, V, D = 200, 3000, 200
    sets = [inputs(n, V, D, 50 + k) for k in range(2)]
    want, outs = [], []
    for h, w, y, _, c in sets:
        lp, lse, _ = logprob(h, w, y)
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw)
        want.append([t.clone() for t in (lp, dh, dw)])
        outs.append((lp, lse, dh, dw))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for (h, w, y, _, c), (lp, lse, dh, dw), st in zip(sets, outs, streams):
            fb.fopd_head_logprob(h, w, y, lp, lse=lse, stream=st)
            fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, stream=st)
    torch.cuda.synchronize()
    for (lp, lse, dh, dw), ref in zip(outs, want):
        assert torch.equal(lp, ref[0]) and torch.equal(dh, ref[1]) and torch.equal(dw, ref[2])
