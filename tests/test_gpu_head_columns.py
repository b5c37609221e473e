"""GPU tests of fopd_head_logprob and fopd_head_grad on column blocks of wider matrices: outputs that lie between an input's rows."""
import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(n, V, D, seed, masked):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h, w = (torch.randn((r, D), generator=g, device=DEV).bfloat16() for r in (n, V))
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(n, generator=g, device=DEV) + 0.1
    return h, w, y, c, (torch.rand(n, generator=g, device=DEV) < 0.6).to(torch.uint8) if masked else None


@pytest.mark.parametrize("n,V,D", [(1, 300, 64), (100, 300, 64), (300, 513, 132), (70, 260, 7)])
@pytest.mark.parametrize("masked", [False, True])
def test_gradients_beside_what_they_are_of(n, V, D, masked):
    h, w, y, c, mask = inputs(n, V, D, n + D, masked)
    up = -(-D // 8) * 8
    wide_h, wide_w = torch.full((n, 3 * up), 9.0, device=DEV).bfloat16(), torch.full((V, 2 * up + 8), 9.0, device=DEV).bfloat16()
    wide_h[:, up:up + D], wide_w[:, :D] = h, w
    h, w, dh, dw = wide_h[:, up:up + D], wide_w[:, :D], wide_h[:, :D], wide_w[:, up:up + D]
    lp, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=mask)
    keep_h, keep_w = wide_h.clone(), wide_w.clone()
    want_h, want_w = (torch.full((r, up), 9.0, device=DEV).bfloat16()[:, :D] for r in (n, V))
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=want_h, d_weight=want_w, mask=mask)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, mask=mask)
    keep_h[:, :D], keep_w[:, up:up + D] = want_h, want_w
    assert torch.equal(wide_h, keep_h) and torch.equal(wide_w, keep_w)
    # d_hidden between the rows of d_weight, d_weight in fp32
    both = torch.full((max(n, V), 2 * up + up), 9.0, device=DEV)
    dw32, dh = both[:V, :D], both.view(torch.bfloat16)[:n, 4 * up:4 * up + D]
    want32 = torch.empty((V, up), device=DEV)[:, :D]
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=want_h, d_weight=want32, mask=mask)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw32, mask=mask)
    assert torch.equal(dw32, want32) and torch.equal(dh, want_h) and (both[:, D:2 * up] == 9).all()


def test_shared_elements_are_refused():
    h, w, y, c, _ = inputs(40, 60, 16, 1, False)
    wide = torch.zeros((60, 40), device=DEV).bfloat16()
    lp, lse = torch.zeros(40, device=DEV), torch.zeros(40, device=DEV)
    hidden, weight = wide[:40, :16], wide[:, 24:40]
    for d_hidden, d_weight in ((wide[:40, 8:24], None), (wide[20:, :16], None), (None, wide[:, 16:32]), (wide[1:41, 16:32], None), (hidden, None),
                               (wide.view(-1)[16:16 + 40 * 16].view(40, 16), None)):
        with pytest.raises(fb.FopdError) as e:
            fb.fopd_head_grad(hidden, weight, y, lp, lse, c, d_hidden=d_hidden, d_weight=d_weight)
        assert e.value.code == -7
