"""GPU tests of fopd_head_grad where rows lie gigabytes apart, and of rows of d_hidden that do not count."""
import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(n, V, D, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn((n, D), generator=g, device=DEV).bfloat16()
    w = torch.randn((V, D), generator=g, device=DEV).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(n, generator=g, device=DEV) + 0.1
    mask = (torch.rand(n, generator=g, device=DEV) < 0.5).to(torch.uint8)
    lp, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=mask)
    return h, w, y, c, mask, lp, lse


@pytest.mark.parametrize("D", [16, 20])
@pytest.mark.parametrize("pitch", [(1 << 30) + 8, 1 << 32])
def test_masked_rows_gigabytes_apart(pitch, D):
    """Pitches of 2^31 + 16 bytes and of 2^33, the largest that is taken, with a mask and without."""
    n, V = 3, 40
    h, w, y, c, mask, lp, lse = inputs(n, V, 16, 1)
    if D > 16:
        h, w = torch.nn.functional.pad(h, (0, 4)), torch.nn.functional.pad(w, (0, 4))
        h = torch.cat([h, h[:, :4]], 1)[:, :20]  # rows at a pitch of 24
        w = torch.cat([w, w[:, :4]], 1)[:, :20]
    mask[:] = torch.tensor([1, 0, 1], dtype=torch.uint8)
    far = torch.empty_strided((n, D), (pitch, 1), dtype=torch.bfloat16, device=DEV)
    for m in (mask, None):
        fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=m)
        near = torch.full((n, 24), 7.0, dtype=torch.bfloat16, device=DEV)[:, :D]
        far.fill_(7.0)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=near, mask=m)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=far, mask=m)
        assert torch.equal(near, far) and bool((near[1] == 0).all()) == (m is not None)
    del far
    torch.cuda.empty_cache()


def test_weights_gradient_of_no_rows_two_gigabytes_apart():
    V, D = 3, 9
    far = torch.empty_strided((V, D), ((1 << 29) + 4, 1), dtype=torch.float32, device=DEV)
    far.fill_(7.0)
    behind = far.as_strided((V - 1, 8), (far.stride(0), 1), D)
    behind.fill_(5.0)
    h, w = torch.empty((0, 16), dtype=torch.bfloat16, device=DEV)[:, :D], torch.ones((V, 16), dtype=torch.bfloat16, device=DEV)[:, :D]
    none = torch.empty(0, device=DEV)
    fb.fopd_head_grad(h, w, none.int(), none, none, none, d_weight=far)
    assert (far == 0).all() and (behind == 5).all()
    del far, behind
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [1, 2, 255, 256, 257, 4096, 5000, 70001])
@pytest.mark.parametrize("D,pad", [(8, 0), (72, 8), (259, 5)])
@pytest.mark.parametrize("kept", [0.0, 0.03, 0.9, 1.0])
def test_rows_that_do_not_count_are_cleared(n, D, pad, kept):
    """Wherever they lie among the others, and nothing beside them is."""
    g = torch.Generator(device=DEV).manual_seed(n + D)
    wide = -(-(D + pad) // 8) * 8
    h, w = (torch.randn((r, wide), generator=g, device=DEV).bfloat16()[:, :D] for r in (n, 30))
    y = torch.randint(0, 30, (n,), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(n, generator=g, device=DEV) + 0.5
    mask = (torch.rand(n, generator=g, device=DEV) < kept).to(torch.uint8)
    c[n // 2], y[n // 3] = 0.0, 30  # (rows that do not count for other reasons)
    lp, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=mask)
    buf = torch.full((n, wide), float("nan"), dtype=torch.bfloat16, device=DEV)
    fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=buf[:, :D], mask=mask)
    counts = mask.bool() & (y < 30) & (c != 0)
    assert buf[:, D:].isnan().all() and (buf[~counts, :D] == 0).all()
    assert ((buf[:, :D] != 0).any(1) == counts).all() and not buf[:, :D].isnan().any()
