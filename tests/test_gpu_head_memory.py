"""GPU test of the memory that fopd_head_logprob takes for large vocabularies."""
import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("masked", [False, True])
def test_rows_kept_at_a_time_follow_the_vocabulary(masked):
    """4,500 rows over 4 million tokens, a maximum and a sum for each 128 of them: 1.2 GB at once, 512 MiB 2,048 rows at a time.  Logits from
    two dimensions repeat every 4,096 tokens, so that the definition is that of those."""
    n, V, few = 4500, (1 << 22) + 4096, 4096
    g = torch.Generator(device=DEV).manual_seed(5)
    w = torch.randn((few, 8), generator=g, device=DEV).bfloat16()
    h = torch.randn((n, 8), generator=g, device=DEV).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    mask = (torch.rand(n, generator=g, device=DEV) < 0.9).to(torch.uint8) if masked else None
    weight = w.repeat(V // few, 1)
    lp, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    torch.cuda.synchronize()
    fb._check(fb.lib().fopd_release_device_memory(), "fopd_release_device_memory")
    before = torch.cuda.mem_get_info()[0]
    fb.fopd_head_logprob(h, weight, y, lp, lse=lse, mask=mask)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] <= (512 + 64) << 20
    fb._check(fb.lib().fopd_release_device_memory(), "fopd_release_device_memory")
    z = h.double() @ w.double().t()
    want = torch.logsumexp(z, 1) + torch.log(torch.tensor(float(V // few), dtype=torch.float64))
    on = torch.ones(n, dtype=torch.bool, device=DEV) if mask is None else mask.bool()
    got = z.gather(1, (y.long() % few).unsqueeze(1)).squeeze(1) - want
    # products of eight bf16 numbers, 2^-19 for the sum of exponentials and one rounding each
    tol = 2.0 ** -22 * z.abs().amax(1) * 8 + 2.0 ** -19 + 2.0 ** -23 * want.abs()
    assert ((lse.double() - want * on).abs() <= tol).all() and ((lp.double() - got * on).abs() <= tol).all()
