"""GPU test of the operators on the tensor cores called from several host threads at once, each on a stream of its own."""
import threading

import pytest
import torch

from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def work(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, V, D = 100 + 70 * seed, 1000 + 333 * seed, 136
    h, w = (torch.randn((r, D), generator=g, device=DEV).bfloat16() for r in (n, V))
    y = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    c = torch.rand(n, generator=g, device=DEV)
    mask = (torch.rand(n, generator=g, device=DEV) < 0.7).to(torch.uint8) if seed % 2 else None
    lp, lse, dh, dw = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros_like(h), torch.zeros((V, D), device=DEV)
    Ms = [torch.randn((200 + 60 * k, 90 + 150 * seed), generator=g, device=DEV) for k in range(3 + seed)]
    outs = [torch.zeros_like(M) for M in Ms]
    listed = fb.MatrixList(Ms, outs)

    def run(stream=None):
        fb.fopd_head_logprob(h, w, y, lp, lse=lse, mask=mask, stream=stream)
        fb.fopd_head_grad(h, w, y, lp, lse, c, d_hidden=dh, d_weight=dw, mask=mask, stream=stream)
        fb.fopd_orthogonalise(listed, stream=stream)

    return run, [lp, lse, dh, dw, *outs]


def test_several_host_threads():
    jobs = [work(k) for k in range(4)]
    want = []
    for run, outs in jobs:
        run()
        want.append([o.clone() for o in outs])
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    streams, start, errors = [torch.cuda.Stream() for _ in jobs], threading.Barrier(len(jobs)), []

    def body(k):
        try:
            torch.cuda.set_device(0)
            start.wait()
            for _ in range(20):
                jobs[k][0](streams[k])
        except BaseException as e:  # noqa: BLE001 (reported by the main thread)
            errors.append(e)

    threads = [threading.Thread(target=body, args=(k,)) for k in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for (_, outs), ref in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, ref))
