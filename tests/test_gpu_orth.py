"""GPU tests of fopd_orthogonalise against the definition in 64 bits.

Tolerances (Frobenius norm).  The oracle plays the roundings of X, A and P to fp16 planes through in 64 bits: the kernel's are other
numbers of the same size, so twice their effect is allowed.  Sums: a matrix instruction adds 16 products to the fp32 accumulator and
drops at most 4 u of it (u = 2^-24), so a product over K terms is off by d = 4 u ceil(K / 16) passes of its size; that moves singular
values by a relative d in each of the three products, and what a step does to a relative error of a singular value, |s p'(s) / p(s)|, is
1 for small ones and below 2.5 on [0.68, 1.2] where they settle (3.4445, -4.7750, 2.0315): five steps, 3 d (1 + 2.5 + ... ) with signs that
alternate between them, 16 d in all.  A result is rounded once: 2^-8 in bf16, u in fp32, of each element."""
import math

import pytest
import torch

from oracle import orth_oracle as oo
from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
FIVE = fb.NEWTON_SCHULZ_COEFFICIENTS


def matrix(m, n, seed, dtype=F32, scale=1e-3, strong=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((m, n), generator=g, device=DEV)
    if strong:
        k = min(4, m, n)
        x = x + torch.randn((m, k), generator=g, device=DEV) @ torch.randn((k, n), generator=g, device=DEV)
    return (x * scale).to(dtype)


def check(M, out, scale=1.0, coefficients=FIVE, eps=1e-7):
    full = out.dtype == F32
    played, want = oo.rounding_error(M, coefficients, eps, full, exact_input=M.dtype == BF16)
    d = 4 * U * (math.ceil(max(M.shape) / 16) + 4) * (3 if full else 2)
    size = float(want.norm())
    tol = 2 * played + 16 * d * size + (U if full else 2.0 ** -8) * size + 1e-30
    err = float((out.double() / scale - want).norm())
    assert math.isfinite(err) and err <= tol, (tuple(M.shape), err / max(size, 1e-300), tol / max(size, 1e-300))


def run(tensors, outs=None, scales=None, status=None, **kw):
    fb.fopd_orthogonalise(fb.MatrixList(tensors, outs, scales), status=status, **kw)


SHAPES = [(1, 1), (1, 7), (5, 1), (2, 3), (8, 8), (63, 65), (64, 64), (65, 63), (100, 700), (700, 100), (128, 128), (129, 257), (255, 300),
          (256, 256), (300, 1025), (1025, 300), (513, 512), (1, 5000), (5000, 1), (40, 3001), (1100, 1300)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("din,dout", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_one_matrix(shape, din, dout):
    M = matrix(*shape, seed=shape[0] * 7 + shape[1], dtype=din)
    keep = M.clone()
    out = torch.full(shape, 7.0, device=DEV, dtype=dout)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    run([M], [out], status=status)
    assert torch.equal(M, keep) and int(status.cpu()[0]) == 0
    check(M, out)


@pytest.mark.parametrize("din", [BF16, F32])
def test_matrices_of_a_few_numbers(din):
    """Roundings that nothing averages out: held in two planes, so that a bf16 result is off by its own rounding (2^-8 of each element
    at most), what 22 bits amplified 485-fold leave (2^-13) and the sums' error."""
    g = torch.Generator().manual_seed(7)
    for lot in range(8):
        Ms = [matrix(int(torch.randint(1, 5, (1,), generator=g)), int(torch.randint(1, 60, (1,), generator=g)), 1000 * lot + k, din,
                     strong=k % 2 == 0) for k in range(240)]
        Ms = [M.t().contiguous() if k % 3 == 0 else M for k, M in enumerate(Ms)]
        outs = [torch.empty_like(M, dtype=BF16) for M in Ms]
        run(Ms, outs)
        for M, o in zip(Ms, outs):
            want = oo.orthogonalise(M, FIVE)
            assert float((o.double() - want).norm()) <= (2.0 ** -8 + 2.0 ** -11) * float(want.norm())


@pytest.mark.parametrize("din", [BF16, F32])
def test_large_tiles(din):
    """Enough of 256 x 256 tiles for pairs of CTAs: odd sizes, wide, tall and square in one list."""
    shapes = [(1000, 1000), (1500, 700), (700, 1500), (2000, 2001), (257, 3000), (3000, 257), (1, 9), (64, 4000)]
    Ms = [matrix(m, n, m + n, din) for m, n in shapes]
    outs = [torch.empty(M.shape, device=DEV, dtype=BF16 if k % 2 else F32) for k, M in enumerate(Ms)]
    scales = [0.5 + k for k in range(len(Ms))]
    run(Ms, outs, scales)
    for M, o, s in zip(Ms, outs, scales):
        check(M, o, s)


@pytest.mark.parametrize("shape", [(64, 2000), (2000, 70), (128, 8192), (300, 5000), (5000, 300), (130, 64 * 35 + 1), (520, 4100)])
@pytest.mark.parametrize("din,dout", [(BF16, BF16), (F32, F32)])
def test_few_tiles_with_long_products(shape, din, dout):
    """One or a few tiles of X X^T, their contraction long; the same bits each time."""
    M = matrix(*shape, seed=shape[0], dtype=din)
    outs = [torch.empty(shape, device=DEV, dtype=dout) for _ in range(3)]
    for o in outs:
        run([M], [o])
    check(M, outs[0])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    other = matrix(90, 3000, 5, dtype=din)
    more = [torch.empty(x.shape, device=DEV, dtype=dout) for x in (M, other)]
    run([M, other], more)
    check(M, more[0])
    check(other, more[1])


@pytest.mark.parametrize("shape", [(8_400_321, 2), (2, 8_400_321)])
def test_more_tiles_along_a_side_than_sixteen_bits_count(shape):
    M = matrix(*shape, seed=3, dtype=BF16, strong=False)
    out = torch.full(shape, 7.0, device=DEV, dtype=BF16)
    run([M], [out])
    check(M, out)
    want = oo.orthogonalise(M, FIVE)  # (sums over millions of rows lose no more than a bf16 rounding: they are taken out every 16,384)
    assert float((out.double() - want).norm()) <= 2.0 ** -8 * float(want.norm())


def test_results_are_near_orthogonal():
    """What it is for: singular values end up in [0.68, 1.21] (five steps reach 0.68 from 0.0035 up), directions stay."""
    M = matrix(300, 500, 3, F32, strong=False)
    out = torch.empty_like(M)
    run([M], [out])
    s = torch.linalg.svdvals(out.double())
    assert 0.67 < float(s.min()) and float(s.max()) < 1.22
    u, _, v = torch.linalg.svd(M.double(), full_matrices=False)
    d = torch.diagonal(u.mT @ out.double() @ v.mT)
    assert float((d - s.max()).abs().max()) < 0.6 and float((u * d @ v - out.double()).norm() / out.double().norm()) < 1e-4


@pytest.mark.parametrize("count", [9, 64, 65, 250, 251, 600])
def test_many_matrices(count):
    g = torch.Generator().manual_seed(count)
    shapes = [tuple(int(x) for x in torch.randint(1, 140, (2,), generator=g)) for _ in range(count)]
    Ms = [matrix(m, n, i, BF16 if i % 2 else F32) for i, (m, n) in enumerate(shapes)]
    want = [M.clone() for M in Ms]
    run(Ms)  # in place
    for k in sorted({0, 1, 2, count // 2, count - 2, count - 1, 249 % count, 250 % count, 499 % count}):
        check(want[k], Ms[k])
    alone = want[-1].clone()
    run([alone])
    assert torch.equal(alone, Ms[-1])  # (small tiles both times)


def test_groups_of_one_workspace():
    """More than a GiB of workspace: several groups, the same results as each matrix by itself."""
    Ms = [matrix(4000, 4100 + 64 * k, k, BF16) for k in range(7)]
    outs = [torch.empty_like(M) for M in Ms]
    run(Ms, outs)
    for k in (0, 3, 6):
        alone = torch.empty_like(Ms[k])
        run([Ms[k]], [alone])
        assert torch.equal(alone, outs[k])
    check(Ms[5], outs[5])


def test_pitches_alignment_transposed_and_stacks():
    wide = matrix(130, 400, 1, BF16)
    keep = wide.clone()
    a, b = wide[:, 3:260], wide[:, 261:399]
    run([a, b])
    check(keep[:, 3:260], a)
    check(keep[:, 261:399], b)
    for c in (slice(0, 3), slice(260, 261), slice(399, 400)):
        assert torch.equal(wide[:, c], keep[:, c])
    buf = matrix(1, 70 * 90 + 9, 2, F32).flatten()
    for off in (0, 1, 3):
        M = buf[off:off + 70 * 90].view(70, 90)
        out = torch.full((70 * 90 + 8,), 5.0, device=DEV)
        run([M], [out[off + 1:off + 1 + 70 * 90].view(70, 90)])
        check(M, out[off + 1:off + 1 + 70 * 90].view(70, 90))
        assert (out[:off + 1] == 5).all() and (out[off + 1 + 70 * 90:] == 5).all()
    t = matrix(300, 200, 3, F32).t()
    out = torch.empty((300, 200), device=DEV).t()
    run([t], [out])
    check(t, out)
    stack = torch.stack([matrix(70, 130, 10 + k, BF16) for k in range(6)]).view(2, 3, 70, 130)
    outs = torch.empty_like(stack)
    run([stack, stack[0, :, :, :64]], [outs, torch.empty((3, 70, 64), device=DEV, dtype=F32)])
    for i in range(2):
        for j in range(3):
            check(stack[i, j], outs[i, j])
    col = matrix(50, 8, 4, F32)[:, 2:3]
    out = torch.zeros((50, 3), device=DEV)
    run([col], [out[:, 1:2]])
    check(col, out[:, 1:2])
    assert (out[:, 0] == 0).all() and (out[:, 2] == 0).all()


@pytest.mark.parametrize("scale", [1e-36, 1e-20, 1.0, 1e20, 1e36])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_magnitudes(scale, dtype):
    """Squares of the elements leave fp32's range both ways."""
    M = matrix(70, 200, 5, dtype, scale)
    out = torch.empty_like(M)
    run([M], [out], eps=0.0)
    check(M, out, eps=0.0)


def test_subnormal_elements():
    M = (torch.randint(-9, 10, (40, 60), device=DEV).double() * 2.0 ** -149).float()
    out = torch.empty_like(M)
    run([M], [out], eps=0.0)
    check(M, out, eps=0.0)


@pytest.mark.parametrize("ratio", [1.0, 1e-3])
def test_eps(ratio):
    """A norm of the size of eps: X starts below one."""
    M = matrix(60, 90, 6, F32)
    eps = float(M.double().norm()) / ratio
    out = torch.empty_like(M)
    run([M], [out], eps=eps)
    check(M, out, eps=float(torch.tensor(eps, dtype=F32)))


def test_zeros_infinities_and_empty_lists():
    good = matrix(70, 90, 7, BF16)
    zero = torch.zeros((65, 300), device=DEV)
    bad = [matrix(100, 80, 8, d) for d in (BF16, F32)]
    bad[0][3, 5] = float("nan")
    bad[1][99, 79] = float("-inf")
    outs = [torch.full(x.shape, 7.0, device=DEV, dtype=x.dtype) for x in (zero, good, *bad)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    run([zero, good], outs[:2], status=status, eps=0.0)
    assert (outs[0] == 0).all() and int(status.cpu()[0]) == 0
    alone = outs[1].clone()
    run([zero, good, *bad], outs, status=status, eps=0.0)
    assert int(status.cpu()[0]) == 128
    assert (outs[0] == 0).all() and torch.equal(outs[1], alone)
    assert outs[2].isnan().all() and outs[3].isnan().all()
    run([])
    run([torch.empty((0, 5), device=DEV), torch.empty((5, 0), device=DEV), good.clone()])


COEFFS = {"one step": [(1.5, -0.5, 0.0)], "cubic": [(1.5, -0.5, 0.0)] * 16, "linear": [(2.0, 0.0, 0.0)] * 3, "zero": [(0.0, 0.0, 0.0)],
          "changing": [(4.0, -6.0, 3.0), (3.0, -3.5, 1.25), (2.5, -2.5, 0.9), (1.875, -1.25, 0.375)], "negative": [(-1.0, 0.5, 0.1)] * 2,
          "quintic": [(1.875, -1.25, 0.375)] * 6}


@pytest.mark.parametrize("name", COEFFS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_other_coefficients(name, dtype):
    cs = COEFFS[name]
    M = matrix(150, 220, 9, dtype, strong=False)
    out = torch.full_like(M, 7.0)
    run([M], [out], coefficients=cs)
    c32 = [tuple(float(x) for x in torch.tensor(c, dtype=F32)) for c in cs]
    check(M, out, coefficients=c32)


def test_coefficients_that_may_diverge_are_refused():
    """(4, -6, 3) takes 0.6 to 1.34, the next step that to 3.7, the third to 1,265, the fourth beyond 10^6."""
    M = matrix(150, 220, 9, F32, strong=False)
    with pytest.raises(fb.FopdError) as e:
        run([M], coefficients=[(4.0, -6.0, 3.0), (3.9, -5.8, 2.9), (3.0, -4.0, 2.0), (1.875, -1.25, 0.375)])
    assert e.value.code == -5


def test_streams_graphs_and_repeats():
    shapes = [(300, 500), (900, 200), (64, 64), (1000, 1000)]
    Ms = [matrix(m, n, m, BF16 if m % 3 else F32) for m, n in shapes]
    outs = [torch.empty_like(M) for M in Ms]
    handle = fb.MatrixList(Ms, outs, [1.0, 2.0, 3.0, 4.0])
    fb.fopd_orthogonalise(handle)
    want = [o.clone() for o in outs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    fb.fopd_orthogonalise(handle, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fb.fopd_orthogonalise(handle)
        graphs.append(g)
    for g in graphs + graphs[::-1]:
        for o in outs:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    for M in Ms:  # other matrices in the same places
        M.mul_(torch.rand_like(M))
    graphs[1].replay()
    got = [o.clone() for o in outs]
    fb.fopd_orthogonalise(handle)
    assert all(torch.equal(a, b) for a, b in zip(outs, got))


def test_two_streams_at_once():
    sets = [[matrix(400 + 100 * k, 300, 20 + k, BF16), matrix(100, 900, 30 + k, F32)] for k in range(2)]
    outs = [[torch.empty_like(M) for M in s] for s in sets]
    handles = [fb.MatrixList(s, o) for s, o in zip(sets, outs)]
    for h in handles:
        fb.fopd_orthogonalise(h)
    want = [[o.clone() for o in s] for s in outs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for h, st in zip(handles, streams):
            fb.fopd_orthogonalise(h, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
