"""GPU tests of fopd_grad_norm, fopd_grad_scale and fopd_grad_clip against the fp64 definitions.

Tolerances.  The sum of squares is formed in fp64 (relative error below 1e-12 for these sizes), norm and coef are
rounded to fp32 once: 2^-24 each.  An output is fl(x fl(coef)), to fp32: 2 * 2^-24 of its size (and half the smallest
subnormal), to bf16: half a bf16 step 2^-8 more of that."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2605_17862_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24 * (1 + 1e-6)


def gradients(shapes, seed, scale=0.01):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(s, generator=g, device=DEV) * scale).to(d) for s, d in shapes]


def scalars():
    return torch.full((1,), 7.0, device=DEV), torch.full((1,), 7.0, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)


def check_values(out, want, dtype):
    out = out.detach().cpu().double().numpy()
    step = 2.0 ** -8 if dtype == BF16 else 0.0
    tiny = (2.0 ** -133 if dtype == BF16 else 2.0 ** -149) * 1.01
    assert np.all(np.abs(out - want) <= np.abs(want) * (2 * U32 + step * (1 + 2 * U32)) + tiny)


def check_clip(tensors, max_norm, outs=None):
    before = [t.detach().cpu().double().numpy().copy() for t in tensors]
    want_norm, want_coef, want = ro.clip(before, float(np.float32(max_norm)))
    norm, coef, status = scalars()
    fb.fopd_grad_clip(fb.GradientList(tensors, outs), max_norm, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
    assert int(status.cpu()[0]) == 0
    assert abs(float(norm) - want_norm) <= U32 * want_norm
    assert abs(float(coef) - want_coef) <= U32 * want_coef
    for k, t in enumerate(tensors):
        check_values(t if outs is None else outs[k], want[k], t.dtype)
        if outs is not None:
            assert np.array_equal(t.detach().cpu().double().numpy(), before[k])
    return float(coef)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 17, 255, 4097, 8191, 8192, 16384, 16385, 1_000_003])
def test_one_tensor_of_any_length(n, dtype):
    x = gradients([((n,), dtype)], n)
    assert check_clip(x, 1e-3) < 1
    assert check_clip(gradients([((n,), dtype)], n + 1), 1e9) == 1


@pytest.mark.parametrize("offset,out_offset", [(0, 0), (1, 1), (3, 3), (1, 0), (0, 5), (7, 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_alignment(dtype, offset, out_offset):
    """Tensors that start at any element, into outputs that start at another one; nothing beside them is written."""
    n = 20011
    buf = gradients([((n + 16,), dtype)], 3)[0]
    out = torch.full((n + 16,), 5.0, device=DEV, dtype=dtype)
    check_clip([buf[offset:offset + n]], 0.1, [out[out_offset:out_offset + n]])
    assert (out[:out_offset] == 5).all() and (out[out_offset + n:] == 5).all()
    copy = buf.clone()
    check_clip([buf[offset:offset + n]], 0.1)
    assert torch.equal(buf[:offset], copy[:offset]) and torch.equal(buf[offset + n:], copy[offset + n:])


def test_mixed_set_pitches_orders_and_empty_tensors():
    wide = gradients([((40, 64), BF16)], 5)[0]
    deep = gradients([((3, 30, 200), F32)], 6)[0]
    keep_w, keep_d = wide.clone(), deep.clone()
    ts = [wide[:, 3:47], wide[:, 48:64], deep[:, :, 10:133], *gradients([((), F32), ((0,), BF16), ((5, 0), F32), ((33, 65), F32)], 7)]
    ts.append(gradients([((70, 90), BF16)], 8)[0].t())
    ts.append(gradients([((4, 5, 6), F32)], 9)[0].permute(2, 0, 1))
    ts.append(gradients([((501,), BF16)], 10)[0][::3])
    assert check_clip(ts, 0.25) < 1
    assert torch.equal(wide[:, :3], keep_w[:, :3]) and torch.equal(wide[:, 47], keep_w[:, 47])
    assert torch.equal(deep[:, :, :10], keep_d[:, :, :10]) and torch.equal(deep[:, :, 133:], keep_d[:, :, 133:])


@pytest.mark.parametrize("count", [16, 17, 48, 112, 113, 257, 999, 1000, 1001, 2500])
def test_many_tensors(count):
    rng = np.random.RandomState(count)
    shapes = [((int(rng.randint(1, 400)),), BF16 if rng.rand() < 0.5 else F32) for _ in range(count)]
    assert check_clip(gradients(shapes, count), 0.5) < 1
    outs = [torch.empty(s, dtype=d, device=DEV) for s, d in shapes]
    check_clip(gradients(shapes, count + 1), 0.5, outs)
    check_clip(gradients(shapes, count + 1), 1e6, outs)  # a plain copy


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pitch", [(5, 1, 3), (70_001, 1, 2), (1000, 7, 8), (333, 1023, 1024), (100, 1024, 1100),
                                             (99, 2047, 2048), (7, 2049, 4000), (3, 20_000, 20_001), (2, 8192, 8200)])
def test_rows_at_a_pitch(rows, cols, pitch, dtype):
    """Short rows share a tile, long ones are cut; what lies between the rows stays."""
    buf = gradients([((rows, pitch), dtype)], rows + cols)[0]
    keep = buf.clone()
    check_clip([buf[:, :cols]], 1e-3)
    assert torch.equal(buf[:, cols:], keep[:, cols:])
    out = torch.full_like(buf, 3.0)
    many = [buf[:, :cols]] * 1 + gradients([((rows, cols), dtype)], 5)
    check_clip(many, 1e-3, [out[:, :cols], torch.empty_like(many[1])])
    assert (out[:, cols:] == 3).all()


def test_many_tensors_with_rows():
    base = [gradients([((37, 40), BF16 if k % 2 else F32)], k)[0] for k in range(700)]
    assert check_clip([b[:, 3:33] for b in base], 0.1) < 1


def test_no_tensors():
    norm, coef, status = scalars()
    fb.fopd_grad_clip(fb.GradientList([]), 1.0, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
    assert float(norm) == 0 and float(coef) == 1 and int(status.cpu()[0]) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e15, 1e30])
def test_squares_beyond_fp32(dtype, scale):
    x = [(torch.randn(5000, device=DEV, dtype=torch.float64) * scale).to(dtype)]
    assert check_clip(x, scale * 10) < 1


def test_unclipped_in_place_leaves_every_bit():
    x = torch.randint(-32768, 32767, (9001,), device=DEV, dtype=torch.int16).view(BF16)
    x = torch.where(x.isfinite() & (x.abs() < 1e18), x, torch.zeros_like(x))
    bits = x.view(torch.int16).clone()
    norm, coef, status = scalars()
    fb.fopd_grad_clip(fb.GradientList([x]), 3e38, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
    assert float(coef) == 1 and torch.equal(x.view(torch.int16), bits)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_is_reported_and_scales_nothing(bad):
    x = gradients([((3000,), F32), ((50, 7), BF16)], 13)
    x[1][3, 3] = bad
    keep = [t.clone() for t in x]
    norm, coef, status = scalars()
    ws = fb.grad_workspace(DEV)
    fb.fopd_grad_clip(fb.GradientList(x), 0.01, ws, norm=norm, coef=coef, status=status)
    assert int(status.cpu()[0]) == 128 and float(coef) == 1 and not math.isfinite(float(norm))
    assert all(torch.equal(a.view(torch.int16 if a.dtype == BF16 else torch.int32),
                           b.view(torch.int16 if b.dtype == BF16 else torch.int32)) for a, b in zip(x, keep))
    outs = [torch.empty_like(t) for t in x]
    fb.fopd_grad_clip(fb.GradientList(x, outs), 0.01, ws, norm=norm, coef=coef)
    assert all(torch.equal(a.nan_to_num(9), b.nan_to_num(9)) for a, b in zip(outs, x))
    # the workspace is good for the next set
    x[1][3, 3] = 0.5
    fb.fopd_grad_clip(fb.GradientList(x), 0.01, ws, norm=norm, coef=coef)
    assert math.isfinite(float(norm)) and float(coef) < 1


def test_norm_in_pieces_then_scale():
    """Chunk by chunk (fopd_grad_norm adds), then every chunk with the whole set's coefficient."""
    chunks = gradients([((100, 1003), BF16), ((57, 1003), BF16), ((1, 1003), F32)], 17)
    want_norm, want_coef, want = ro.clip(chunks, 0.5)
    ws = fb.grad_workspace(DEV)
    norm, coef, status = scalars()
    lists = [fb.GradientList([c]) for c in chunks]
    for l in lists:
        fb.fopd_grad_norm(l, ws, norm=norm, status=status)
    assert abs(float(norm) - want_norm) <= U32 * want_norm
    for l in lists:
        fb.fopd_grad_scale(l, ws, 0.5, norm=norm, coef=coef, status=status)
    assert abs(float(coef) - want_coef) <= U32 * want_coef and int(status.cpu()[0]) == 0
    for c, w in zip(chunks, want):
        check_values(c, w, c.dtype)
    # optional outputs
    fb.fopd_grad_norm(lists[0], ws)
    fb.fopd_grad_scale(lists[0], ws, 0.5)


def test_results_are_the_same_bits_every_time_and_on_any_stream():
    x = gradients([((3_000_001,), BF16), ((777, 1001), F32)], 19)
    norms = []
    for k in range(4):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        ws = fb.grad_workspace(DEV)
        norm = torch.empty(1, device=DEV)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            fb.fopd_grad_norm(fb.GradientList(x), ws, norm=norm, stream=s)
        s.synchronize()
        norms.append(float(ws[0]))
    assert len(set(norms)) == 1


def test_captured_and_replayed():
    x = gradients([((70_000,), BF16), ((33, 77), F32)], 23)
    outs = [torch.empty_like(t) for t in x]
    gl, ws = fb.GradientList(x, outs), fb.grad_workspace(DEV)
    norm, coef, status = scalars()
    fb.fopd_grad_clip(gl, 0.3, ws, norm=norm, coef=coef, status=status)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fb.fopd_grad_clip(gl, 0.3, ws, norm=norm, coef=coef, status=status)
    for k in range(3):
        for t in x:
            t.copy_((torch.randn(t.shape, device=DEV) * (k + 1)).to(t.dtype))
        g.replay()
        torch.cuda.synchronize()
        want_norm, want_coef, want = ro.clip(x, float(np.float32(0.3)))
        assert abs(float(norm) - want_norm) <= U32 * want_norm and abs(float(coef) - want_coef) <= U32 * want_coef
        for o, w in zip(outs, want):
            check_values(o, w, o.dtype)


def test_a_tensor_beyond_32_bit_offsets():
    n = (1 << 31) + 12345
    x = torch.zeros(n, device=DEV, dtype=BF16)
    x[:5] = 3.0
    x[-7:] = 4.0
    norm, coef, status = scalars()
    fb.fopd_grad_clip(fb.GradientList([x]), 1.0, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
    want = math.sqrt(5 * 9 + 7 * 16)
    assert abs(float(norm) - want) <= U32 * want
    assert torch.allclose(x[-7:].float(), torch.tensor(4 / want, device=DEV), rtol=2 ** -8) and float(x[5:-7].abs().max()) == 0


def test_refusals():
    x = gradients([((64,), F32)], 29)[0]
    ws = fb.grad_workspace(DEV)
    with pytest.raises(fb.FopdError) as e:
        fb.fopd_grad_clip(fb.GradientList([x, x]), 1.0, ws)
    assert e.value.code == -7
    with pytest.raises(fb.FopdError):
        fb.fopd_grad_clip(fb.GradientList([x[:40], x[30:]]), 1.0, ws)
    with pytest.raises(fb.FopdError) as e:
        fb.fopd_grad_clip(fb.GradientList([x]), 0.0, ws)
    assert e.value.code == -5
    with pytest.raises(AssertionError):
        fb.GradientList([x.half()])
    with pytest.raises(AssertionError):
        fb.GradientList([x[:1].expand(9)])
    with pytest.raises(AssertionError):
        fb.fopd_grad_clip(fb.GradientList([x]), 1.0, ws[:100])
    fb.fopd_grad_norm(fb.GradientList([x, x]), ws)  # reading twice is no harm


def test_rows_and_columns_of_one_matrix():
    """Blocks that share no element: a block of columns beside single rows, every second row, and pieces without a gap."""
    for pick in [lambda w: [w[:, :8], w[3:4, 8:16]], lambda w: [w[3:4, 8:16], w[:, :8]], lambda w: [w[:, 8:], w[2, :7]],
                 lambda w: [w[:, :8], w[::2, 8:20], w[1::2, 20:], w[1, 9:19]], lambda w: [w[1:9:2], w[:9:2]],
                 lambda w: [w[:, :8], w[1::3, 8:31], w[5, 8:24].view(2, 8), w[6, 9]], lambda w: [w[:, :31], w[:, 31]]]:
        whole = gradients([((12, 32), BF16)], 31)[0]
        assert check_clip(pick(whole), 0.02) < 1


def test_sets_of_random_blocks_are_refused_or_right():
    """Random views of one buffer: where two share an element the set is refused, and a set that is taken comes out right."""
    rng = np.random.RandomState(32)
    taken = refused = 0
    for _ in range(400):
        whole = gradients([((1500,), F32)], 33)[0]
        tensors, used, clash = [], np.zeros(1500, dtype=int), False
        for _ in range(rng.randint(2, 4)):
            pitch = int(rng.choice([12, 24, 24, 36, 48]))
            cols, rows = int(rng.randint(1, 12)), int(rng.randint(1, 9))
            at = int(rng.randint(0, 200))
            tensors.append(whole.as_strided((rows, cols), (pitch, 1), at))
            index = (at + pitch * np.arange(rows)[:, None] + np.arange(cols)).ravel()
            clash |= bool(used[index].any())
            used[index] = 1
        try:
            check_clip(tensors, 0.001)
            taken += 1
            assert not clash
        except fb.FopdError as e:
            assert e.code == -7
            refused += 1
    assert taken > 40 and refused > 40


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale,max_norm", [(1e38, 1e-3), (1e38, 1.0), (1e30, 1e-20), (3e37, 1e-37), (1e10, 1e-35), (2e37, 1e-3)])
def test_coefficients_below_fp32(dtype, scale, max_norm):
    """The coefficient is subnormal in fp32 or nothing there; the gradients come out with norm max_norm all the same.  An
    output is rounded once from the fp64 product (relative error of that below 1e-14).  (At 1e38 some of the normal numbers
    are infinite: that is said, and nothing is scaled.)"""
    shapes = [((50_000,), dtype), ((37, 1000), dtype), ((9, 8), dtype), ((1,), dtype)]
    for place in ("in", "out", "shifted"):
        x = gradients(shapes, 34, scale)
        x[2] = x[2][:, :5]
        whole = [torch.empty(2 * t.numel() + 8, dtype=dtype, device=DEV) for t in x]
        outs = None if place == "in" else [w[(k if place == "out" else 1):].as_strided(t.shape, t.stride())
                                           for k, (w, t) in enumerate(zip(whole, x))]
        if outs:
            outs[2] = torch.empty(9, 8, dtype=dtype, device=DEV)[:, :5]
        m = float(np.float32(max_norm))
        want_norm, want_coef, want = ro.clip(x, m)
        norm, coef, status = scalars()
        fb.fopd_grad_clip(fb.GradientList(x, outs), m, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
        if not math.isfinite(want_norm):
            assert scale == 1e38 and int(status.cpu()[0]) == 128 and float(coef) == 1 and float(norm) == math.inf
            assert all(np.array_equal(o.cpu().double().numpy(), w) for o, w in zip(x if outs is None else outs, want))
            continue
        assert int(status.cpu()[0]) == 0
        assert float(norm) == math.inf if want_norm > 3.5e38 else abs(float(norm) - want_norm) <= U32 * want_norm
        assert want_coef < 2.0 ** -126 and abs(float(coef) - want_coef) <= 2.0 ** -150 * 1.01  # half the smallest subnormal
        step, tiny = (2.0 ** -8, 2.0 ** -134) if dtype == BF16 else (2.0 ** -24, 2.0 ** -150)
        for o, w in zip(x if outs is None else outs, want):
            o = o.cpu().double().numpy()
            assert np.all(np.abs(o - w) <= np.maximum(np.abs(w) * step, tiny) * (1 + 1e-10))


@pytest.mark.parametrize("max_norm", [1.0, 1e38])
def test_a_norm_beyond_fp32_is_finite(max_norm):
    """Two fp32 gradients of 3e38 have a norm of 4.2e38: status and coefficient go by that, the fp32 norm is infinite."""
    x = [torch.full((1,), 3e38, device=DEV), torch.full((1,), -3e38, device=DEV)]
    norm, coef, status = scalars()
    fb.fopd_grad_clip(fb.GradientList(x), max_norm, fb.grad_workspace(DEV), norm=norm, coef=coef, status=status)
    want = float(np.float32(max_norm)) / math.sqrt(2)
    assert int(status.cpu()[0]) == 0 and float(norm) == math.inf
    assert abs(float(x[0]) - want) <= 4 * U32 * want and float(x[1]) == -float(x[0])
    ws = fb.grad_workspace(DEV)
    fb.fopd_grad_norm(fb.GradientList([torch.full((2,), 3e38, device=DEV)]), ws, norm=norm, status=status)
    assert int(status.cpu()[0]) == 0 and float(norm) == math.inf and math.isfinite(float(ws[0]))


def test_clip_of_an_empty_set():
    from paper_2605_17862_b200 import pipeline as pl

    clip = pl.GradientClip([], 1.0)
    assert float(clip()) == 0 and float(clip.coef) == 1
