"""CPU tests of the rollout and clipping entry points: the oracle against its pins, the host-side
argument checks of the library, and the binding's own checks.  No kernel is launched here."""
import ctypes
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2605_17862_b200 import binding as fb
from paper_2605_17862_b200 import build as fbuild
from paper_2605_17862_b200 import pipeline as pl

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    fbuild.build_lib()
    return fb.lib()


# ---- the oracle ----

def test_probabilities_against_torch_and_closed_forms():
    rng = np.random.RandomState(0)
    x = rng.randn(37) * 3
    for T in (0.25, 1.0, 2.0):
        assert np.allclose(ro.probabilities(x, T), torch.softmax(torch.tensor(x) / T, 0).numpy(), rtol=1e-13)
    assert np.allclose(ro.probabilities([0.0, math.log(3.0)], 1.0), [0.25, 0.75], rtol=1e-15)
    assert np.array_equal(ro.probabilities([1.0, 4.0, 4.0], 0), [0, 1, 0])  # ties go to the lowest index
    assert np.array_equal(ro.probabilities([-np.inf, 2.0, -np.inf], 1.0), [0, 1, 0])
    for bad in ([np.nan, 1.0], [np.inf, 1.0], [-np.inf, -np.inf]):
        assert ro.probabilities(bad, 1.0) is None and ro.probabilities(bad, 0) is None


def test_inverse_of_the_distribution_function():
    w = [0.0, 2.0, 0.0, 1.0, 1.0, 0.0]
    assert [ro.invert(w, v) for v in (0.0, 0.49, 0.5, 0.7499, 0.75, 1 - 2 ** -53)] == [1, 1, 3, 3, 4, 4]
    # frequencies over an even grid of numbers are the probabilities
    p = ro.probabilities(np.random.RandomState(1).randn(7), 1.0)
    got = np.bincount([ro.invert(p, (k + 0.5) / 4096) for k in range(4096)], minlength=7) / 4096
    assert np.abs(got - p).max() <= 1 / 4096


@pytest.mark.parametrize("certain", [False, True])
def test_verified_tokens_are_distributed_as_the_target(certain):
    """Over all drafted tokens (weighted by q) and a grid of (u, v): the first token that comes out has the
    target's probabilities, whatever the draft's are."""
    rng = np.random.RandomState(2)
    V, M = 4, 64
    t, d = rng.randn(2, V) * 1.5, rng.randn(1, V) * 1.5
    p = ro.probabilities(t[0], 1.0)
    q = np.eye(V)[2] if certain else ro.probabilities(d[0], 1.0)
    got = np.zeros(V)
    grid = (np.arange(M) + 0.5) / M
    for x in range(V):
        if q[x] == 0:
            continue
        for u, v in itertools.product(grid, grid):
            tokens, lps, acc, why, bad = ro.verify(t, None if certain else d, [x], 1, [u, v], 1.0, 1.0)
            assert why == "" and not bad and len(tokens) == acc + 1
            assert np.allclose(lps, [math.log(ro.probabilities(t[k], 1.0)[y]) for k, y in enumerate(tokens)])
            got[tokens[0]] += q[x] / M ** 2
    assert np.abs(got - p).max() <= 3 / M  # a grid of M points has every probability to 1/M: test, residual


def test_verify_hand_cases():
    u8 = np.zeros((2, 8))
    half = np.where(np.arange(8) < 4, 0.0, -np.inf)[None]
    # p = 1/8, q = 1/4: accepted below u = 1/2, not at it; the residual is even over the other half
    assert ro.verify(u8, half, [1], 1, [0.4999, 0.3], 1.0, 1.0)[0][0] == 1
    tokens, lps, acc, why, bad = ro.verify(u8, half, [1], 1, [0.5, 0.3], 1.0, 1.0)
    assert tokens == [5] and acc == 0 and lps == [math.log(1 / 8)]
    # the draft is the target: always accepted, unless it has probability 0 in both, when the residual is empty
    assert ro.verify(u8, u8[:1], [3], 1, [0.999, 0.0], 1.0, 1.0)[2] == 1
    m = np.where(np.arange(8) < 4, 0.0, -np.inf)[None].repeat(2, 0)
    assert ro.verify(m, m[:1], [6], 1, [0.0, 0.6], 1.0, 1.0)[:3] == ([2], [math.log(1 / 4)], 0)
    # a certain draft: accepted with its own probability, else drawn from the others
    assert ro.verify(u8, None, [3], 1, [0.124, 0.0], 1.0, 1.0)[2] == 1
    assert ro.verify(u8, None, [3], 1, [0.125, 0.5], 1.0, 1.0)[0] == [4]
    # temperature 0: the draft's probabilities decide nothing
    assert ro.verify(np.eye(8)[[2, 5]], u8[:1], [2], 1, [0.99, 0.99], 0.0, 1.0)[0] == [2, 5]
    assert ro.verify(u8, None, [9], 1, [0.1, 0.0], 1.0, 1.0)[4]  # out of range


def test_clip_hand_cases():
    norm, coef, out = ro.clip([np.array([3.0]), np.array([[4.0, 0.0]])], 2.5)
    assert (norm, coef) == (5.0, 0.5) and np.array_equal(out[1], [[2.0, 0.0]])
    assert ro.clip([np.array([3.0])], 3.0)[1] == 1.0
    assert ro.clip([np.array([np.inf])], 3.0)[1] == 1.0 and ro.clip([], 1.0)[:2] == (0.0, 1.0)


# ---- the library's host-side checks ----

def _draft(**kw):
    base = dict(target=0x10000, draft=0x20000, tokens=0x30000, n_draft=None, uniform=0x40000, vocab=64,
                target_seq_stride=320, target_row_stride=64, draft_seq_stride=256, draft_row_stride=64, B=2, K=4, dtype=0,
                temperature=1.0, draft_temperature=1.0)
    base.update(kw)
    return fb.fopd_draft(*[base[f] for f, _ in fb.fopd_draft._fields_])


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -4), (dict(B=-1), -3), (dict(K=-1), -3), (dict(K=1 << 20), -3), (dict(vocab=0), -3),
    (dict(vocab=(1 << 30) + 1), -3), (dict(target_row_stride=56), -3), (dict(draft_row_stride=56), -3),
    (dict(target_seq_stride=-64), -3), (dict(draft_seq_stride=-64), -3),
    (dict(temperature=-1.0), -5), (dict(temperature=float("nan")), -5), (dict(temperature=float("inf")), -5),
    (dict(temperature=1e-4), -5), (dict(draft_temperature=-0.5), -5), (dict(draft_temperature=4096.0), -5),
    (dict(target=0), -1), (dict(tokens=0), -1), (dict(uniform=0), -1),
    (dict(target=0x10008), -2), (dict(draft=0x20002), -2), (dict(target_row_stride=68), -2), (dict(draft_row_stride=65), -2),
    (dict(target_seq_stride=324), -2), (dict(draft_seq_stride=260), -2),
    (dict(B=0), 0),
])
def test_verify_checks_its_arguments_on_the_host(lib, kw, code):
    d = _draft(**kw)
    assert lib.fopd_verify_draft(ctypes.byref(d), vp(0x50000), None, None, None, None, None) == code


@pytest.mark.parametrize("kw,outs,code", [
    (dict(tokens=0x50000), {}, -7),                                  # tokens onto the drafted ones
    (dict(tokens=0x50000 + 39), {}, -7), (dict(tokens=0x50000 - 31), {}, -7),
    (dict(uniform=0x50000 + 39), {}, -7), (dict(n_draft=0x50000 - 7), {}, -7),
    (dict(), dict(logprob=0x40000 + 79), -7), (dict(), dict(mask=0x30000 - 9), -7),
    (dict(n_draft=0x60000), dict(n_accepted=0x60000), -7), (dict(n_draft=0x60000), dict(n_accepted=0x60000 + 7), -7),
    (dict(K=0, uniform=0x50000), {}, -7), (dict(B=0, tokens=0x50000), {}, 0),
])
def test_outputs_on_inputs_are_refused(lib, kw, outs, code):
    d = _draft(**kw)
    out = [vp(outs[k]) if k in outs else None for k in ("logprob", "mask", "n_accepted")]
    assert lib.fopd_verify_draft(ctypes.byref(d), vp(0x50000), *out, None, None) == code


def test_draws_onto_their_numbers_are_refused(lib):
    f = lib.fopd_draw_tokens
    assert f(vp(0x10000), vp(0x40000), 2, 64, 64, 0, 1.0, vp(0x40000 + 15), None, None, None) == -7
    assert f(vp(0x10000), vp(0x40000), 2, 64, 64, 0, 1.0, vp(0x50000), vp(0x40000 - 7), None, None) == -7


def test_draw_and_null_arguments(lib):
    f = lib.fopd_draw_tokens
    ok = [vp(0x10000), vp(0x40000), 2, 64, 64, 0, 1.0, vp(0x50000), None, None, None]

    def call(i, x):
        a = list(ok)
        a[i] = x
        return f(*a)

    assert lib.fopd_verify_draft(None, vp(0x50000), None, None, None, None, None) == -1
    assert lib.fopd_verify_draft(ctypes.byref(_draft()), None, None, None, None, None, None) == -1
    assert [call(0, None), call(1, None), call(7, None)] == [-1, -1, -1]
    assert [call(2, -1), call(2, 1 << 31), call(3, 0), call(4, 63)] == [-3] * 4
    assert [call(0, vp(0x10004)), call(4, 68)] == [-2, -2]
    assert call(5, 9) == -4 and call(6, -0.1) == -5 and call(2, 0) == 0


def _tensor(**kw):
    base = dict(data=0x10000, out=None, rows=4, cols=8, row_stride=8, dtype=0, reserved=0)
    base.update(kw)
    return fb.fopd_tensor(*[base[f] for f, _ in fb.fopd_tensor._fields_])


def test_gradient_calls_check_their_arguments_on_the_host(lib):
    ws = vp(0x80000)

    def norm(*ts, ws=ws, n=None):
        arr = (fb.fopd_tensor * max(1, len(ts)))(*ts)
        return lib.fopd_grad_norm(arr, len(ts) if n is None else n, ws, None, None, None)

    def scale(*ts, m=1.0):
        arr = (fb.fopd_tensor * max(1, len(ts)))(*ts)
        rc = lib.fopd_grad_scale(arr, len(ts), ws, m, None, None, None, None)
        assert rc == lib.fopd_grad_clip(arr, len(ts), ws, m, None, None, None, None)
        return rc

    assert norm(_tensor(), ws=None) == -1 and norm(_tensor(), ws=vp(0x80008)) == -2 and norm(_tensor(), n=-1) == -3
    assert lib.fopd_grad_norm(None, 1, ws, None, None, None) == -1
    for kw, code in [(dict(dtype=2), -4), (dict(rows=-1), -3), (dict(cols=-1), -3), (dict(cols=1 << 43, rows=1), -3),
                     (dict(row_stride=7), -3), (dict(rows=1 << 30, row_stride=1 << 20), -3), (dict(data=0), -1),
                     (dict(data=0x10001), -2), (dict(out=0x20001), -2), (dict(dtype=1, data=0x10002), -2)]:
        assert norm(_tensor(**kw)) == code and scale(_tensor(), _tensor(data=0x90000, **kw) if "data" not in kw else
                                                     _tensor(**kw)) == code, kw
    for m in (0.0, -1.0, float("nan"), float("inf")):
        assert scale(_tensor(), m=m) == -5
    # overlaps with something that is written
    assert scale(_tensor(), _tensor()) == -7                                    # the same tensor twice
    assert scale(_tensor(), _tensor(data=0x10000 + 62)) == -7
    assert scale(_tensor(out=0x10002)) == -7                                    # shifted against its own data
    assert scale(_tensor(out=0x20000), _tensor(data=0x20010, out=0x30000)) == -7
    assert scale(_tensor(data=0x30000, out=0x20000), _tensor(data=0x10000, out=0x20000)) == -7
    # column blocks of one matrix meet only where their columns do
    a = _tensor(cols=8, row_stride=32)
    assert scale(a, _tensor(data=0x10000 + 14, cols=8, row_stride=32)) == -7


def test_rows_and_columns_of_one_matrix_that_meet_are_refused(lib):
    """bf16 blocks of a matrix with 32 columns (64 bytes)."""
    def scale(*ts):
        arr = (fb.fopd_tensor * len(ts))(*ts)
        return lib.fopd_grad_scale(arr, len(ts), vp(0x80000), 1.0, None, None, None, None)

    def block(row, col, rows, cols, stride=32):
        return _tensor(data=0x10000 + 2 * (32 * row + col), rows=rows, cols=cols, row_stride=stride)

    a = block(0, 8, 6, 8)
    for other in [block(2, 15, 1, 4), block(2, 4, 1, 5), block(5, 8, 1, 8), block(1, 0, 1, 64), block(0, 0, 1, 9),
                  block(1, 15, 3, 2, 64), block(0, 30, 3, 11, 64), block(2, 16, 2, 25, 64), block(3, 16, 4, 8, 8)]:
        assert scale(a, other) == -7 and scale(other, a) == -7
    assert scale(block(0, 0, 3, 8, 64), block(1, 4, 3, 8, 96)) == -7  # every second row and every third from row 1: row 4


# ---- the binding's view of a tensor ----

def test_layouts_of_tensors():
    f = fb._as_rows
    x = torch.zeros(6, 5, 4)
    assert f(x) == f(x.permute(2, 0, 1)) == (1, 120, 120) and f(torch.zeros(())) == (1, 1, 1)
    assert f(x[:, :, :3]) == (30, 3, 4) and f(x[:, 1:3]) == (6, 8, 20) and f(x[2:4]) == (1, 40, 40)
    assert f(x[:, ::2]) is None and f(x[:, 1:3, :2]) is None and f(torch.zeros(3, 1).expand(3, 4)) is None
    assert f(torch.zeros(0, 5)) == (0, 0, 0) and f(torch.zeros(5, 7).t()) == (1, 35, 35)
    assert f(torch.zeros(9, 8)[:, :1]) == (9, 1, 8)
    wide = torch.zeros(4, 16)
    assert f(wide[:, 3:9]) == (4, 6, 16) and f(wide[:, 3:9].t()) == (4, 6, 16)


def test_cpu_tensors_are_refused():
    x = torch.zeros(2, 8)
    with pytest.raises(AssertionError):
        fb.fopd_draw_tokens(x, torch.zeros(2, dtype=torch.float64), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(AssertionError):
        fb.GradientList([x])


# ---- a rollout as a chunk of the loss ----

def test_log_probs_at_another_temperature_are_not_taken_for_the_policys():
    B, K, V = 2, 3, 16
    target, teacher = torch.zeros(2, B, K + 1, V).unbind(0)
    sid = torch.arange(B, dtype=torch.int32)
    out = pl.Rollout.alloc(B, K, "cpu")
    assert out.temperature == 1.0
    assert pl.rollout_chunk(target, teacher, out, sid).behav_logprob.data_ptr() == out.logprob.data_ptr()
    lp = torch.ones(B, K + 1)
    for T in (0.7, 0.0):
        out.temperature = T
        with pytest.raises(AssertionError):
            pl.rollout_chunk(target, teacher, out, sid)
        assert torch.equal(pl.rollout_chunk(target, teacher, out, sid, behav_logprob=lp).behav_logprob, lp.view(-1))


def test_rollouts_of_one_sequence_or_one_row_as_chunks():
    """Views whose stride along a dimension of one is not what rows at one pitch would have."""
    buf = torch.arange(2 * 5 * 16, dtype=torch.float32).view(2, 5, 16)
    for target in (buf[:1, :3, :9], buf[1:, 1:4, :9], buf[:, :1, :9], buf[:, 4, :9].unsqueeze(1), buf[:1, :1, :9], buf[:, :, :9]):
        B, W, V = target.shape
        out = pl.Rollout.alloc(B, W - 1, "cpu")
        chunk = pl.rollout_chunk(target, target.clone() if target.is_contiguous() else target, out, torch.arange(B))
        assert torch.equal(chunk.student, target.reshape(B * W, V)) and torch.equal(chunk.teacher, chunk.student)
        assert chunk.student.data_ptr() == target.data_ptr()
    for bad in (buf[:, :3, :9], buf.transpose(0, 1)[:, :, :9]):
        with pytest.raises(AssertionError):
            pl.rollout_chunk(bad, None, pl.Rollout.alloc(bad.shape[0], bad.shape[1] - 1, "cpu"), torch.arange(bad.shape[0]))
    with pytest.raises(AssertionError):  # the teacher's rows
        pl.rollout_chunk(buf[:, :, :9], buf[:, :3, :9], pl.Rollout.alloc(2, 4, "cpu"), torch.arange(2))


@pytest.mark.parametrize("code,words", [(-2, ("16-byte", "gradient")), (-3, ("cols",)), (-5, ("temperature", "max_norm", "alpha")),
                                        (-7, ("output", "set", "dlogits")), (-8, ("logits", "uniform", "gradient"))])
def test_errors_name_what_these_calls_refuse(lib, code, words):
    text = str(fb.FopdError(code, "f"))
    assert all(w in text for w in words), text
