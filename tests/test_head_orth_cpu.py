"""CPU tests of the head and orthogonalisation entry points: what the host refuses before any CUDA call, and the oracle against
cases that can be worked out by hand."""
import ctypes
import math

import pytest
import torch

from oracle import orth_oracle as oo
from paper_2605_17862_b200 import binding as fb
from paper_2605_17862_b200 import build as fbuild

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    fbuild.build_lib()
    return fb.lib()


def head(**kw):
    base = dict(hidden=0x10000, weight=0x20000, tokens=0x30000, mask=0, n_rows=4, vocab=64, dim=40, hidden_stride=40, weight_stride=48,
                dtype=0, reserved=0)
    base.update(kw)
    return fb.fopd_head(*[base[f] for f, _ in fb.fopd_head._fields_])


BAD_HEADS = [(dict(dtype=1), -4), (dict(dtype=7), -4), (dict(n_rows=-1), -3), (dict(n_rows=(1 << 27) + 1), -3), (dict(vocab=0), -3),
             (dict(vocab=(1 << 30) + 1), -3), (dict(dim=0), -3), (dict(dim=(1 << 20) + 1), -3), (dict(hidden_stride=32), -3),
             (dict(weight_stride=32), -3), (dict(weight_stride=1 << 40), -3), (dict(hidden=0), -1), (dict(weight=0), -1), (dict(tokens=0), -1),
             (dict(hidden=0x10008), -2), (dict(weight=0x20002), -2), (dict(hidden_stride=44), -2), (dict(weight_stride=50), -2)]


@pytest.mark.parametrize("kw,code", BAD_HEADS)
def test_head_refusals(lib, kw, code):
    h = head(**kw)
    assert lib.fopd_head_logprob(ctypes.byref(h), vp(0x40000), None, None, None) == code
    assert lib.fopd_head_grad(ctypes.byref(h), vp(0x40000), vp(0x41000), vp(0x42000), vp(0x50000), 40, vp(0x60000), 48, 0, 0, None,
                              None) == code


def test_head_more_refusals(lib):
    h, lp, lse, coef, dh, dw = head(), vp(0x40000), vp(0x41000), vp(0x42000), vp(0x50000), vp(0x60000)
    logprob = lambda *a, h=h: lib.fopd_head_logprob(ctypes.byref(h), *a, None, None)
    grad = lambda *a, h=h: lib.fopd_head_grad(ctypes.byref(h), *a, None, None)
    assert lib.fopd_head_logprob(None, lp, None, None, None) == -1
    assert logprob(None, lse) == -1
    for out in (0x10000, 0x10000 + 3 * 80 + 76, 0x20000, 0x30000, 0x30000 - 12, 0x30000 + 12):  # on hidden states, weights, tokens
        assert logprob(vp(out), None) == -7 and logprob(lp, vp(out)) == -7
    assert logprob(lp, vp(0x40000 + 12)) == -7
    assert logprob(vp(0x70000), None, h=head(mask=0x70003)) == -7
    assert logprob(lp, None, h=head(n_rows=0, hidden=0, weight=0, tokens=0)) == 0
    assert grad(lp, lse, coef, None, 0, None, 0, 0, 0) == -1
    assert grad(None, lse, coef, dh, 40, dw, 48, 0, 0) == grad(lp, None, coef, dh, 40, dw, 48, 0, 0) == -1
    assert grad(lp, lse, None, dh, 40, dw, 48, 0, 0) == -1
    assert grad(lp, lse, coef, dh, 40, dw, 48, 2, 0) == -4
    assert grad(lp, lse, coef, dh, 32, dw, 48, 0, 0) == grad(lp, lse, coef, dh, 40, dw, 39, 0, 0) == -3
    assert grad(lp, lse, coef, vp(0x50008), 40, dw, 48, 0, 0) == grad(lp, lse, coef, dh, 44, dw, 48, 0, 0) == -2
    assert grad(lp, lse, coef, dh, 40, vp(0x60004), 48, 0, 0) == grad(lp, lse, coef, dh, 40, dw, 42, 1, 0) == -2
    for out in (0x10000, 0x20000 + 63 * 96 + 64, 0x30000, 0x40000, 0x41000, 0x42000):
        assert grad(lp, lse, coef, vp(out), 40, None, 0, 0, 0) == -7
        assert grad(lp, lse, coef, None, 0, vp(out), 48, 0, 0) == -7
    assert grad(lp, lse, coef, vp(0x60000 + 128), 40, dw, 48, 0, 0) == -7


def matrix(**kw):
    base = dict(data=0x10000, out=0x20000, rows=8, cols=10, row_stride=10, out_stride=12, scale=1.0, dtype=0, out_dtype=1, reserved=0)
    base.update(kw)
    return fb.fopd_matrix(*[base[f] for f, _ in fb.fopd_matrix._fields_])


def orth(lib, ms, cs=((1.5, -0.5, 0.0),), eps=1e-7, n=None, steps=None):
    flat = [x for c in cs for x in c]
    arr = (fb.fopd_matrix * max(1, len(ms)))(*ms)
    return lib.fopd_orthogonalise(arr, len(ms) if n is None else n, (ctypes.c_float * max(1, len(flat)))(*flat),
                                  len(cs) if steps is None else steps, eps, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -4), (dict(out_dtype=-1), -4), (dict(scale=math.inf), -5), (dict(scale=math.nan), -5), (dict(rows=-1), -3),
    (dict(cols=(1 << 24) + 1), -3), (dict(row_stride=9), -3), (dict(out_stride=9), -3), (dict(row_stride=1 << 40), -3),
    (dict(rows=1 << 24, cols=1 << 14, row_stride=1 << 14, out_stride=1 << 14), -3), (dict(data=0), -1), (dict(out=0), -1),
    (dict(data=0x10001), -2), (dict(out=0x20002), -2), (dict(out=0x10000), -7), (dict(out=0x10000 + 20, out_dtype=0), -7),
    (dict(data=0x20000, out=0x20000, out_dtype=0), -7),  # in place at another pitch
])
def test_orthogonalise_refusals(lib, kw, code):
    assert orth(lib, [matrix(**kw)]) == code


def test_orthogonalise_more_refusals(lib):
    m = matrix()
    assert lib.fopd_orthogonalise(None, 1, (ctypes.c_float * 3)(1, 0, 0), 1, 0.0, None, None) == -1
    assert lib.fopd_orthogonalise((fb.fopd_matrix * 1)(m), 1, None, 1, 0.0, None, None) == -1
    assert orth(lib, [m], n=-1) == -3
    for steps in (0, -1, 17):
        assert orth(lib, [m], [(1.0, 0.0, 0.0)] * 17, steps=steps) == -5
    for eps in (-1e-9, math.inf, math.nan):
        assert orth(lib, [m], eps=eps) == -5
    for c in ((math.nan, 0, 0), (0, math.inf, 0), (0, 0, -math.inf), (2e6, 0, 0), (1, 2e6, 0)):
        assert orth(lib, [m], [c]) == -5
    assert orth(lib, [m], [(100.0, 0, 0)] * 4) == -5  # 100^4
    # two results on one another, a result on another matrix, the same matrix twice in place
    assert orth(lib, [matrix(), matrix(data=0x30000, out=0x20000 + 40)]) == -7
    assert orth(lib, [matrix(), matrix(data=0x20000 + 16, out=0x40000)]) == -7
    same = dict(data=0x10000, out=0x10000, out_stride=10, out_dtype=0)
    assert orth(lib, [matrix(**same), matrix(**same)]) == -7
    # nothing to do: no CUDA call
    assert orth(lib, []) == 0
    assert orth(lib, [matrix(rows=0, data=0, out=0), matrix(cols=0, data=0, out=0)]) == 0


@pytest.mark.parametrize("shape", [(3, 3), (2, 5), (6, 2)])
def test_oracle_on_diagonal_matrices(shape):
    """Singular values go through a s + b s^3 + c s^5 one by one."""
    cs = [(3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375)]
    s = torch.tensor([3.0, -0.5, 0.01][:min(shape)], dtype=torch.float64)
    M = torch.zeros(shape, dtype=torch.float64)
    M[range(len(s)), range(len(s))] = s
    x = s / (s.square().sum().sqrt() + 0.25)
    for a, b, c in cs:
        x = a * x + b * x ** 3 + c * x ** 5
    want = torch.zeros(shape, dtype=torch.float64)
    want[range(len(s)), range(len(s))] = 2 * x
    assert torch.allclose(oo.orthogonalise(M, cs, eps=0.25, scale=2.0), want, rtol=1e-13, atol=1e-15)


def test_oracle_leaves_singular_vectors_alone():
    g = torch.Generator().manual_seed(0)
    M = torch.randn((7, 11), generator=g, dtype=torch.float64)
    u, s, v = torch.linalg.svd(M, full_matrices=False)
    x = s / s.square().sum().sqrt()
    for a, b, c in fb.NEWTON_SCHULZ_COEFFICIENTS:
        x = a * x + b * x ** 3 + c * x ** 5
    assert torch.allclose(oo.orthogonalise(M, fb.NEWTON_SCHULZ_COEFFICIENTS, eps=0.0), u * x @ v, rtol=0, atol=1e-12)
    assert oo.rounding_error(M, fb.NEWTON_SCHULZ_COEFFICIENTS, full=True)[0] < 1e-5
    assert 1e-5 < oo.rounding_error(M, fb.NEWTON_SCHULZ_COEFFICIENTS)[0] < 1e-1


def test_structs_match_the_header():
    assert ctypes.sizeof(fb.fopd_head) == 4 * 8 + 5 * 8 + 8
    assert ctypes.sizeof(fb.fopd_matrix) == 2 * 8 + 4 * 8 + 16


def test_matrix_list_takes_device_matrices_only():
    with pytest.raises(AssertionError):
        fb.MatrixList([torch.zeros(3, 4)])
