"""Thin ctypes binding of libfopd.so: same names as the C ABI, torch tensors in,
pointers out.  Argument marshalling only -- every step of the path runs in the
library's CUDA kernels.  There is no CPU fallback: if the shared library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfopd.so")

FOPD_BF16, FOPD_F32 = 0, 1
LOSS_FULL_KL, LOSS_SAMPLED_KL = 0, 1  # forms of the token loss (fopd_loss_kind)

EXPORTS = (
    "fopd_token_stats", "fopd_sample_freshness", "fopd_loss_fwd_bwd", "fopd_loss_finalize",
    "fopd_check_status", "fopd_strerror", "fopd_version", "fopd_step_host", "fopd_step_host_workspace_bytes",
    "fopd_token_stats_static", "fopd_loss_fwd_bwd_plan", "fopd_row_divergence", "fopd_supervision_drift",
    "fopd_refresh_decision", "fopd_shard_stats", "fopd_shard_merge", "fopd_shard_loss_fwd_bwd",
    "fopd_loss_fwd_bwd_set_plan", "fopd_release_device_memory", "fopd_selftest_bounded_wait",
    "fopd_token_stats_student", "fopd_draw_tokens", "fopd_verify_draft", "fopd_grad_norm", "fopd_grad_scale",
    "fopd_grad_clip", "fopd_head_logprob", "fopd_head_grad", "fopd_orthogonalise",
)
GRAD_WS = 2048  # doubles of the workspace of fopd_grad_norm, fopd_grad_scale and fopd_grad_clip


class FopdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (status {code})")


class fopd_params(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("beta", ctypes.c_float), ("xi", ctypes.c_float),
                ("lam", ctypes.c_float)]


class fopd_chunk(ctypes.Structure):
    _fields_ = [
        ("student", ctypes.c_void_p), ("teacher", ctypes.c_void_p), ("behav_logprob", ctypes.c_void_p),
        ("tokens", ctypes.c_void_p), ("mask", ctypes.c_void_p), ("sample_id", ctypes.c_void_p),
        ("n_rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("row_stride", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("loss_kind", ctypes.c_int32),
    ]


class fopd_host_outputs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("f", "w", "d_roll", "l_distill", "m_align", "per_sample_loss", "buffer_means", "loss",
                 "status_bits", "copied_bytes")]


class fopd_draft(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("target", "draft", "tokens", "n_draft", "uniform")] + \
        [(n, ctypes.c_int64) for n in ("vocab", "target_seq_stride", "target_row_stride", "draft_seq_stride",
                                       "draft_row_stride")] + \
        [("temperature", ctypes.c_double), ("draft_temperature", ctypes.c_double), ("B", ctypes.c_int32),
         ("K", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class fopd_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class fopd_head(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("hidden", "weight", "tokens", "mask")] + \
        [(n, ctypes.c_int64) for n in ("n_rows", "vocab", "dim", "hidden_stride", "weight_stride")] + \
        [("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class fopd_matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p)] + \
        [(n, ctypes.c_int64) for n in ("rows", "cols", "row_stride", "out_stride")] + \
        [("scale", ctypes.c_float), ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libfopd.so (built in-tree by ``build.build_lib``); fails loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2605_17862_b200.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        L.fopd_version.restype = ctypes.c_int
        L.fopd_strerror.restype = ctypes.c_char_p
        L.fopd_strerror.argtypes = [ctypes.c_int]
        L.fopd_token_stats.argtypes = [ctypes.POINTER(fopd_chunk), i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.fopd_token_stats_student.argtypes = [ctypes.POINTER(fopd_chunk), i32, vp, vp, vp, vp, vp]
        L.fopd_token_stats_static.argtypes = [ctypes.POINTER(fopd_chunk), i32, vp, vp, vp, vp, vp, vp, vp]
        L.fopd_sample_freshness.argtypes = [vp, vp, vp, vp, i32, fopd_params, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.fopd_loss_fwd_bwd.argtypes = [ctypes.POINTER(fopd_chunk), i32, vp, vp, fopd_params, vp, vp, vp, vp]
        L.fopd_loss_fwd_bwd_plan.argtypes = [i32, ctypes.c_int64] + [ctypes.POINTER(ctypes.c_int32)] * 4
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.fopd_loss_fwd_bwd_set_plan.argtypes = [i32, i64, i32]
        L.fopd_release_device_memory.argtypes = []
        L.fopd_selftest_bounded_wait.argtypes = [i64, vp, vp, vp]
        L.fopd_row_divergence.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp]
        L.fopd_supervision_drift.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        L.fopd_refresh_decision.argtypes = [vp, vp, vp, i32, f32, f32, f32, i64, i64, vp, vp, vp]
        L.fopd_shard_stats.argtypes = [ctypes.POINTER(fopd_chunk), i64, i64, vp, vp]
        L.fopd_shard_merge.argtypes = [vp, i32, ctypes.POINTER(fopd_chunk), i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.fopd_shard_loss_fwd_bwd.argtypes = [ctypes.POINTER(fopd_chunk), i64, i64, i32, vp, vp, fopd_params, vp, vp,
                                              vp]
        L.fopd_loss_finalize.argtypes = [vp, vp, vp, i32, fopd_params, vp, vp, vp]
        L.fopd_check_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
        L.fopd_step_host_workspace_bytes.restype = ctypes.c_uint64
        L.fopd_step_host_workspace_bytes.argtypes = [ctypes.POINTER(fopd_chunk), i32, i32, i32]
        L.fopd_step_host.argtypes = [ctypes.POINTER(fopd_chunk), i32, i32, vp, vp, vp, fopd_params,
                                     ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(fopd_host_outputs), vp,
                                     ctypes.c_uint64, vp]
        L.fopd_draw_tokens.argtypes = [vp, vp, i64, i64, i64, i32, ctypes.c_double, vp, vp, vp, vp]
        L.fopd_verify_draft.argtypes = [ctypes.POINTER(fopd_draft), vp, vp, vp, vp, vp, vp]
        L.fopd_grad_norm.argtypes = [vp, i32, vp, vp, vp, vp]
        L.fopd_grad_scale.argtypes = [vp, i32, vp, f32, vp, vp, vp, vp]
        L.fopd_grad_clip.argtypes = [vp, i32, vp, f32, vp, vp, vp, vp]
        L.fopd_head_logprob.argtypes = [ctypes.POINTER(fopd_head), vp, vp, vp, vp]
        L.fopd_head_grad.argtypes = [ctypes.POINTER(fopd_head), vp, vp, vp, vp, i64, vp, i64, i32, i32, vp, vp]
        L.fopd_orthogonalise.argtypes = [vp, i32, vp, i32, f32, vp, vp]
        for name in EXPORTS:
            getattr(L, name)
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().fopd_strerror(int(code)).decode()


def version() -> int:
    return int(lib().fopd_version())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    # (the raw handle of the current stream: torch.cuda.current_stream() takes longer than a small kernel)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _check(rc: int, where: str):
    if rc != 0:
        raise FopdError(rc, where)


def params(alpha=1.0, beta=1.0, xi=0.15, lam=0.1) -> fopd_params:
    return fopd_params(float(alpha), float(beta), float(xi), float(lam))


@dataclass
class Chunk:
    """Device tensors of one chunk of token rows (see ``fopd_chunk`` in fopd.h)."""
    student: torch.Tensor  # [n, V] (row pitch = student.stride(0)), bf16 or fp32
    teacher: torch.Tensor | None  # None only for fopd_token_stats_student
    behav_logprob: torch.Tensor  # [n] fp32
    tokens: torch.Tensor  # [n] int32
    mask: torch.Tensor  # [n] uint8
    sample_id: torch.Tensor  # [n] int32
    vocab: int | None = None  # columns in use; defaults to student.shape[1]
    loss_kind: int = LOSS_FULL_KL

    def c_struct(self) -> fopd_chunk:
        S, T = self.student, self.teacher
        assert S.dtype in (torch.bfloat16, torch.float32) and S.dim() == 2 and S.stride(1) == 1
        assert T is None or (S.dtype == T.dtype and S.shape == T.shape and S.stride() == T.stride())
        assert self.behav_logprob.dtype == torch.float32 and self.tokens.dtype == torch.int32
        assert self.mask.dtype == torch.uint8 and self.sample_id.dtype == torch.int32
        n = S.shape[0]
        for t in (self.behav_logprob, self.tokens, self.mask, self.sample_id):
            assert t.is_contiguous() and t.numel() == n and t.device == S.device
        return fopd_chunk(
            S.data_ptr(), None if T is None else T.data_ptr(), self.behav_logprob.data_ptr(), self.tokens.data_ptr(),
            self.mask.data_ptr(), self.sample_id.data_ptr(), n, self.vocab or S.shape[1],
            S.stride(0) if n > 1 else max(S.stride(0), S.shape[1]),
            FOPD_BF16 if S.dtype == torch.bfloat16 else FOPD_F32, int(self.loss_kind),
        )


def fopd_token_stats(chunk: Chunk, B: int, acc, *, lp_s=None, lp_t=None, kl=None, ratio=None,
                     row_ws=None, status=None, stream=None):
    c = chunk.c_struct()
    _check(lib().fopd_token_stats(ctypes.byref(c), B, _ptr(lp_s), _ptr(lp_t), _ptr(kl), _ptr(ratio),
                                  _ptr(row_ws), _ptr(acc), _ptr(status), _stream(stream)),
           "fopd_token_stats")


def fopd_token_stats_student(chunk: Chunk, B: int, acc, *, lp_s=None, ratio=None, status=None, stream=None):
    """The student's half of fopd_token_stats (chunk.teacher may be None): enough for
    fopd_sample_freshness; the loss call that follows gets no row_ws."""
    c = chunk.c_struct()
    _check(lib().fopd_token_stats_student(ctypes.byref(c), B, _ptr(lp_s), _ptr(ratio), _ptr(acc), _ptr(status),
                                          _stream(stream)),
           "fopd_token_stats_student")


STATIC_MAX_ROWS = 65536
STATIC_MAX_SAMPLES = 16384


def fopd_token_stats_static(chunk: Chunk, B: int, acc, *, lp_s=None, lp_t=None, kl=None, ratio=None,
                            status=None, stream=None):
    """fopd_token_stats without any device allocation: the per-row scratch is a
    fixed 1 MiB array inside the library (at most STATIC_MAX_ROWS rows per call).
    For callers that have given all GPU memory to their own allocator or that
    forbid allocations inside their step loop.  Calls on one device share the
    scratch, so keep them on one stream."""
    c = chunk.c_struct()
    _check(lib().fopd_token_stats_static(ctypes.byref(c), B, _ptr(lp_s), _ptr(lp_t), _ptr(kl), _ptr(ratio),
                                         _ptr(acc), _ptr(status), _stream(stream)),
           "fopd_token_stats_static")


def fopd_sample_freshness(acc, staleness, seq_len, d_sup, B: int, p: fopd_params, *, coef, f=None,
                          w=None, d_roll=None, l_distill=None, m_align=None, buffer_means=None,
                          status=None, stream=None):
    _check(lib().fopd_sample_freshness(_ptr(acc), _ptr(staleness), _ptr(seq_len), _ptr(d_sup), B, p,
                                       _ptr(f), _ptr(w), _ptr(d_roll), _ptr(l_distill), _ptr(m_align),
                                       _ptr(coef), _ptr(buffer_means), _ptr(status), _stream(stream)),
           "fopd_sample_freshness")


def fopd_loss_fwd_bwd(chunk: Chunk, B: int, coef, p: fopd_params, dlogits, loss_acc, *, row_ws=None,
                      status=None, stream=None):
    c = chunk.c_struct()
    assert dlogits.dtype == chunk.student.dtype and dlogits.stride() == chunk.student.stride()
    _check(lib().fopd_loss_fwd_bwd(ctypes.byref(c), B, _ptr(coef), _ptr(row_ws), p, _ptr(dlogits),
                                   _ptr(loss_acc), _ptr(status), _stream(stream)),
           "fopd_loss_fwd_bwd")


def fopd_loss_fwd_bwd_plan(dtype: torch.dtype, vocab: int) -> dict:
    """Launch shape of fopd_loss_fwd_bwd(row_ws=None) on the current device (cluster_size 0:
    the streaming kernel pair is used instead)."""
    out = [ctypes.c_int32(0) for _ in range(4)]
    _check(lib().fopd_loss_fwd_bwd_plan(FOPD_BF16 if dtype == torch.bfloat16 else FOPD_F32, int(vocab),
                                        *[ctypes.byref(o) for o in out]), "fopd_loss_fwd_bwd_plan")
    return dict(zip(("cluster_size", "block_threads", "resident_clusters", "smem_bytes"),
                    (int(o.value) for o in out)))


def fopd_loss_fwd_bwd_set_plan(dtype: torch.dtype, vocab: int, cluster_size: int) -> None:
    """Pins the on-chip launch shape for (current device, dtype, vocab): cluster_size > 0 CTAs per
    cluster, < 0 the streaming kernel pair, 0 back to the library's own choice."""
    _check(lib().fopd_loss_fwd_bwd_set_plan(FOPD_BF16 if dtype == torch.bfloat16 else FOPD_F32, int(vocab),
                                            int(cluster_size)), "fopd_loss_fwd_bwd_set_plan")


def fopd_release_device_memory() -> None:
    """Trims the library's memory pool on the current device and drops fopd_step_host's streams."""
    _check(lib().fopd_release_device_memory(), "fopd_release_device_memory")


def fopd_selftest_bounded_wait(limit_cycles: int, status, waited_cycles=None, *, stream=None) -> None:
    """Runs one bounded barrier wait that cannot complete; the kernel sets the timeout bit in ``status``."""
    _check(lib().fopd_selftest_bounded_wait(int(limit_cycles), _ptr(status), _ptr(waited_cycles), _stream(stream)),
           "fopd_selftest_bounded_wait")


def fopd_loss_finalize(loss_acc, acc, w, B: int, p: fopd_params, loss_out, *, per_sample_loss=None,
                       stream=None):
    _check(lib().fopd_loss_finalize(_ptr(loss_acc), _ptr(acc), _ptr(w), B, p, _ptr(per_sample_loss),
                                    _ptr(loss_out), _stream(stream)),
           "fopd_loss_finalize")


def fopd_row_divergence(first, second, mask, sample_id, B: int, acc, *, kl=None, entropy=None, vocab=None,
                        status=None, stream=None):
    assert first.dtype == second.dtype and first.shape == second.shape and first.stride() == second.stride()
    n = first.shape[0]
    _check(lib().fopd_row_divergence(_ptr(first), _ptr(second), _ptr(mask), _ptr(sample_id), n,
                                     vocab or first.shape[1], first.stride(0) if n > 1 else first.shape[1],
                                     FOPD_BF16 if first.dtype == torch.bfloat16 else FOPD_F32, B, _ptr(kl),
                                     _ptr(entropy), _ptr(acc), _ptr(status), _stream(stream)),
           "fopd_row_divergence")


def fopd_supervision_drift(acc, seq_len, B: int, *, d_sup=None, m_sup=None, mean_entropy=None, stream=None):
    _check(lib().fopd_supervision_drift(_ptr(acc), _ptr(seq_len), B, _ptr(d_sup), _ptr(m_sup), _ptr(mean_entropy),
                                        _stream(stream)), "fopd_supervision_drift")


def fopd_refresh_decision(f, m_roll, m_sup, B: int, kappa_f, kappa_roll, kappa_sup, steps_since_refresh: int,
                          min_interval: int, decision, *, means=None, stream=None):
    _check(lib().fopd_refresh_decision(_ptr(f), _ptr(m_roll), _ptr(m_sup), B, float(kappa_f), float(kappa_roll),
                                       float(kappa_sup), int(steps_since_refresh), int(min_interval), _ptr(means),
                                       _ptr(decision), _stream(stream)), "fopd_refresh_decision")


def fopd_shard_stats(shard: Chunk, vocab_offset: int, vocab_total: int, partial, *, stream=None):
    """Partial sums [n_rows, 8] of the columns [vocab_offset, vocab_offset + W) held in ``shard``."""
    c = shard.c_struct()
    assert partial.dtype == torch.float32 and partial.is_contiguous() and partial.numel() == 8 * c.n_rows
    _check(lib().fopd_shard_stats(ctypes.byref(c), int(vocab_offset), int(vocab_total), _ptr(partial),
                                  _stream(stream)), "fopd_shard_stats")


def fopd_shard_merge(partials, behav_logprob, tokens, mask, sample_id, vocab_total: int, B: int, acc, row_ws, *,
                     lp_s=None, lp_t=None, kl=None, ratio=None, status=None, stream=None):
    """Merge of all parts ([n_parts, n_rows, 8]) into the row statistics and the per-sample sums."""
    n = tokens.numel()
    assert partials.dtype == torch.float32 and partials.is_contiguous() and partials.dim() == 3
    assert partials.shape[1] == n and partials.shape[2] == 8
    rows = fopd_chunk(None, None, behav_logprob.data_ptr(), tokens.data_ptr(), mask.data_ptr(),
                      sample_id.data_ptr(), n, int(vocab_total), int(vocab_total), FOPD_F32, LOSS_FULL_KL)
    _check(lib().fopd_shard_merge(_ptr(partials), partials.shape[0], ctypes.byref(rows), B, _ptr(lp_s), _ptr(lp_t),
                                  _ptr(kl), _ptr(ratio), _ptr(row_ws), _ptr(acc), _ptr(status), _stream(stream)),
           "fopd_shard_merge")


def fopd_shard_loss_fwd_bwd(shard: Chunk, vocab_offset: int, vocab_total: int, B: int, coef, row_ws,
                            p: fopd_params, dlogits, *, loss_acc=None, stream=None):
    c = shard.c_struct()
    assert dlogits.dtype == shard.student.dtype and dlogits.stride() == shard.student.stride()
    _check(lib().fopd_shard_loss_fwd_bwd(ctypes.byref(c), int(vocab_offset), int(vocab_total), B, _ptr(coef),
                                         _ptr(row_ws), p, _ptr(dlogits), _ptr(loss_acc), _stream(stream)),
           "fopd_shard_loss_fwd_bwd")


def _dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return FOPD_BF16
    assert t.dtype == torch.float32, t.dtype
    return FOPD_F32


def _flat(t, dtype, n):
    """An array of n elements as the library takes it: contiguous, on the device of the call's logits."""
    return t.dtype == dtype and t.numel() == n and t.is_contiguous()


def _out(t, dtype, n, device):
    """Address of an output (or of None)."""
    if t is None:
        return None
    assert _flat(t, dtype, n) and t.device == device
    return t.data_ptr()


def _status_word(status, device):
    if status is None:
        return None
    assert status.dtype == torch.int32 and status.numel() >= 1 and status.device == device
    return status.data_ptr()


def _on_current_device(t):
    """The library launches on the current device."""
    assert t.is_cuda and t.get_device() == torch._C._cuda_getDevice(), t.device


def fopd_draw_tokens(logits, uniform, tokens, *, logprob=None, temperature=1.0, vocab=None, status=None, stream=None):
    """One token from each row of ``logits`` [n, V] by the given fp64 numbers ``uniform`` [n]: the
    inverse of the distribution function of softmax(logits / temperature) (temperature 0: the best
    token).  ``tokens`` int32 [n], ``logprob`` fp32 [n] or None."""
    _on_current_device(logits)
    n, cols = logits.shape
    pitch, unit = logits.stride()
    dev, bf16 = logits.device, logits.dtype == torch.bfloat16
    assert (unit == 1 or cols <= 1) and (bf16 or logits.dtype == torch.float32)
    assert _flat(uniform, torch.float64, n) and uniform.device == dev
    assert vocab is None or 0 < vocab <= cols
    if n == 1:
        pitch = (cols + 7) // 8 * 8
    _check(lib().fopd_draw_tokens(logits.data_ptr(), uniform.data_ptr(), n, vocab or cols, pitch,
                                  FOPD_BF16 if bf16 else FOPD_F32, temperature, _out(tokens, torch.int32, n, dev),
                                  _out(logprob, torch.float32, n, dev), _status_word(status, dev), _stream(stream)),
           "fopd_draw_tokens")


def fopd_verify_draft(target, draft, draft_tokens, uniform, tokens, *, n_draft=None, logprob=None, mask=None,
                      n_accepted=None, temperature=1.0, draft_temperature=1.0, vocab=None, status=None, stream=None):
    """Verification of drafted tokens (see ``fopd_verify_draft`` in fopd.h): ``target`` [B, K + 1, V],
    ``draft`` [B, K, V] or None (certain drafts), ``draft_tokens`` int32 [B, K], ``uniform`` fp64
    [B, K + 1], ``n_draft`` int32 [B] or None.  Outputs ``tokens`` int32, ``logprob`` fp32 and ``mask``
    uint8 [B, K + 1], ``n_accepted`` int32 [B]; all but the first may be None."""
    _on_current_device(target)
    B, W, cols = target.shape
    seq, row, unit = target.stride()
    K, dev, bf16 = W - 1, target.device, target.dtype == torch.bfloat16
    assert (unit == 1 or cols <= 1) and (bf16 or target.dtype == torch.float32)
    assert _flat(draft_tokens, torch.int32, B * K) and _flat(uniform, torch.float64, B * W)
    assert draft_tokens.device == dev and uniform.device == dev
    draft_at, dseq, drow = None, 0, 0
    if draft is not None:
        assert draft.shape == (B, K, cols) and draft.dtype == target.dtype and draft.device == dev
        draft_at = draft.data_ptr()
        dseq, drow, unit = draft.stride()
        assert unit == 1 or cols <= 1
    assert vocab is None or 0 < vocab <= cols
    d = fopd_draft(target.data_ptr(), draft_at, draft_tokens.data_ptr(), _out(n_draft, torch.int32, B, dev),
                   uniform.data_ptr(), vocab or cols, seq, row, dseq, drow, temperature, draft_temperature, B, K,
                   FOPD_BF16 if bf16 else FOPD_F32)
    _check(lib().fopd_verify_draft(ctypes.byref(d), _out(tokens, torch.int32, B * W, dev),
                                   _out(logprob, torch.float32, B * W, dev), _out(mask, torch.uint8, B * W, dev),
                                   _out(n_accepted, torch.int32, B, dev), _status_word(status, dev), _stream(stream)),
           "fopd_verify_draft")


def _as_rows(t: torch.Tensor):
    """(rows, cols, pitch) under which the elements of ``t`` lie in memory, in any order; None if they do not."""
    dims = sorted((st, n) for n, st in zip(t.shape, t.stride()) if n != 1)
    if t.numel() == 0:
        return 0, 0, 0
    cols = 1
    while dims and dims[0][0] == cols:
        cols *= dims.pop(0)[1]
    if not dims:
        return 1, cols, cols
    pitch, rows = dims[0][0], 1
    while dims and dims[0][0] == pitch * rows:
        rows *= dims.pop(0)[1]
    return (rows, cols, pitch) if not dims and pitch >= cols else None


class GradientList:
    """The tensors of one fopd_grad_* call, marshalled once: keep it as long as the tensors keep their
    memory (it holds them).  bf16 and fp32, mixed; dense in any order of dimensions, or rows at a pitch.
    ``outs``: where the scaled values go (same shapes, types and strides); None: in place."""

    def __init__(self, tensors, outs=None):
        self.tensors, self.outs = list(tensors), None if outs is None else list(outs)
        assert self.outs is None or len(self.outs) == len(self.tensors)
        self.n = len(self.tensors)
        self.array = (fopd_tensor * max(1, self.n))()
        self.device = self.tensors[0].device if self.n else None
        for i, t in enumerate(self.tensors):
            _on_current_device(t)
            layout = (1, t.numel(), t.numel()) if t.is_contiguous() else _as_rows(t)
            assert layout is not None, f"tensor {i}: strides {t.stride()} of shape {tuple(t.shape)}"
            o = None if self.outs is None else self.outs[i]
            assert o is None or (o.shape == t.shape and o.dtype == t.dtype and o.device == t.device and
                                 ((o.is_contiguous() and t.is_contiguous()) or o.stride() == t.stride()))
            assert self.device == t.device
            self.array[i] = fopd_tensor(t.data_ptr(), None if o is None else o.data_ptr(), *layout, _dtype(t), 0)


def grad_workspace(device) -> torch.Tensor:
    """The fopd_grad_* workspace of one set: fp64, zeroed."""
    return torch.zeros(GRAD_WS, dtype=torch.float64, device=device)


def _grad_args(grads, ws):
    assert ws.dtype == torch.float64 and ws.numel() >= GRAD_WS and ws.is_contiguous()
    _on_current_device(ws)
    assert grads.device is None or grads.device == ws.device
    return ws.device


def _scalar(t, device):
    if t is None:
        return None
    assert t.dtype == torch.float32 and t.numel() >= 1 and t.device == device
    return t.data_ptr()


def fopd_grad_norm(grads: GradientList, ws, *, norm=None, status=None, stream=None):
    """ws[0] += sum of squares; ``norm`` fp32 [1] = sqrt(ws[0])."""
    dev = _grad_args(grads, ws)
    _check(lib().fopd_grad_norm(grads.array, grads.n, ws.data_ptr(), _scalar(norm, dev), _status_word(status, dev),
                                _stream(stream)), "fopd_grad_norm")


def fopd_grad_scale(grads: GradientList, ws, max_norm, *, norm=None, coef=None, status=None, stream=None):
    """Every element times min(1, max_norm / sqrt(ws[0])), into ``outs`` or in place."""
    dev = _grad_args(grads, ws)
    _check(lib().fopd_grad_scale(grads.array, grads.n, ws.data_ptr(), max_norm, _scalar(norm, dev),
                                 _scalar(coef, dev), _status_word(status, dev), _stream(stream)), "fopd_grad_scale")


def fopd_grad_clip(grads: GradientList, max_norm, ws, *, norm=None, coef=None, status=None, stream=None):
    """Norm of the whole set and scaling in one call."""
    dev = _grad_args(grads, ws)
    _check(lib().fopd_grad_clip(grads.array, grads.n, ws.data_ptr(), max_norm, _scalar(norm, dev),
                                _scalar(coef, dev), _status_word(status, dev), _stream(stream)), "fopd_grad_clip")


def _row_pitch(t, per=8):
    """Pitch of a matrix whose rows lie whole in memory (a single row: any that the library takes)."""
    rows, cols = t.shape
    assert t.stride(1) == 1 or cols <= 1
    return t.stride(0) if rows > 1 else -(-cols // per) * per


def _head(hidden, weight, tokens, mask):
    _on_current_device(hidden)
    (n, dim), dev = hidden.shape, hidden.device
    assert weight.dim() == 2 and weight.shape[1] == dim and weight.device == dev
    assert hidden.dtype == torch.bfloat16 and weight.dtype == torch.bfloat16
    assert _flat(tokens, torch.int32, n) and tokens.device == dev
    return fopd_head(hidden.data_ptr(), weight.data_ptr(), tokens.data_ptr(), _out(mask, torch.uint8, n, dev), n,
                     weight.shape[0], dim, _row_pitch(hidden), _row_pitch(weight), FOPD_BF16, 0)


def fopd_head_logprob(hidden, weight, tokens, logprob, *, lse=None, mask=None, status=None, stream=None):
    """Log-probs of ``tokens`` int32 [n] under softmax(hidden weight^T) without the logits: ``hidden`` bf16 [n, D],
    ``weight`` bf16 [V, D] -> ``logprob``, ``lse`` fp32 [n] (the latter may be None).  ``mask`` uint8 [n] or None: rows
    with 0 are not read and get 0."""
    h, n, dev = _head(hidden, weight, tokens, mask), hidden.shape[0], hidden.device
    assert logprob is not None
    _check(lib().fopd_head_logprob(ctypes.byref(h), _out(logprob, torch.float32, n, dev), _out(lse, torch.float32, n, dev),
                                   _status_word(status, dev), _stream(stream)), "fopd_head_logprob")


def fopd_head_grad(hidden, weight, tokens, logprob, lse, coef, *, d_hidden=None, d_weight=None, add_d_weight=False, mask=None,
                   status=None, stream=None):
    """Gradient of -sum coef logprob: ``d_hidden`` bf16 [n, D] and ``d_weight`` bf16 or fp32 [V, D] (either may be None; the
    latter is added to with ``add_d_weight``), from the ``logprob`` and ``lse`` that fopd_head_logprob gave."""
    h, (n, dim), dev = _head(hidden, weight, tokens, mask), hidden.shape, hidden.device
    for t in (logprob, lse, coef):
        assert _flat(t, torch.float32, n) and t.device == dev
    assert d_hidden is None or (d_hidden.shape == hidden.shape and d_hidden.dtype == torch.bfloat16 and d_hidden.device == dev)
    assert d_weight is None or (d_weight.shape == weight.shape and d_weight.device == dev)
    _check(lib().fopd_head_grad(ctypes.byref(h), logprob.data_ptr(), lse.data_ptr(), coef.data_ptr(), _ptr(d_hidden),
                                0 if d_hidden is None else _row_pitch(d_hidden), _ptr(d_weight),
                                0 if d_weight is None else _row_pitch(d_weight), FOPD_BF16 if d_weight is None else _dtype(d_weight),
                                int(bool(add_d_weight)), _status_word(status, dev), _stream(stream)), "fopd_head_grad")


class MatrixList:
    """The matrices of an fopd_orthogonalise call, marshalled once: keep it as long as they keep their memory (it holds them).
    bf16 and fp32, mixed; the last two dimensions are a matrix's rows and columns, those before them count matrices.  Rows lie
    whole in memory, or columns do (a transposed matrix: the result is transposed as well).  ``outs``: where the results go (same
    shapes, bf16 or fp32, same order of dimensions in memory); None: in place.  ``scales``: of the results, one per tensor."""

    def __init__(self, tensors, outs=None, scales=None):
        self.tensors, self.outs = list(tensors), None if outs is None else list(outs)
        scales = [1.0] * len(self.tensors) if scales is None else [float(s) for s in scales]
        assert len(scales) == len(self.tensors) and (self.outs is None or len(self.outs) == len(self.tensors))
        self.device = self.tensors[0].device if self.tensors else None
        items = []
        for i, t in enumerate(self.tensors):
            o = t if self.outs is None else self.outs[i]
            _on_current_device(t)
            assert t.device == self.device == o.device and t.dim() >= 2 and o.shape == t.shape, i
            t, o = t.detach(), o.detach()
            if t.shape[-1] > 1 and t.stride(-1) != 1:  # columns whole: the transposed matrix
                t, o = t.mT, o.mT
            rows, cols = t.shape[-2:]
            for x in (t, o):
                assert cols <= 1 or x.stride(-1) == 1, f"matrix {i}: strides {x.stride()} of shape {tuple(x.shape)}"
            if t.numel() == 0:
                continue
            # (of a single column the pitch is what counts, of a single row nothing)
            pitches = [x.stride(-2) if rows > 1 else cols for x in (t, o)]
            lead = [()]
            for n in t.shape[:-2]:
                lead = [k + (j,) for k in lead for j in range(n)]
            for k in lead:
                at = [x.data_ptr() + x.element_size() * sum(a * b for a, b in zip(k, x.stride())) for x in (t, o)]
                items.append(fopd_matrix(at[0], at[1], rows, cols, pitches[0], pitches[1], scales[i], _dtype(t), _dtype(o), 0))
        self.n = len(items)
        self.array = (fopd_matrix * max(1, self.n))(*items)


NEWTON_SCHULZ_COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5


def fopd_orthogonalise(matrices: MatrixList, *, coefficients=NEWTON_SCHULZ_COEFFICIENTS, eps=1e-7, status=None, stream=None):
    """Every matrix of the list through the Newton-Schulz steps of ``coefficients`` (a, b, c): out = scale times its orthogonal
    factor, nearly (see ``fopd_orthogonalise`` in fopd.h)."""
    flat = [float(x) for step in coefficients for x in step]
    assert len(flat) == 3 * len(coefficients)
    dev = matrices.device
    if dev is not None:
        assert dev.index == torch._C._cuda_getDevice(), dev
    _check(lib().fopd_orthogonalise(matrices.array, matrices.n, (ctypes.c_float * max(1, len(flat)))(*flat), len(coefficients), eps,
                                    None if dev is None else _status_word(status, dev), _stream(stream)), "fopd_orthogonalise")


def fopd_check_status(status, stream=None) -> int:
    """Synchronises the stream and returns the device status bits (0 = clean)."""
    bits = ctypes.c_int32(0)
    rc = lib().fopd_check_status(_ptr(status), ctypes.byref(bits), _stream(stream))
    if rc not in (0, -8):
        raise FopdError(rc, "fopd_check_status")
    return int(bits.value)


def _chunk_array(chunks):
    arr = (fopd_chunk * len(chunks))()
    for j, ch in enumerate(chunks):
        arr[j] = ch.c_struct()
    return arr


def fopd_step_host_workspace_bytes(chunks, B: int, resident: bool) -> int:
    """Device workspace size fopd_step_host needs for these HOST chunks."""
    return int(lib().fopd_step_host_workspace_bytes(_chunk_array(chunks), len(chunks), B, int(resident)))


def fopd_step_host(chunks, B: int, staleness, seq_len, d_sup, p: fopd_params, dlogits, workspace, *,
                   stream=None) -> dict:
    """Whole batch from HOST tensors (``chunks`` hold CPU tensors, ideally pinned;
    ``dlogits`` is a list of CPU tensors receiving the gradients).  Returns the
    per-sample outputs as CPU tensors plus the scalar loss and status bits."""
    arr = _chunk_array(chunks)
    z = lambda n: torch.zeros(n, dtype=torch.float32)
    res = dict(f=z(B), w=z(B), d_roll=z(B), l_distill=z(B), m_align=z(B), per_sample_loss=z(B),
               buffer_means=z(2), loss=z(1), status_bits=torch.zeros(1, dtype=torch.int32),
               copied_bytes=torch.zeros(2, dtype=torch.int64))
    outs = fopd_host_outputs(*[res[n].data_ptr() for n, _ in fopd_host_outputs._fields_])
    dl = (ctypes.c_void_p * len(dlogits))(*[d.data_ptr() for d in dlogits])
    rc = lib().fopd_step_host(arr, len(chunks), B, _ptr(staleness), _ptr(seq_len), _ptr(d_sup), p, dl,
                              ctypes.byref(outs), _ptr(workspace), workspace.numel() * workspace.element_size(),
                              _stream(stream))
    if rc not in (0, -8):
        raise FopdError(rc, "fopd_step_host")
    return res
